"""Every form of the cache attention against its 64-bit oracle: masks, absent
blocks, queries and scales out of the ordinary, at sizes whose form the library
itself names (tests.kv_forms)."""
import numpy as np
import pytest
import torch

from oracle import kv_cache as ok
from tests.kv_forms import AT_128_ONLY, AT_256_TOO, SIZES, WINDOWS, kind
from tests.test_gpu_kv import KT, Cache, _attend, _i32, _lib, _offsets, _poison_unused, _random_cache

pytestmark = pytest.mark.gpu

TILES = ("tiles/1", "tiles/0")


def _cases(names):
    for n in names:
        yield n, "e4m3", 128
        if n not in AT_128_ONLY:
            yield n, "i8", 64
        if n in AT_256_TOO:
            yield n, "i8", 256


def _cache(name, kt, D, seed=80):
    s = SIZES[name]
    c = s.cache(_random_cache, kt, D, seed)
    _poison_unused(c, s.lens)
    return s, c


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name,kt,D", _cases(SIZES))
def test_every_form(name, kt, D, causal):
    s, c = _cache(name, kt, D)
    assert s.form(D) == kind(name)
    got, _ = _attend(c, s.new, s.lens, s.Hk * s.G, causal, pad=2)
    assert (got[sum(s.new):] == 55).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("name,kt,D", _cases(WINDOWS))
def test_windows(name, kt, D, causal):
    s, c = _cache(name, kt, D)
    assert s.form(D, WINDOWS[name]) == kind(name)
    _attend(c, s.new, s.lens, s.Hk * s.G, causal, WINDOWS[name])


@pytest.mark.parametrize("causal,windowed", [(True, False), (True, True), (False, False)])
@pytest.mark.parametrize("name,kt,D", _cases(TILES))
def test_absent_blocks(name, kt, D, causal, windowed):
    """Blocks absent first, last, between and all, in requests of several."""
    s = SIZES[name]
    c = s.cache(_random_cache, kt, D, 81)
    c.table[0, 0] = -1
    c.table[1, 1] = 1 << 30
    c.table[3, :] = -5
    c.table[5, 2:4] = -1
    c.table[5, 1] = -(1 << 31)
    _poison_unused(c, s.lens)
    got, _ = _attend(c, s.new, s.lens, s.Hk * s.G, causal, WINDOWS[name] if windowed else 0)
    off = _offsets(s.new)
    assert (got[off[3]:off[4]] == 0).all()


@pytest.mark.parametrize("name,kt,D", [("tiles/1", "i8", 64), ("tiles/0", "e4m3", 128), ("tiles/0", "i8", 256)])
def test_peaked_and_flat(name, kt, D):
    """One token takes all of a row, rows of zeros, very large and very small
    rows, beside each other in a tile."""
    s, c = _cache(name, kt, D, 82)
    q = c.rng.standard_normal((sum(s.new), s.Hk * s.G, D))
    kinds = np.arange(q.shape[0] * q.shape[1]).reshape(q.shape[:2]) % 5
    q *= np.choose(kinds, [300.0, 0.0, 1e-30, 1e4, 1.0])[..., None]
    _attend(c, s.new, s.lens, s.Hk * s.G, q=torch.from_numpy(q).bfloat16())
    _attend(c, s.new, s.lens, s.Hk * s.G, q=torch.from_numpy(q).bfloat16(), scale=1e-6, causal=False)


@pytest.mark.parametrize("value,half", [(float("nan"), 0), (float("inf"), 1), (float("nan"), 1)])
@pytest.mark.parametrize("name,kt,D", [("tiles/1", "i8", 64), ("tiles/0", "e4m3", 128)])
def test_scales_that_are_not_finite(name, kt, D, value, half):
    """The rows that see a token of the block are NaN, every other row keeps its
    value (within twice _attend's bound, of the values finite scales give)."""
    L, s = _lib(), SIZES[name]
    c = s.cache(_random_cache, kt, D, 83)
    _poison_unused(c, s.lens)
    H, T, off = s.Hk * s.G, sum(s.new), _offsets(s.new)
    q = torch.from_numpy(c.rng.standard_normal((T, H * D))).bfloat16()
    at = {0: 1, 5: 2, 4: 0}                        # request: block
    for window in (0, WINDOWS[name]):
        run = lambda: L.readme_attention_kv(  # noqa: E731
            KT[kt], q.cuda(), _i32(off), _i32(s.lens), *c.args(), H=H, window=window).float().cpu()
        was, scales = run(), c.scales.clone()
        for r, j in at.items():
            c.scales[int(c.table[r, j]), :, half] = value
        now = run()
        c.scales.copy_(scales)
        sees = torch.zeros(T, dtype=torch.bool)
        for r, j in at.items():
            p = torch.arange(s.lens[r] - s.new[r], s.lens[r])
            lo = torch.clamp(p - window + 1, min=0) if window else torch.zeros_like(p)
            sees[off[r]:off[r + 1]] = torch.clamp(lo, min=64 * j) < torch.clamp(p + 1, max=64 * j + 64)
        assert sees.any() and not sees.all()
        assert torch.isnan(now[sees]).all()
        assert not torch.isnan(was).any()
        _, vmax, zabs = ok.attention(c.ref, q.double().numpy().reshape(T, H, D), off, s.lens, c.table,
                                     D ** -0.5, True, window)
        delta = (D + 8) * 2.0 ** -24 * zabs + 2.0 ** -18
        tol = torch.from_numpy((2.0 ** -11 + 2 * delta) * vmax)[..., None] + \
            2.0 ** -8 * was.view(T, H, D).abs()
        assert ((now - was).view(T, H, D).abs() <= 2 * tol)[~sees].all()


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
@pytest.mark.parametrize("name", TILES)
def test_every_code_value_comes_back(name, kt):
    """The row at position 0 sees one token: it is that token's values."""
    s = SIZES[name]
    c = s.cache(Cache, kt, 256, 84)
    vals = np.arange(-127, 128) if kt == "i8" else ok.e4m3_values()
    vals = np.resize(np.concatenate([vals[np.isfinite(vals)], np.zeros(8)]), 256)
    c.ref["codes"][:, :, 1] = vals
    c.ref["scales"][:] = 1.0
    c.codes.copy_(torch.from_numpy(ok.to_bytes(kt, c.ref["codes"])))
    c.scales.copy_(torch.from_numpy(c.ref["scales"]))
    got, _ = _attend(c, s.new, s.new, s.Hk * s.G)
    first = _offsets(s.new)[:-1][np.array(s.new) > 0]
    np.testing.assert_array_equal(got[first], np.broadcast_to(vals, got[first].shape))


@pytest.mark.parametrize("name", TILES)
def test_slices_of_wider_rows(name):
    """Q and O as slices of wider rows; what lies beside O stays."""
    L, s = _lib(), SIZES[name]
    c = s.cache(_random_cache, "i8", 64, 85)
    W, T = s.Hk * s.G * 64, sum(s.new)
    wide = torch.randn(T, W + 24, device="cuda:0").bfloat16()
    o = torch.full((T, W + 40), 9.0, dtype=torch.bfloat16, device="cuda:0")
    args = (_i32(_offsets(s.new)), _i32(s.lens), *c.args())
    L.readme_attention_kv(0, wide[:, 16:16 + W], *args, H=s.Hk * s.G, o=o[:, 8:8 + W])
    ref = L.readme_attention_kv(0, wide[:, 16:16 + W].contiguous(), *args, H=s.Hk * s.G)
    assert torch.equal(o[:, 8:8 + W], ref)
    assert (o[:, :8] == 9).all() and (o[:, 8 + W:] == 9).all()


@pytest.mark.parametrize("name", SIZES)
def test_captured_forms_follow_the_lengths(name):
    """Captured once, replayed as lengths and rows change, against eager calls
    with a workspace of their own."""
    L, s = _lib(), SIZES[name]
    c = s.cache(_random_cache, "e4m3", 128, 86)
    table, codes, scales = c.args()
    H, T = s.Hk * s.G, sum(s.new)
    off, lens = _i32(_offsets(s.new)), _i32(s.lens)
    q = torch.randn(T, H * 128, device="cuda:0").bfloat16()
    o = torch.empty_like(q)
    ws = torch.empty(L.readme_attention_kv_workspace_bytes(T, len(s.new), H, s.Hk, 128, s.max_blocks),
                     dtype=torch.uint8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.readme_attention_kv(1, q, off, lens, table, codes, scales, H=H, o=o, workspace=ws)
    for now in (s.lens, s.new, s.lens[::-1], [max(s.lens)] * len(s.lens)):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        q.copy_(torch.randn(T, H * 128, device="cuda:0"))
        graph.replay()
        got = o.clone()
        ref = L.readme_attention_kv(1, q, off, lens, table, codes, scales, H=H)
        torch.cuda.synchronize()
        assert torch.equal(got, ref)
