"""readme_attention_kv_tree on the GPU against its 64-bit oracle, at sizes whose
form the library itself names (tests.kv_forms), with the bound that
tests.test_gpu_kv derives."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from tests.kv_forms import SIZES, WINDOWS, Size
from tests.test_gpu_kv import KT, _i32, _offsets, _poison_unused, _random_cache

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def _parents(rng, n, fan=4):
    return [-1] + [int(rng.integers(max(0, i - fan), i)) for i in range(1, n)]


def _masks(rng, new, what="tree"):
    """Python integers, a row each: trees, random bits (rows that see nothing of
    the call among them), nothing at all."""
    out = []
    for n in new:
        if what == "tree":
            out += od.bits(_parents(rng, n)) if n else []
        elif what == "random":
            out += [0 if rng.random() < 0.2 else int.from_bytes(rng.bytes(n // 8 + 1), "little")
                    for _ in range(n)]
        else:
            out += [0] * n
    return out


def _attend(c, new, lens, H, masks, words=None, pos=None, window=0, pad=0, q=None, scale=None):
    L = _lib()
    off, T, D = _offsets(new), sum(new) + pad, c.D
    words = words or max(1, -(-max(new) // 64))
    rows = np.concatenate([od.words(masks, words), np.full((pad, words), -1, np.int64)]) if masks else \
        np.full((pad, words), -1, np.int64)
    tree = torch.from_numpy(rows).cuda()
    if q is None:
        q = torch.from_numpy(c.rng.standard_normal((T, H, D)) * 1.5).bfloat16()
    o = torch.full((T, H * D), 55.0, dtype=torch.bfloat16, device="cuda:0")
    scale = D ** -0.5 if scale is None else scale
    at = None if pos is None else _i32(np.concatenate([pos, np.zeros(pad)]))
    L.readme_attention_kv_tree(KT[c.kt], q.reshape(T, -1).cuda(), _i32(off), _i32(lens), *c.args(), H, tree,
                               at, scale, window, o)
    torch.cuda.synchronize()
    ref, vmax, zabs = od.attention_tree(c.ref, q.double().numpy(), off, lens, c.table, masks + [0] * pad,
                                        float(np.float32(scale)), pos, window, words, 55.0)
    got = o.cpu().double().numpy().reshape(T, H, D)
    delta = (D + 8) * 2.0 ** -24 * zabs + 2.0 ** -18
    tol = 2.0 ** -8 * np.abs(ref) + ((2.0 ** -11 + 2 * delta) * vmax)[..., None]
    err = np.abs(got - ref)
    assert np.isfinite(got).all()
    assert (err <= tol).all(), (err - tol).max()
    assert (got[sum(new):] == 55).all()
    return got, o


def form(s, D, window=0):
    """The form that the library takes: query rows of a pair / waves to a whole
    pair, 0 where shares are dealt."""
    import ctypes
    fn = _lib().load().readme_internal_attention_kv_tree_form
    fn.restype = ctypes.c_int32
    fn.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 4 + [ctypes.c_int64] * 2
    rows, waves = divmod(fn(sum(s.new), len(s.new), s.Hk * s.G, s.Hk, D, s.max_blocks, window), 256)
    return f"{rows}/{waves}"


_FEW, _MORE = [8, 3, 0, 5], [40, 30, 0, 65]
# Sizes named after the form that heads of up to 128 take at them; others of the
# plain call's, which reach the same forms and those of heads of 256.
TREES = {
    "16/1": Size(_FEW, [100, 3, 9, 128], 3, 2, 2), "16/2": Size(_FEW, [300, 2, 9, 191], 3, 2, 5),
    "16/4": Size(_FEW, [600, 64, 9, 450], 2, 3, 10), "16/8": Size(_FEW, [1100, 577, 0, 70], 2, 3, 18),
    "16/0": Size(_FEW, [1100, 64, 2, 450], 2, 2, 66), "32/1": Size(_MORE, [100, 30, 9, 128], 2, 4, 2),
    "32/2": Size(_MORE, [300, 22, 9, 191], 2, 4, 5), "32/4": Size(_MORE, [600, 94, 9, 450], 2, 4, 10),
    "32/8": Size(_MORE, [900, 577, 0, 70], 1, 5, 18), "32/0": Size(_MORE, [900, 64, 2, 450], 2, 1, 66),
    "128/0": Size(_MORE, [900, 64, 2, 450], 1, 3, 66),
    "16/1 of 300": Size([2, 0, 5, 1] * 75, [70, 1, 100, 64] * 75, 2, 2, 2),
    "32/0 of 70": Size([9, 0, 21, 13, 40] * 14, [70, 1, 100, 64, 150] * 14, 1, 2, 70),
}


def _size(name):
    return TREES.get(name) or SIZES[name]


def _sizes():
    for name in TREES:
        yield name, "e4m3", 128
        if " " not in name:
            yield name, "i8", 64
    for name in ("rows/1", "rows/8", "rows/0 of 300", "tiles/1", "tiles/0"):
        yield name, "i8", 128
    for name in ("rows/2", "rows/0", "tiles/1", "tiles/0"):
        yield name, "i8", 256


@pytest.mark.parametrize("name", TREES)
@pytest.mark.parametrize("D", [64, 128])
def test_sizes_take_the_form_they_are_named_after(name, D):
    assert form(TREES[name], D) == name.split()[0]


@pytest.mark.parametrize("what", ["tree", "random", "nothing"])
@pytest.mark.parametrize("name,kt,D", _sizes())
def test_every_form(name, kt, D, what):
    s = _size(name)
    c = s.cache(_random_cache, kt, D, 90)
    _poison_unused(c, s.lens)
    got, _ = _attend(c, s.new, s.lens, s.Hk * s.G, _masks(c.rng, s.new, what), pad=2)
    if what == "nothing":  # rows without earlier tokens see none
        off = _offsets(s.new)
        for r, (n, ln) in enumerate(zip(s.new, s.lens)):
            if ln <= n:
                assert (got[off[r]:off[r + 1]] == 0).all()


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("name,kt,D", [(n, k, d) for n, k, d in _sizes() if n in WINDOWS or n in TREES])
def test_windows(name, kt, D, given):
    """Positions of the stored rows and given ones, below the first row and far
    above it among them."""
    s = _size(name)
    c = s.cache(_random_cache, kt, D, 91)
    _poison_unused(c, s.lens)
    window, pos = WINDOWS.get(name, 45), None
    if given:
        first = np.concatenate([np.full(n, ln - n) for n, ln in zip(s.new, s.lens)])
        pos = first + c.rng.integers(-9, 60, len(first))
        pos[::17] = 2 ** 31 - 1
        pos[5::19] = -2 ** 31
    _attend(c, s.new, s.lens, s.Hk * s.G, _masks(c.rng, s.new), window=window, pos=pos, pad=1)


@pytest.mark.parametrize("new,D", [(5, 64), (40, 128), (70, 256)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31, 2 ** 32 - 3, 2 ** 33, 2 ** 40, 2 ** 63 - 1])
def test_windows_wider_than_every_position_are_none(window, new, D):
    L = _lib()
    c = _random_cache("i8", 2, 2, D, 6, seed=75)
    lens, off = _i32([350, 260]), _i32(_offsets([new] * 2))
    tree = torch.from_numpy(od.words(_masks(c.rng, [new] * 2), 2)).cuda()
    q = torch.randn(2 * new, 4 * D, device="cuda:0").bfloat16()
    for pos in (None, _i32(list(range(345, 345 + 2 * new)))):
        wide = L.readme_attention_kv_tree(0, q, off, lens, *c.args(), 4, tree, pos, window=window)
        assert torch.equal(wide, L.readme_attention_kv_tree(0, q, off, lens, *c.args(), 4, tree, pos))


@pytest.mark.parametrize("D,Hk,G", [(64, 2, 1), (64, 1, 7), (128, 2, 4), (256, 1, 3)])
@pytest.mark.parametrize("new,lens", [
    ([1], [1]), ([8], [517]), ([64, 65, 63], [64, 200, 127]), ([130, 1, 200], [700, 64, 200]),
    ([3, 0, 5, 8, 4, 2], [3, 100, 200, 64, 0, 1]), ([90], [60]), ([600], [650])])
def test_trees(D, Hk, G, new, lens):
    """One word and several, rows before the first token, one row alone."""
    c = _random_cache("i8", len(new), Hk, D, 12, seed=len(new) + D)
    _poison_unused(c, lens)
    _attend(c, new, lens, Hk * G, _masks(c.rng, new), pad=1)
    _attend(c, new, lens, Hk * G, _masks(c.rng, new, "random"), window=30)


def test_fewer_words_than_rows_and_more():
    """Rows past the bits are seen by none; words past the rows mean nothing."""
    c = _random_cache("e4m3", 2, 2, 64, 6, seed=7)
    new, lens = [100, 150], [300, 190]
    masks = [(1 << 200) - 1] * 250
    _attend(c, new, lens, 4, masks, words=1)
    _attend(c, new, lens, 4, masks, words=2)
    _attend(c, new, lens, 4, masks, words=9)


def test_absent_blocks_and_shared_ones():
    for new in ([1] * 5, [40] * 5):
        c = _random_cache("e4m3", 5, 2, 128, 4, seed=20)
        c.table[0, 0] = -1
        c.table[1, 3] = 1 << 20
        c.table[2, 1] = -5
        c.table[3, :] = -1
        c.table[4, :2] = c.table[0, 1]
        lens = [250, 250, 200, 256, 130]
        _poison_unused(c, lens)
        got, _ = _attend(c, new, lens, 4, _masks(c.rng, new, "random"))
        assert (got[3 * new[0]:4 * new[0]] == 0).all()


@pytest.mark.parametrize("new", [5, 90])
def test_bad_scales_reach_only_their_readers(new):
    """A block of drafts whose scale is NaN: rows whose bits name none of its
    tokens keep their values."""
    L = _lib()
    c = _random_cache("i8", 2, 1, 64, 5, seed=24)
    first = 128
    lens, off = _i32([first + new] * 2), _i32(_offsets([new] * 2))
    masks = [1 << (i % 64) if i % 2 else 1 << i for i in range(new)] * 2
    tree = torch.from_numpy(od.words(masks, 2)).cuda()
    q = torch.randn(2 * new, 64, device="cuda:0").bfloat16()
    was = L.readme_attention_kv_tree(0, q, off, lens, *c.args(), 1, tree)
    for block, half in ((2, 0), (2, 1), (1, 0)):
        scales = c.scales.clone()
        c.scales[int(c.table[0, block]), 0, half] = float("nan")
        now = L.readme_attention_kv_tree(0, q, off, lens, *c.args(), 1, tree)
        c.scales.copy_(scales)
        sees = torch.tensor([block == 1 or any((m >> b) & 1 for b in range(0, min(64, new))) for m in masks[:new]],
                            device="cuda:0")
        sees = torch.cat([sees, torch.zeros_like(sees)])
        assert torch.isnan(now[sees].float()).all()
        tol = 2.0 ** -7 * was.float().abs() + 2.0 ** -9 * 127 * float(scales[..., 1].max())
        assert ((now.float() - was.float()).abs() <= tol)[~sees].all()


def test_captured_trees_follow_lengths_and_bits():
    L = _lib()
    for new, mb in (([1, 30, 8], 90), ([1, 40, 200], 90), ([4, 7, 3], 6)):
        c = _random_cache("e4m3", 3, 2, 128, mb, seed=60)
        cache, T, words = c.args(), sum(new), 4
        off, lens, pos = _i32(_offsets(new)), _i32([200, 201, 202]), _i32(range(200, 200 + T))
        q, tree = torch.randn(T, 512, device="cuda:0").bfloat16(), torch.zeros((T, words), dtype=torch.int64,
                                                                                device="cuda:0")
        o = torch.empty_like(q)
        ws = torch.empty(L.readme_attention_kv_tree_workspace_bytes(T, 3, 4, 2, 128, mb), dtype=torch.uint8,
                         device="cuda:0")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            L.readme_attention_kv_tree(1, q, off, lens, *cache, 4, tree, pos, window=150, o=o, workspace=ws)
        for now in ([200, 201, 202], [mb * 64, 230, 1], [0, 0, 0], [330, mb * 64 - 1, 260]):
            lens.copy_(torch.tensor(now, dtype=torch.int32))
            tree.copy_(torch.from_numpy(od.words(_masks(c.rng, new), words)))
            q.copy_(torch.randn(T, 512, device="cuda:0"))
            graph.replay()
            got = o.clone()
            ref = L.readme_attention_kv_tree(1, q, off, lens, *cache, 4, tree, pos, window=150)
            torch.cuda.synchronize()
            assert torch.equal(got, ref), now


def test_two_streams_at_once():
    L = _lib()
    work = []
    for i, (R, new, mb, Hk) in enumerate(((2, 12, 300, 2), (1, 300, 100, 1), (3, 4, 9, 4))):
        c = _random_cache("i8", R, Hk, 128, mb, seed=50 + i)
        T, words = R * new, -(-new // 64)
        q = torch.randn(T, Hk * 4 * 128, device="cuda:0").bfloat16()
        tree = torch.from_numpy(od.words(_masks(c.rng, [new] * R), words)).cuda()
        ws = torch.empty(L.readme_attention_kv_tree_workspace_bytes(T, R, Hk * 4, Hk, 128, mb),
                         dtype=torch.uint8, device="cuda:0")
        work.append((q, _i32(_offsets([new] * R)), _i32([mb * 64 - 5] * R), c.args(), Hk * 4, tree, ws))

    def call(w, o):
        return L.readme_attention_kv_tree(0, w[0], w[1], w[2], *w[3], w[4], w[5], o=o, workspace=w[6])
    alone = [call(w, torch.empty_like(w[0])) for w in work]
    torch.cuda.synchronize()
    outs = [[torch.empty_like(w[0]) for _ in range(4)] for w in work]
    streams = [torch.cuda.Stream() for _ in work]
    for k in range(4):
        for w, o, s in zip(work, outs, streams):
            with torch.cuda.stream(s):
                call(w, o[k])
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(torch.equal(a, x) for x in o)


def test_long_contexts():
    """Work split over the keys and joined: against float64 torch on the GPU."""
    L = _lib()
    Hk, G, D, new, lens = 2, 4, 128, [40, 8, 33], [30000, 20001, 9000]
    rng = np.random.default_rng(33)
    mb = (max(lens) + 63) // 64
    table = _i32(rng.permutation(3 * mb).reshape(3, mb))
    g = torch.Generator(device="cuda:0").manual_seed(3)
    codes = torch.randint(1, 256, (3 * mb, Hk, 2, 64 * D), generator=g, device="cuda:0",
                          dtype=torch.int32).to(torch.uint8)
    scales = torch.rand((3 * mb, Hk, 2), generator=g, device="cuda:0") * 0.02 + 0.01
    q = torch.randn((sum(new), Hk * G * D), generator=g, device="cuda:0").bfloat16()
    masks, off = _masks(rng, new), _offsets(new)
    tree = torch.from_numpy(od.words(masks, 1)).cuda()
    args = (_i32(off), _i32(lens), table, codes, scales, Hk * G, tree)
    o = L.readme_attention_kv_tree(0, q, *args)
    assert torch.equal(o, L.readme_attention_kv_tree(0, q, *args))
    for r, (n, x) in enumerate(zip(new, lens)):
        raw = codes[table[r].long()].double() - 128
        kk = raw[:, :, 0].view(-1, Hk, 2, D // 16, 32, 16).permute(1, 0, 2, 4, 3, 5).reshape(Hk, -1, 64, D)
        vv = raw[:, :, 1].view(-1, Hk, 2, D, 32).permute(1, 0, 2, 4, 3).reshape(Hk, -1, 64, D)
        sc = scales[table[r].long()].double().permute(2, 1, 0)
        kk = (kk * sc[0][..., None, None]).reshape(Hk, -1, D)[:, :x]
        vv = (vv * sc[1][..., None, None]).reshape(Hk, -1, D)[:, :x]
        qq = q[off[r]:off[r + 1]].double().view(n, Hk, G, D).permute(1, 0, 2, 3).reshape(Hk, n * G, D)
        z = torch.matmul(qq, kk.transpose(1, 2).contiguous()) * D ** -0.5
        seen = torch.ones((n, x), dtype=torch.bool)
        for i in range(n):
            for b in range(n):
                seen[i, x - n + b] = bool((masks[off[r] + i] >> b) & 1)
        z.masked_fill_(~seen.cuda().repeat_interleave(G, 0), float("-inf"))
        ref = torch.matmul(torch.softmax(z, -1), vv)
        got = o[off[r]:off[r + 1]].double().view(n, Hk, G, D).permute(1, 0, 2, 3).reshape(Hk, n * G, D)
        vmax = float(vv.abs().max())
        delta = (D + 8) * 2.0 ** -24 * float(qq.abs().max() * kk.abs().max() * D ** 0.5) + 2.0 ** -18
        delta += 2.0 ** -24 * (64 + x / 64)
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -11 + 2 * delta) * vmax
        assert ((got - ref).abs() <= tol).all(), r


def test_python_form_refuses():
    L = _lib()
    c = _random_cache("i8", 1, 2, 64, 2, seed=1)
    q = torch.randn(5, 256, device="cuda:0").bfloat16()
    tree = torch.ones((5, 1), dtype=torch.int64, device="cuda:0")
    at = (_i32([0, 5]), _i32([70]), *c.args())
    for call in (lambda: L.readme_attention_kv_tree(0, q, *at, 4, tree[:4]),
                 lambda: L.readme_attention_kv_tree(0, q, *at, 4, tree.int()),
                 lambda: L.readme_attention_kv_tree(0, q, *at, 4, tree.cpu()),
                 lambda: L.readme_attention_kv_tree(0, q, *at, 4, tree, _i32([1])),
                 lambda: L.readme_attention_kv_tree(0, q.float(), *at, 4, tree),
                 lambda: L.readme_attention_kv_tree(0, q, *at, 3, tree)):
        with pytest.raises(ValueError):
            call()
