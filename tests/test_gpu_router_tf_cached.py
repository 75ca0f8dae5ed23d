"""The router G over new tokens with the earlier ones in the 8-bit cache
(readme_router_tf_cached), step by step: prompts, pieces of prompts, decode
steps and empty turns of several requests.

Each stage is checked from the GPU's own input of that stage, with the bounds
of the uncached router's stages; between q, k, v and o stand the cache's oracle
(codes and scales exactly) and its attention (the bound of the attention alone).
"""
import numpy as np
import pytest
import torch

from oracle import kv_cache as ok
from oracle import router_tf as R
from paper_2410_19123_amd import workloads as wl
from tests._util import from_dev, to_dev
from tests.test_gpu_kv import KT, Cache, _i32, _offsets
from tests.test_gpu_router_tf import HD, _abs_sum, _ulps

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def _near(got, ref, what):
    """At most one bf16 ulp (a step of few rows is too small for a share of
    equal elements)."""
    assert _ulps(got, ref).max() <= 1, what


def _gemm_near(got, ref, scale, what):
    """bf16 of an fp32 sum: the output's rounding and 2^-16 of the sum of
    magnitudes."""
    err = np.abs(R._f(got) - ref)
    assert np.all(err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * scale), what


class Router:
    def __init__(self, shape, seed):
        L = _lib()
        self.shape, self.w = shape, wl.make_router_tf(shape, seed)
        self.dw = {n: to_dev(x) for n, x in self.w.items() if x is not None}
        self.packed = L.readme_router_tf_pack(*(self.dw[n] for n in ("wq", "wk", "wv", "wo", "w1",
                                                                     "w3", "w2")))

    def step(self, c, tokens, new, lens):
        """(ids, logits, regions) of one call over cache c."""
        L, s = _lib(), self.shape
        T = len(tokens)
        logits = torch.empty(T, s.E, dtype=torch.float32, device="cuda:0")
        ids, logits, ws = L.readme_router_tf_cached(
            KT[c.kt], to_dev(tokens), _i32(_offsets(new)), _i32(lens), *c.args(), self.dw["emb"],
            self.packed, s.F, self.dw["w_router"], logits=logits)
        g = {n: from_dev(L.router_tf_region(ws, T, s.D, s.F, n)) for n in L.RTF_REGIONS}
        return from_dev(ids), from_dev(logits), g


def _positions(new, lens):
    return np.concatenate([np.arange(ln - n, ln) for n, ln in zip(new, lens)]).astype(np.int64)


def _check_projections(w, tokens, pos, g):
    D = w["wq"].shape[0]
    assert np.array_equal(g["POS"], pos)
    assert np.array_equal(g["OFFS"], [0, len(tokens)])
    _near(g["A"], R.rmsnorm_bf16(R.embed(tokens.astype(np.int64), w["emb"])), "a")
    af = R._f(g["A"])
    _gemm_near(g["QKV"][:, 2 * D:], af @ R._f(w["wv"]).T, _abs_sum(g["A"], w["wv"]), "v")
    for what, wn, got in (("q", "wq", g["QKV"][:, :D]), ("k", "wk", g["QKV"][:, D:2 * D])):
        ref = R.rope(R.bf16(af @ R._f(w[wn]).T), pos)
        sc = _abs_sum(g["A"], w[wn]).reshape(-1, D // HD, 2, 64)
        gf, rf = R._f(got).reshape(sc.shape), R._f(ref).reshape(sc.shape)
        norm = np.sqrt((rf ** 2).sum(axis=2, keepdims=True))
        assert np.all(np.abs(gf - rf) <= 2.0 ** -7 * norm + 2.0 ** -16 * sc.sum(axis=2, keepdims=True)), what


def _check_attention(c, new, lens, g, rows=None):
    """The rows of the first `rows` requests (all of them if None)."""
    D = g["O"].shape[1]
    n = len(new) if rows is None else rows
    T = int(sum(new[:n]))
    q = R._f(g["QKV"][:T, :D]).astype(np.float64).reshape(T, -1, HD)
    ref, vmax, zabs = ok.attention(c.ref, q, _offsets(new[:n]), lens[:n], c.table[:n],
                                   float(np.float32(HD ** -0.5)))
    delta = (HD + 8) * 2.0 ** -24 * zabs + 2.0 ** -18
    tol = 2.0 ** -8 * np.abs(ref) + ((2.0 ** -11 + 2 * delta) * vmax)[..., None]
    err = np.abs(R._f(g["O"][:T]).reshape(T, -1, HD) - ref)
    assert (err <= tol).all(), float((err - tol).max())


def _check_rest(w, tokens, ids, logits, g):
    from oracle import oracle as O
    F = w["w1"].shape[0]
    x0 = R.embed(tokens.astype(np.int64), w["emb"])
    of = R._f(g["O"])
    x1 = x0.astype(np.float64) + of @ R._f(w["wo"]).T
    b1 = np.abs(x0) + np.abs(of) @ np.abs(R._f(w["wo"])).T
    r = 1.0 / np.sqrt((x1 ** 2).mean(axis=1, keepdims=True) + R.EPS)
    _gemm_near(g["M"], x1 * r, r * b1, "m")
    mf = R._f(g["M"])
    gt, up = mf @ R._f(w["w1"]).T, mf @ R._f(w["w3"]).T
    sc = 1.1 * np.abs(up) * _abs_sum(g["M"], w["w1"]) + np.abs(gt) * _abs_sum(g["M"], w["w3"])
    _gemm_near(g["H"][:, :F], R.mlp_hidden(g["M"], w["w1"], w["w3"]), sc, "h")
    hf = R._f(g["H"][:, :F])
    bound = b1 + np.abs(hf) @ np.abs(R._f(w["w2"])).T
    err = np.abs(g["X"].astype(np.float64) - (x1 + hf @ R._f(w["w2"]).T))
    assert np.all(err <= 2.0 ** -16 * bound)
    _near(g["FEAT"], R.rmsnorm_bf16(g["X"]), "f")
    ids_ref, logits_ref = O.route(g["FEAT"], w["w_router"], None)
    assert np.array_equal(ids, ids_ref) and np.array_equal(logits, logits_ref)


def _oracle_write(c, new, lens, g):
    D = g["O"].shape[1]
    k, v = (R._f(g["QKV"][:, i * D:(i + 1) * D]).astype(np.float64).reshape(len(g["O"]), -1, HD)
            for i in (1, 2))
    ok.write(c.kt, c.ref, k, v, _offsets(new), lens, c.table)
    np.testing.assert_array_equal(c.scales.cpu().numpy(), c.ref["scales"])
    # Codes by value: e4m3 has a zero of either sign
    np.testing.assert_array_equal(ok.from_bytes(c.kt, c.codes.cpu().numpy(), HD), c.ref["codes"])


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
@pytest.mark.parametrize("D", [128, 256])
def test_steps_of_a_batch(oracle_mod, kt, D):
    shape = wl.RouterShape(D=D, F=192, V=1000, E=5)
    r = Router(shape, 3)
    c = Cache(kt, 4, D // HD, HD, 4, seed=40)
    rng = np.random.default_rng(41)
    lens = np.zeros(4, np.int64)
    for new in ([70, 0, 130, 1],       # prompts
                [1, 33, 0, 1],         # a late one beside decode steps
                [1, 1, 1, 1], [60, 1, 2, 0], [0, 0, 1, 0]):
        lens = lens + new
        tokens = rng.integers(0, shape.V, int(sum(new))).astype(np.int32)
        if len(tokens) > 60:
            tokens[5] = -1             # outside the vocabulary: embeds as zeros
        ids, logits, g = r.step(c, tokens, new, lens)
        _check_projections(r.w, tokens, _positions(new, lens), g)
        _oracle_write(c, new, lens, g)
        _check_attention(c, new, lens, g)
        _check_rest(r.w, tokens, ids, logits, g)


def test_a_request_batch_of_prompts(oracle_mod):
    """8192 tokens at the paper's width, where the block passes its own tiles:
    the first requests' rows."""
    shape = wl.RouterShape(D=512, F=512, V=2000, E=8)
    r = Router(shape, 4)
    new = [32] * 256
    c = Cache("i8", 256, 4, HD, 1, seed=42)
    tokens = np.random.default_rng(43).integers(0, shape.V, 8192).astype(np.int32)
    ids, logits, g = r.step(c, tokens, new, new)
    assert np.array_equal(g["POS"], _positions(new, new))
    n = 96
    head = {k: (v if k in ("POS", "OFFS") else v[:n]) for k, v in g.items()}
    few = dict(head, POS=g["POS"][:n], OFFS=np.array([0, n]))
    _check_projections(r.w, tokens[:n], _positions(new[:3], new[:3]), few)
    D = shape.D
    k, v = (R._f(g["QKV"][:n, i * D:(i + 1) * D]).astype(np.float64).reshape(n, 4, HD) for i in (1, 2))
    ok.write("i8", c.ref, k, v, _offsets(new[:3]), new[:3], c.table[:3])
    _check_attention(c, new, new, g, rows=3)
    _check_rest(r.w, tokens[:n], ids[:n], logits[:n], few)


def test_keys_are_the_uncached_routers():
    """One call over whole prompts: q, k, v as readme_router_tf leaves them."""
    L = _lib()
    shape = wl.RouterShape(D=256, F=64, V=300, E=4)
    r = Router(shape, 5)
    new = [40, 1, 90]
    c = Cache("i8", 3, 2, HD, 2, seed=44)
    tokens = np.random.default_rng(45).integers(0, shape.V, 131).astype(np.int32)
    _, _, g = r.step(c, tokens, new, new)
    _, _, ws = L.readme_router_tf(to_dev(tokens), _i32(_offsets(new)), r.dw["emb"], r.packed, shape.F,
                                  r.dw["w_router"])
    for n in ("A", "QKV", "POS"):
        assert np.array_equal(from_dev(L.router_tf_region(ws, 131, 256, 64, n)), g[n]), n


def test_a_captured_decode_step_replays():
    """A decode step captured once and replayed as the requests grow, against
    eager calls on a second cache."""
    L = _lib()
    shape = wl.RouterShape(D=256, F=128, V=500, E=6)
    r = Router(shape, 6)
    rng = np.random.default_rng(46)
    a, b = (Cache("e4m3", 3, 2, HD, 3, seed=47) for _ in range(2))
    start = [62, 5, 127]
    tokens = rng.integers(0, shape.V, sum(start)).astype(np.int32)
    for c in (a, b):
        r.step(c, tokens, start, start)
    off, tok, lens = _i32([0, 1, 2, 3]), _i32([0, 0, 0]), _i32(start)
    table = _i32(a.table)
    ids = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    logits = torch.zeros(3, shape.E, dtype=torch.float32, device="cuda:0")
    ws = torch.zeros(L.readme_router_tf_cached_workspace_bytes(3, 3, 256, 128, 3), dtype=torch.uint8,
                     device="cuda:0")

    def call():
        L.readme_router_tf_cached(KT["e4m3"], tok, off, lens, table, a.codes, a.scales, r.dw["emb"],
                                  r.packed, 128, r.dw["w_router"], expert_ids=ids, logits=logits,
                                  workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for k in range(1, 6):
        t = rng.integers(0, shape.V, 3).astype(np.int32)
        now = [x + k for x in start]
        tok.copy_(torch.from_numpy(t))
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        e_ids, e_logits, _ = r.step(b, t, [1, 1, 1], now)
        assert np.array_equal(from_dev(ids), e_ids) and np.array_equal(from_dev(logits), e_logits)
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
