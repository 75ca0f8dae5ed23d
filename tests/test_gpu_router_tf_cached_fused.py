"""The router over new tokens at the paper's width and batches where its fused
head and tail run (D = 512, from 1800 + 1.4 F tokens): positions come from the
cache's lengths, so requests with earlier tokens in the cache, each with its own
count, are what these tests hold."""
import numpy as np
import pytest
import torch

from paper_2410_19123_amd import workloads as wl
from tests._util import from_dev
from tests.test_gpu_kv import KT, Cache, _i32, _offsets
from tests.test_gpu_router_tf_cached import (HD, Router, _check_attention, _check_projections,
                                             _check_rest, _lib, _oracle_write, _positions)

pytestmark = pytest.mark.gpu

SHAPE = wl.RouterShape(D=512, F=320, V=3000, E=8)
R = 70


def _fused(T):
    return T >= 1800 + SHAPE.F * 7 // 5


def _pieces(rng, calls):
    """New rows and lengths of each call: every request at its own position, some
    without rows, one begun anew in each call, with rows before its position 0."""
    lens = np.zeros(R, np.int64)
    for k in range(calls):
        new = rng.integers(20, 60, R)
        new[rng.integers(0, R - 1, 3)] = 0
        lens = lens + new
        again = 5 + k
        lens[again] = max(0, int(new[again]) - 3)
        assert _fused(int(new.sum()))
        yield new, lens.copy()


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
def test_pieces_of_a_batch(oracle_mod, kt):
    """Prompts in two pieces, every stage on every row."""
    r = Router(SHAPE, 7)
    c = Cache(kt, R, SHAPE.D // HD, HD, 2, seed=90)
    rng = np.random.default_rng(91)
    for new, lens in _pieces(rng, 2):
        tokens = rng.integers(0, SHAPE.V, int(new.sum())).astype(np.int32)
        ids, logits, g = r.step(c, tokens, new, lens)
        pos = _positions(new, lens)
        assert (pos < 0).any()
        _check_projections(r.w, tokens, pos, g)
        _oracle_write(c, new, lens, g)
        _check_attention(c, new, lens, g)
        _check_rest(r.w, tokens, ids, logits, g)


def test_a_captured_piece_replays():
    """One call captured and replayed as the requests grow, against eager calls
    on a second cache."""
    L = _lib()
    r = Router(SHAPE, 8)
    a, b = (Cache("i8", R, SHAPE.D // HD, HD, 4, seed=92) for _ in range(2))
    rng = np.random.default_rng(93)
    new = rng.integers(30, 50, R)
    T = int(new.sum())
    assert _fused(T)
    off, lens = _i32(_offsets(new)), _i32(new)
    tok = torch.zeros(T, dtype=torch.int32, device="cuda:0")
    args = a.args()
    ids = torch.zeros(T, dtype=torch.int32, device="cuda:0")
    logits = torch.zeros(T, SHAPE.E, dtype=torch.float32, device="cuda:0")
    ws = torch.zeros(L.readme_router_tf_cached_workspace_bytes(T, R, SHAPE.D, SHAPE.F, 4),
                     dtype=torch.uint8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.readme_router_tf_cached(KT["i8"], tok, off, lens, *args, r.dw["emb"], r.packed, SHAPE.F,
                                  r.dw["w_router"], expert_ids=ids, logits=logits, workspace=ws)
    at = np.zeros(R, np.int64)
    for k in range(3):
        at = at + new
        t = rng.integers(0, SHAPE.V, T).astype(np.int32)
        tok.copy_(torch.from_numpy(t))
        lens.copy_(torch.from_numpy(at.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        e_ids, e_logits, _ = r.step(b, t, new, at)
        assert np.array_equal(from_dev(ids), e_ids) and np.array_equal(from_dev(logits), e_logits)
        assert torch.equal(args[1], b.codes) and torch.equal(args[2], b.scales)
