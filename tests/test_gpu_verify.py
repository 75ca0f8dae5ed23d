"""readme_verify_drafts on the GPU against its 64-bit oracle: paths, counts and
tokens are equal wherever no comparison is nearer to its border than the order of
fp64 sums."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from tests.test_gpu_kv import _i32, _offsets

pytestmark = pytest.mark.gpu

# Sums of up to 2^18 terms in fp64, in any order, agree to 2^18 2^-53; the chain of
# refusals at a node adds a few of those.
SAFE = 2.0 ** -30


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def _padded(a, dtype, fill=float("nan")):
    """Rows [T][V] on the GPU as a slice of wider rows that begin at 16 bytes."""
    T, V = a.shape
    out = torch.full((T, (V + 7) // 8 * 8 + 8), fill, dtype=dtype, device="cuda:0")
    out[:, :V] = a.to(dtype)
    return out[:, :V]


class Case:
    def __init__(self, new, V, fan=1, kind="given", dtype=torch.float32, seed=0, sharp=1.5):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        T = int(sum(new))
        self.new, self.V, self.kind = list(new), V, kind
        z = sharp * torch.randn((T, V), generator=g)
        self.p = _padded(torch.softmax(z, 1), dtype)
        self.q = _padded(torch.softmax(z + 0.7 * torch.randn((T, V), generator=g), 1), dtype)
        if kind == "certain":
            self.q = None
        self.parent, self.tokens = np.zeros(T, np.int64), np.zeros(T, np.int64)
        o = 0
        for n in new:
            for i in range(1, n):
                a = int(rng.integers(max(0, i - fan), i))
                self.parent[o + i] = a
                w = (self.p if self.q is None else self.q)[o + a].double().cpu().numpy().copy()
                if kind == "distinct":
                    taken = [self.tokens[o + j] for j in range(1, i) if self.parent[o + j] == a]
                    w[taken] = 0.0
                w = w if w.sum() > 0 else np.ones(V)
                self.tokens[o + i] = rng.choice(V, p=w / w.sum())
            o += n
        self.u = rng.random(T).astype(np.float32)

    def run(self, offsets=None, pad=0, **out):
        L = _lib()
        off = _offsets(self.new) if offsets is None else offsets
        return L.readme_verify_drafts(_i32(off), _i32(self.tokens), _i32(self.parent), self.p, self.q,
                                      torch.from_numpy(self.u).cuda(), self.kind == "distinct", **out)

    def check(self, got=None, safe=True):
        got = self.run() if got is None else got
        torch.cuda.synchronize()
        f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        path, acc, tok, margin = od.verify(_offsets(self.new), self.tokens, self.parent, f(self.p), f(self.q),
                                           self.u, self.kind == "distinct")
        assert not safe or margin > SAFE, margin
        np.testing.assert_array_equal(got[1].cpu().numpy(), acc)
        np.testing.assert_array_equal(got[2].cpu().numpy(), tok)
        np.testing.assert_array_equal(got[0].cpu().numpy(), path)
        return acc, tok


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
@pytest.mark.parametrize("new,V,fan", [
    ([1], 1, 1), ([3, 1, 2], 2, 2), ([6] * 40, 63, 1), ([0, 9, 0, 1, 33, 0], 65, 6),
    ([17, 64, 65, 130], 1000, 9), ([5] * 7, 4097, 5), ([24, 3], 32003, 8), ([12], 131075, 12)])
def test_verify(new, V, fan, kind, dtype):
    for seed in range(4 if V < 5000 else 2):
        Case(new, V, fan, kind, dtype, seed=seed + V, sharp=1.5 if kind != "certain" else 4.0).check()


@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
def test_many_requests_and_refusals(kind):
    """All children of one node, so that many are refused there."""
    c = Case([1 + i % 40 for i in range(300)], 300, 1, kind, seed=3)
    c.parent[:] = 0
    acc, tok = c.check()
    assert acc.max() == 1 and (acc == 0).any() and (tok >= 0).all()


def test_certain_drafts_are_distinct_or_not_alike():
    c = Case([1 + i % 9 for i in range(40)], 50, 3, "certain", seed=17, sharp=3.0)
    L = _lib()
    args = (_i32(_offsets(c.new)), _i32(c.tokens), _i32(c.parent), c.p, None, torch.from_numpy(c.u).cuda())
    for a, b in zip(L.readme_verify_drafts(*args), L.readme_verify_drafts(*args, distinct=True)):
        assert torch.equal(a, b)


def test_rows_past_the_limit_are_not_tried():
    c = Case([1500, 1100], 40, 1, seed=5)
    c.u[:] = 0.0   # everything is taken
    acc, _ = c.check()
    assert (acc == 1023).all()


def test_one_hot_targets():
    """A target that is certain takes the one draft it would have drawn."""
    c = Case([9] * 6, 50, 3, seed=6)
    best = torch.randint(0, 50, (54,), generator=torch.Generator().manual_seed(1))
    c.p.zero_()
    c.p[torch.arange(54), best] = 1.0
    c.tokens[::2] = best.numpy()[np.maximum(np.arange(54) - 1, 0)][::2]
    acc, tok = c.check(safe=False)
    assert (tok >= 0).all()


def test_odd_parents_and_tokens():
    """Parents that no row has, tokens outside the vocabulary: below no row, or
    never taken, and no access outside the arrays."""
    for kind in ("given", "distinct", "certain"):
        c = Case([12, 12, 12], 77, 2, kind, seed=7)
        c.parent[3], c.parent[5], c.parent[14], c.parent[26] = -1, 5, 11, 2 ** 31 - 1
        c.tokens[1], c.tokens[13], c.tokens[27] = 77, -1, -2 ** 31
        c.parent[0], c.tokens[0] = -2 ** 31, 2 ** 31 - 1  # row 0's are not read
        f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        path, acc, tok, _ = od.verify(_offsets(c.new), c.tokens, np.where(
            (c.parent >= 0) & (c.parent < np.tile(np.arange(12), 3)), c.parent, -1), f(c.p), f(c.q), c.u,
            kind == "distinct")
        got = c.run()
        torch.cuda.synchronize()
        for a, b in zip(got, (path, acc, tok)):
            np.testing.assert_array_equal(a.cpu().numpy(), b)


def test_entries_that_count_as_nothing():
    """NaN and negative entries; a target of zeros has no token; a draft beside a
    target equal to the drafts' own is refused by chance alone, and never where
    nothing would be left."""
    c = Case([5, 5, 5, 5], 300, 2, seed=8)
    c.p[0, ::3] = float("nan")
    c.p[1, ::2] = -1.0
    c.q[0, 5::7] = float("nan")
    c.p[5:10] = 0.0
    c.p[10:15] = c.q[10:15]
    acc, tok = c.check()
    assert tok[1] == -1 and (tok[[0, 2, 3]] >= 0).all()


def test_nothing_left():
    """p below q everywhere: a refusal leaves nothing, and the token is drawn from
    p; the node's other drafts are passed over."""
    c = Case([4], 64, 1, seed=9)
    c.parent[:] = 0
    c.p[:] = c.q * 0.25
    c.u[:] = [0.5, 0.9, 0.1, 0.1]
    acc, tok = c.check()
    assert acc[0] == 0 and tok[0] >= 0


@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_little_left_after_refusals(kind, dtype):
    """Nearly all of both distributions lies on the tokens refused first, so that what
    is left of them is far below what was taken away."""
    for seed in range(6):
        c = Case([6, 5, 6], 700, 1, kind, dtype, seed=seed)
        c.parent[:] = 0
        heavy = torch.tensor([[13, 699, 350], [0, 64, 512], [8, 9, 10]])
        for r, o in enumerate((0, 6, 11)):
            c.p[o, heavy[r]] = torch.tensor([1e3, 5e6, 2e4], device="cuda:0").to(dtype)
            if c.q is not None:
                c.q[o, heavy[r]] = torch.tensor([3e3, 2e7, 7e4], device="cuda:0").to(dtype)
            c.tokens[o + 1:o + 4] = heavy[r].numpy()
        c.u[:] = np.where(np.arange(17) % 5 == 0, 0.3, 1.0 - 2.0 ** -24)
        c.check(safe=False)


def test_borders_and_extreme_random_numbers():
    """Sums that are exact: a border that a sum meets belongs to the entry after it.
    0 and the number below 1 pick the first and the last entry."""
    V = 1024
    p = torch.full((3, V), 1.0 / V)
    for u, token in ((0.0, 0), (0.5, 512), (1.0 - 2.0 ** -24, V - 1), (511 / 1024, 511), (0.25, 256)):
        c = Case([1, 1, 1], V, seed=1)
        c.p, c.u = _padded(p, torch.float32), np.full(3, u, np.float32)
        acc, tok = c.check(safe=False)
        assert (tok == token).all()
    # Zeros before, between and after are never drawn
    p[:, :100] = 0
    p[:, 300:1000] = 0
    for u in (0.0, 200 / 224, 1.0 - 2.0 ** -24):
        c.p, c.u = _padded(p, torch.float32), np.full(3, u, np.float32)
        c.check(safe=False)


def test_rows_of_no_request_keep_what_they_held():
    c = Case([4, 0, 3, 5], 130, 2, seed=11)
    off = _offsets([4, 0, 3])
    new = [torch.full((n,), 77, dtype=torch.int32, device="cuda:0") for n in (12, 3, 3)]
    path, acc, tok = c.run(off, path=new[0], accepted=new[1], token=new[2])
    assert path is new[0] and (path[7:] == 77).all()
    whole = c.run()
    assert torch.equal(path[:7], whole[0][:7]) and torch.equal(acc, whole[1][:3]) and torch.equal(tok, whole[2][:3])
    assert int(acc[1]) == 0 and int(tok[1]) == -1


def test_no_rows_at_all():
    L = _lib()
    i = lambda n: torch.empty(n, dtype=torch.int32, device="cuda:0")  # noqa: E731
    path, acc, tok = L.readme_verify_drafts(_i32([0, 0, 0]), i(0), i(0), torch.empty((0, 50), device="cuda:0"), None,
                                            torch.empty(0, device="cuda:0"))
    assert path.numel() == 0 and acc.tolist() == [0, 0] and tok.tolist() == [-1, -1]


def test_offsets_past_32_bits():
    """Rows of p and q beyond 2^31 entries."""
    L = _lib()
    c = Case([4], 1000, 1, dtype=torch.bfloat16, seed=12)
    ld = (1 << 30) + 8
    base = torch.empty(3 * ld + 1008, dtype=torch.bfloat16, device="cuda:0")
    far = torch.as_strided(base, (4, 1000), (ld, 1))
    ref = c.run()
    far.copy_(c.p)
    q = c.q.contiguous()
    got = L.readme_verify_drafts(_i32([0, 4]), _i32(c.tokens), _i32(c.parent), far, q,
                                 torch.from_numpy(c.u).cuda())
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


@pytest.mark.parametrize("R,V", [(40, 5000), (3, 70001)])
def test_captured_and_on_two_streams(R, V):
    L = _lib()
    cases = [Case([7] * R, V, 3, "distinct", seed=s) for s in range(3)]
    ins = [(_i32(c.tokens), _i32(c.parent), c.p, c.q, torch.from_numpy(c.u).cuda()) for c in cases]
    refs = [c.run() for c in cases]
    off = _i32(_offsets(cases[0].new))
    state = [t.clone() if t.dim() == 1 else _padded(t, t.dtype) for t in ins[0]]
    outs = [torch.empty_like(t) for t in refs[0]]
    ws = torch.empty(max(1, L.readme_verify_drafts_workspace_bytes(7 * R, R, V)), dtype=torch.uint8, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.readme_verify_drafts(off, *state, distinct=True, path=outs[0], accepted=outs[1], token=outs[2],
                               workspace=ws)
    for i in (0, 1, 2, 1):
        for dst, src in zip(state, ins[i]):
            dst.copy_(src)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, refs[i]):
            assert torch.equal(a, b)
    streams, got = [torch.cuda.Stream() for _ in cases], []
    torch.cuda.synchronize()
    for s, x in zip(streams, ins):
        with torch.cuda.stream(s):
            got.append([L.readme_verify_drafts(off, *x, distinct=True) for _ in range(4)])
    torch.cuda.synchronize()
    for ref, runs in zip(refs, got):
        for one in runs:
            for a, b in zip(one, ref):
                assert torch.equal(a, b)


def test_python_form_refuses():
    L = _lib()
    c = Case([4, 4], 64, seed=13)
    off, tok, par, u = _i32([0, 4, 8]), _i32(c.tokens), _i32(c.parent), torch.from_numpy(c.u).cuda()
    for call in (lambda: L.readme_verify_drafts(off, tok[:7], par, c.p, c.q, u),
                 lambda: L.readme_verify_drafts(off, tok.long(), par, c.p, c.q, u),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p, c.q.bfloat16(), u),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p, c.q[:, :32], u),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p, c.q, u.double()),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p, c.q, u.cpu()),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p, c.q, u, path=tok[:4]),
                 lambda: L.readme_verify_drafts(off, tok, par, c.p[:, ::2], None, u)):
        with pytest.raises(ValueError):
            call()
    one = (_i32([0, 1]), tok[:1], par[:1])  # a single row too has its entries side by side
    with pytest.raises(ValueError):
        L.readme_verify_drafts(*one, c.p[:, :1].t(), None, u[:1])
    with pytest.raises(ValueError):
        L.readme_verify_drafts(*one, c.p[:1, :8], c.q[:, :1].t(), u[:1])
    with pytest.raises(ValueError):
        L.readme_verify_drafts(off, tok, par, c.p.half(), c.q.half(), u)
