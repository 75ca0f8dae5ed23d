"""Steps with drafted tokens, as a server runs them: queries and keys turned by
their depth in the tree, keys and values appended, attention over the tree, the
drafts verified, and the taken rows moved to where they belong."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from oracle import kv_cache as ok
from tests.test_gpu_kv import Cache, _i32, _offsets

pytestmark = pytest.mark.gpu

Hk, G, D, V = 2, 2, 64, 200


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def _model(gen, T):
    """A stand-in for the model's layers: q, k, v of the rows."""
    return [torch.randn((T, n * D), generator=gen, device="cuda:0").bfloat16() for n in (Hk * G, Hk, Hk)]


def _distributions(o, seed):
    """The target's and the drafts' distributions, from the attention's rows."""
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    w = torch.randn((Hk * G * D, V), generator=g, device="cuda:0")
    z = 0.5 * o.float() @ w
    return torch.softmax(z, 1), torch.softmax(z + 0.3 * torch.randn(z.shape, generator=g, device="cuda:0"), 1)


def test_conversations_with_drafts():
    L = _lib()
    R, trees = 3, [[-1, 0, 0, 1, 2, 2], [-1, 0, 1, 2], [-1, 0, 0, 0, 3, 3, 5]]
    new, T = [len(t) for t in trees], sum(len(t) for t in trees)
    off = _offsets(new)
    parent = np.concatenate(trees).clip(0)
    masks = sum((od.bits(t) for t in trees), [])
    depth = np.concatenate([od.depths(t) for t in trees])
    c = Cache("i8", R, Hk, D, 4, seed=70)
    freqs = L.readme_rotary_freqs(D, device="cuda:0")
    gen = torch.Generator(device="cuda:0").manual_seed(71)
    # Prompts, the positions those they are stored at
    lens = np.array([60, 1, 125], np.int32)
    _, k, v = _model(gen, int(lens.sum()))
    L.readme_kv_append(0, k, v, _i32(_offsets(lens)), _i32(lens), *c.args(), freqs)
    pos = np.concatenate([np.arange(n) for n in lens])
    turned = L.readme_rotary(k.float(), _i32(pos), freqs, D)
    as64 = lambda t, h: t.double().cpu().numpy().reshape(-1, h, D)  # noqa: E731
    ok.write("i8", c.ref, as64(turned, Hk), as64(v, Hk), _offsets(lens), lens, c.table)
    c.check()
    rng = np.random.default_rng(72)
    for step in range(4):
        full = (lens + np.array(new)).astype(np.int32)
        pos = np.repeat(lens, new) + depth
        q, k, v = _model(gen, T)
        q = L.readme_rotary(q, _i32(pos), freqs, D)
        L.readme_kv_append(0, k, v, _i32(off), _i32(full), *c.args(), freqs, _i32(pos))
        turned = L.readme_rotary(k.float(), _i32(pos), freqs, D)
        ok.write("i8", c.ref, as64(turned, Hk), as64(v, Hk), off, full, c.table)
        c.check()
        tree = torch.from_numpy(od.words(masks, 1)).cuda()
        o = L.readme_attention_kv_tree(0, q, _i32(off), _i32(full), *c.args(), Hk * G, tree, _i32(pos))
        ref, vmax, _ = od.attention_tree(c.ref, as64(q, Hk * G), off, full, c.table, masks, D ** -0.5)
        assert (np.abs(as64(o, Hk * G) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10 * vmax[..., None]).all()
        p, pq = _distributions(o, step)
        at = off[:-1].repeat(new) + parent
        tokens = torch.multinomial(pq[torch.from_numpy(at).cuda()], 1, generator=gen)[:, 0].int()
        u = rng.random(T).astype(np.float32)
        path, taken, token = L.readme_verify_drafts(_i32(off), tokens, _i32(parent), p, pq, torch.from_numpy(u).cuda())
        rp, ra, rt, margin = od.verify(off, tokens.cpu().numpy(), parent, p.double().cpu().numpy(),
                                       pq.double().cpu().numpy(), u)
        assert margin > 2.0 ** -30
        assert path.tolist() == rp.tolist() and taken.tolist() == ra.tolist() and token.tolist() == rt.tolist()
        # The taken rows read from where the call left them, and written behind each
        # other: all on the device, rows past the last one belonging to no request
        kb, vb = L.readme_kv_read(0, _i32(off), _i32(full), *c.args(), T=T, dtype=torch.float32)
        count = taken + 1
        keep_off = torch.cat([torch.zeros_like(count[:1]), count.cumsum(0).int()]).int()
        real = path >= 0
        rows = torch.zeros(T, dtype=torch.long, device="cuda:0")
        rows[torch.cumsum(real, 0)[real] - 1] = (_i32(off[:-1].repeat(new)) + path)[real].long()
        lens = lens + count.cpu().numpy()
        L.readme_kv_write(0, kb[rows].contiguous(), vb[rows].contiguous(), keep_off, _i32(lens), *c.args())
        ok.write("i8", c.ref, as64(kb[rows], Hk), as64(vb[rows], Hk), keep_off.cpu().numpy(), lens, c.table)
        c.check()
    assert lens.sum() > 186 + 4 * R  # some drafts were taken


def test_a_captured_step():
    """Rotation, append, attention and verification in one graph, replayed on other
    rows, lengths, trees and random numbers with eager work between."""
    L = _lib()
    R, n, mb = 4, 9, 6
    T = R * n
    rng = np.random.default_rng(80)
    freqs = L.readme_rotary_freqs(D, device="cuda:0")
    table = _i32(rng.permutation(R * mb).reshape(R, mb))
    base = (torch.randint(1, 255, (R * mb, Hk, 2, 64 * D), device="cuda:0", dtype=torch.int32).to(torch.uint8),
            torch.rand((R * mb, Hk, 2), device="cuda:0") * 0.02 + 0.01)
    codes, scales = (t.clone() for t in base)
    off = _i32(_offsets([n] * R))
    gen = torch.Generator(device="cuda:0").manual_seed(81)
    ws = torch.empty(L.readme_attention_kv_tree_workspace_bytes(T, R, Hk * G, Hk, D, mb), dtype=torch.uint8,
                     device="cuda:0")
    ws2 = torch.empty(max(1, L.readme_verify_drafts_workspace_bytes(T, R, V)), dtype=torch.uint8, device="cuda:0")
    i32 = lambda m: torch.zeros(m, dtype=torch.int32, device="cuda:0")  # noqa: E731

    def inputs(seed):
        r = np.random.default_rng(seed)
        trees = [[-1] + [int(r.integers(max(0, i - 3), i)) for i in range(1, n)] for _ in range(R)]
        ln = r.integers(n, mb * 64, R)
        pos = np.repeat(ln - n, n) + np.concatenate([od.depths(t) for t in trees])
        z = torch.randn((T, V), generator=gen, device="cuda:0")
        return [*_model(gen, T), _i32(ln), _i32(pos), torch.from_numpy(od.words(sum(map(od.bits, trees), []), 1)).cuda(),
                _i32(np.concatenate(trees).clip(0)), _i32(r.integers(0, V, T)), torch.softmax(2 * z, 1),
                torch.softmax(z, 1), torch.rand(T, generator=gen, device="cuda:0")]

    sets = [inputs(s) for s in range(3)]
    state = [t.clone() for t in sets[0]]
    qt, o = torch.empty_like(state[0]), torch.empty_like(state[0])
    outs = [o, i32(T), i32(R), i32(R), codes, scales]

    def step():
        q, k, v, lens, pos, tree, parent, tokens, p, pq, u = state
        L.readme_rotary(q, pos, freqs, D, y=qt)
        L.readme_kv_append(0, k, v, off, lens, table, codes, scales, freqs, pos)
        L.readme_attention_kv_tree(0, qt, off, lens, table, codes, scales, Hk * G, tree, pos, o=o, workspace=ws)
        L.readme_verify_drafts(off, tokens, parent, p, pq, u, path=outs[1], accepted=outs[2], token=outs[3],
                               workspace=ws2)

    def load(i):
        for dst, src in zip(state, sets[i]):
            dst.copy_(src)
        codes.copy_(base[0])
        scales.copy_(base[1])

    refs = []
    for i in range(3):
        load(i)
        step()
        torch.cuda.synchronize()
        refs.append([t.clone() for t in outs])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 2, 0):
        load(i)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, refs[i]):
            assert torch.equal(a, b), i
