"""readme_kv_append on the GPU: bit for bit readme_rotary in fp32 and
readme_kv_write, and the oracle's codes of the turned keys."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from oracle import kv_cache as ok
from tests.test_gpu_kv import KT, Cache, _i32, _offsets, _rows

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


class Appended(Cache):
    """A cache that calls append to, with the oracle's turned by readme_rotary in
    fp32 (whose own bound tests.test_gpu_rotary holds it to)."""

    def append(self, new, lens, dtype, freqs, layout=0, amplitude=1.0, pos=None, k=None, v=None, pad=0):
        L = _lib()
        off, T = _offsets(new), int(sum(new)) + pad
        k = _rows(self.rng, T, self.Hk, self.D, dtype) if k is None else k
        v = _rows(self.rng, T, self.Hk, self.D, dtype) if v is None else v
        at = np.concatenate([np.arange(ln - n, ln) for n, ln in zip(new, lens)] + [np.zeros(pad)])
        p = None if pos is None else _i32(pos)
        L.readme_kv_append(KT[self.kt], k.reshape(T, -1).cuda(), v.reshape(T, -1).cuda(), _i32(off),
                           _i32(lens), *self.args(), freqs, p, layout, amplitude)
        turned = L.readme_rotary(k.reshape(T, -1).float().cuda(), _i32(at) if p is None else p, freqs,
                                 self.D, layout, amplitude)
        torch.cuda.synchronize()
        ok.write(self.kt, self.ref, turned.cpu().double().numpy().reshape(T, self.Hk, self.D),
                 v.double().numpy(), off, lens, self.table)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kt", ["i8", "e4m3"])
@pytest.mark.parametrize("D,Hk,rot,layout", [(64, 3, 64, 0), (64, 2, 32, 1), (128, 2, 128, 0),
                                             (128, 1, 48, 0), (256, 1, 256, 1), (256, 2, 80, 0)])
def test_append(D, Hk, rot, layout, kt, dtype):
    """Prompts, single tokens, drafts and pieces across block borders, positions
    stored and given, blocks that grow."""
    L = _lib()
    freqs = L.readme_rotary_freqs(rot, device="cuda:0")
    c = Appended(kt, 5, Hk, D, 4, seed=D + rot)
    lens = np.zeros(5, np.int32)
    for step, new in enumerate(([1, 63, 64, 65, 130], [1, 1, 1, 1, 1], [5, 0, 3, 62, 1], [60, 2, 70, 0, 1])):
        lens = lens + np.array(new, np.int32)
        pos = c.rng.integers(-50, 100000, sum(new)) if step % 2 else None
        c.append(new, lens, dtype, freqs, layout, 1.0 if step < 2 else 1.25, pos)
        c.check()


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
def test_append_against_the_formula(kt):
    """Read back: within the rotation's bound and half a step of the code (int8
    amax / 254, e4m3 2^-4 of the value) of the 64-bit keys."""
    L = _lib()
    c = Appended(kt, 2, 2, 128, 3, seed=5)
    freqs = L.readme_rotary_freqs(128, 5e5, L.README_ROTARY_BANDED, 8.0, 4096.0, device="cuda:0")
    new, lens = [100, 64], [100, 64]
    k = torch.randn(164, 2, 128)
    pos = c.rng.integers(0, 131072, 164)
    c.append(new, lens, torch.float32, freqs, 0, 1.0, pos, k=k)
    kb, _ = L.readme_kv_read(KT[kt], _i32(_offsets(new)), _i32(lens), *c.args(), T=164, dtype=torch.float32)
    ref = od.rotary(k.double().numpy(), pos, freqs.cpu().numpy())
    err = np.abs(kb.cpu().double().numpy().reshape(ref.shape) - ref)
    big = np.abs(ref).max()
    step = big / 254 if kt == "i8" else 2.0 ** -4 * np.abs(ref) + 2.0 ** -10 * big / 448
    assert (err <= step * (1 + 2.0 ** -20) + 2.0 ** -20 * big).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D,Hk,rot,layout,kt,new", [
    (128, 9, 128, 0, "e4m3", [3001, 1, 0, 64, 2500]), (64, 2, 32, 1, "i8", [9000, 17, 16000, 63, 1]),
    (128, 4, 48, 1, "i8", [65] * 200), (64, 7, 64, 0, "e4m3", [4000, 3100, 5, 0, 70]),
    (256, 5, 256, 0, "i8", [6000, 4000, 1, 30, 2])])
def test_many_rows(D, Hk, rot, layout, kt, new, dtype):
    """Bit for bit the rotation in fp32 and the write, at sizes where heads share
    their sines and cosines, on empty blocks and on blocks that hold tokens and grow,
    with rows of no request and an absent block."""
    L = _lib()
    g = torch.Generator().manual_seed(D + Hk)
    freqs = L.readme_rotary_freqs(rot, device="cuda:0")
    R, T = len(new), sum(new) + 3
    mb = -(-(2 * max(new)) // 64) + 1
    table = torch.randperm(R * mb, generator=g).int().reshape(R, mb)
    table[0, 1] = -1
    table = table.cuda()
    caches = [(torch.zeros((R * mb, Hk, 2, 64 * D), dtype=torch.uint8, device="cuda:0"),
               torch.zeros((R * mb, Hk, 2), device="cuda:0")) for _ in range(2)]
    off = _i32(_offsets(new))
    assert T * Hk >= 49152
    for step in (1, 2):
        lens = _i32([step * n for n in new])
        k, v = (torch.randn((T, Hk * D), generator=g).mul_(step).to(dtype).cuda() for _ in range(2))
        at = torch.cat([torch.arange((step - 1) * n, step * n) for n in new] + [torch.zeros(3)]).int().cuda()
        pos = torch.randint(-99, 200000, (T,), generator=g).int().cuda() if step == 2 else None
        L.readme_kv_append(KT[kt], k, v, off, lens, table, *caches[0], freqs, pos, layout, 1.25)
        turned = L.readme_rotary(k.float(), at if pos is None else pos, freqs, D, layout, 1.25)
        L.readme_kv_write(KT[kt], turned, v.float(), off, lens, table, *caches[1])
        torch.cuda.synchronize()
        assert torch.equal(caches[0][0], caches[1][0])
        assert torch.equal(caches[0][1].view(torch.int32), caches[1][1].view(torch.int32))


def test_absent_foreign_and_bad_rows():
    """Absent blocks and positions before the first token drop their rows, rows past
    offsets[R] are not read, an infinity turns its block's keys NaN and no other's."""
    L = _lib()
    freqs = L.readme_rotary_freqs(64, device="cuda:0")
    c = Appended("i8", 4, 2, 64, 2, seed=9)
    c.table[1, 0] = -1
    c.table[2, 1] = 1 << 30
    new, lens = [10, 100, 100, 40], [4, 100, 100, 140]
    k, v = (_rows(c.rng, 257, 2, 64, torch.float32) for _ in range(2))
    k[250:] = float("nan")
    v[250:] = float("nan")
    c.append(new, lens, torch.float32, freqs, k=k, v=v, pad=7)
    c.check()
    bad = int(torch.isnan(c.scales).sum())  # request 3's block, begun past its first token
    k[3, 0, 5] = float("inf")
    c.append([1, 0, 0, 1], [5, 100, 100, 90], torch.float32, freqs, k=k[3:5], v=v[3:5])
    c.check()
    assert torch.isnan(c.scales).sum() == bad + 1


def test_slices_of_a_projection():
    """Keys and values as columns of one q|k|v row."""
    L = _lib()
    freqs = L.readme_rotary_freqs(128, device="cuda:0")
    qkv = torch.randn(70, 8 * 128, device="cuda:0").bfloat16()
    k, v = qkv[:, 512:768], qkv[:, 768:]
    table, off, lens = _i32([[1, 0]]), _i32([0, 70]), _i32([90])
    caches = [L.readme_kv_cache(2, 2, 128, "cuda:0") for _ in range(2)]
    for codes, scales in caches:
        codes.fill_(130)
        scales.fill_(0.125)
    L.readme_kv_append(0, k, v, off, lens, table, *caches[0], freqs)
    pos = torch.arange(20, 90, dtype=torch.int32, device="cuda:0")
    turned = L.readme_rotary(k.float(), pos, freqs, 128)
    L.readme_kv_write(0, turned, v.float(), off, lens, table, *caches[1])
    assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


def test_captured_append_follows_the_lengths():
    L = _lib()
    freqs = L.readme_rotary_freqs(64, device="cuda:0")
    table = _i32(np.random.default_rng(1).permutation(20).reshape(4, 5))
    base = (torch.randint(1, 255, (20, 2, 2, 64 * 64), device="cuda:0", dtype=torch.int32).to(torch.uint8),
            torch.rand((20, 2, 2), device="cuda:0") * 0.02 + 0.001)
    caches = [tuple(t.clone() for t in base) for _ in range(2)]
    k, v = (torch.randn(7, 128, device="cuda:0").bfloat16() for _ in range(2))
    off, lens, pos = _i32([0, 1, 3, 3, 7]), _i32([10, 20, 30, 40]), _i32(range(7))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.readme_kv_append(0, k, v, off, lens, table, *caches[0], freqs, pos)
    for cache in caches:
        for t, b in zip(cache, base):
            t.copy_(b)
    for i, now in enumerate(([1, 64, 0, 66], [65, 66, 5, 320], [300, 2, 5, 100])):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        k.copy_(torch.randn(7, 128, device="cuda:0"))
        pos.copy_(torch.arange(7, dtype=torch.int32) + 1000 * i)
        graph.replay()
        L.readme_kv_append(0, k, v, off, lens, table, *caches[1], freqs, pos)
        torch.cuda.synchronize()
        assert torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


def test_python_form_refuses():
    L = _lib()
    freqs = L.readme_rotary_freqs(64, device="cuda:0")
    codes, scales = L.readme_kv_cache(3, 2, 64, "cuda:0")
    k = torch.randn(5, 128, device="cuda:0")
    at = (_i32([0, 5]), _i32([5]), _i32([[0, 1]]), codes, scales)
    for call in (lambda: L.readme_kv_append(0, k, k, *at, freqs.float()),
                 lambda: L.readme_kv_append(0, k, k, *at, freqs.cpu()),
                 lambda: L.readme_kv_append(0, k, k, *at, freqs, _i32([1, 2])),
                 lambda: L.readme_kv_append(0, k, k.bfloat16(), *at, freqs),
                 lambda: L.readme_kv_append(0, k[:, :64], k, *at, freqs)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(L.ReadmeError):
        L.readme_kv_append(0, k, k, *at, L.readme_rotary_freqs(128, device="cuda:0"))
