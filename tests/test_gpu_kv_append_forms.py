"""readme_kv_append in each of its forms, which the library itself names: bit for bit
readme_rotary in fp32 and readme_kv_write, at sizes on both sides of every rule."""
import ctypes
import os

import pytest
import torch

from tests.test_gpu_kv import KT, _i32, _offsets


def _lib():
    from paper_2410_19123_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libreadme.so not built")
    return _lib


def form(new, Hk, D):
    fn = _lib().load().readme_internal_kv_append_form
    fn.restype = ctypes.c_int32
    fn.argtypes = [ctypes.c_int64] + [ctypes.c_int32] * 3
    return ("one by one", "second apart", "heads share")[fn(sum(new), len(new), Hk, D)]


# Rows of the requests, key heads, head dims.  Blocks of 64 tokens: requests of 70 and
# more rows have a third one.
CASES = {
    "one by one": [([1] * 300, 2, 128), ([1] * 129 + [3], 2, 64), ([1 + i % 9 for i in range(129)], 2, 128),
                   ([0, 65, 70, 2] * 33, 3, 64), ([165] * 300, 1, 64), ([47] * 260, 1, 256),
                   ([700] * 18, 15, 256)],
    "second apart": [([2], 1, 64), ([1 + i % 9 for i in range(128)], 2, 128), ([130, 1, 0, 63, 64, 200], 5, 64),
                     ([24575, 0], 2, 64), ([49152], 1, 64), ([6000, 6300, 1], 4, 256), ([12287], 4, 128)],
    "heads share": [([24576, 0], 2, 64), ([12288], 4, 128), ([1] * 24576, 2, 64), ([7] * 1405, 5, 128),
                    ([65, 0, 1, 70] * 242, 3, 64)],
}
ALL = [(name, *case) for name, cases in CASES.items() for case in cases]


@pytest.mark.parametrize("name,new,Hk,D", ALL)
def test_sizes_take_the_form_they_are_named_after(name, new, Hk, D):
    assert form(new, Hk, D) == name


@pytest.mark.gpu
@pytest.mark.parametrize("kt,dtype,layout", [("e4m3", torch.bfloat16, 0), ("i8", torch.float32, 1)])
@pytest.mark.parametrize("name,new,Hk,D", ALL)
def test_append_in_every_form(name, new, Hk, D, kt, dtype, layout):
    """Behind up to 90 tokens, on blocks that hold some and grow; absent blocks and rows
    of no request among them, positions stored and given."""
    L = _lib()
    g = torch.Generator().manual_seed(len(new) + Hk)
    freqs = L.readme_rotary_freqs(D // 2, device="cuda:0")
    R, T = len(new), sum(new)
    mb = (max(new) + 90) // 64 + 1
    table = torch.randperm(R * mb, generator=g).int().reshape(R, mb)
    table[torch.rand((R, mb), generator=g) < 0.05] = -1
    table = table.cuda()
    on = {"generator": torch.Generator(device="cuda:0").manual_seed(Hk + D), "device": "cuda:0"}
    codes = torch.randint(1, 120, (R * mb, Hk, 2, 64 * D), dtype=torch.uint8, **on)
    scales = torch.rand((R * mb, Hk, 2), **on) * 0.02 + 0.001
    caches = [(codes.clone(), scales.clone()) for _ in range(2)]
    before = torch.randint(0, 91, (R,), generator=g).tolist()
    off, lens = _i32(_offsets(new)), _i32([b + n for b, n in zip(before, new)])
    k, v = (torch.randn((T + 3, Hk * D), **on).to(dtype) for _ in range(2))
    at = torch.cat([torch.arange(b, b + n) for b, n in zip(before, new)] + [torch.zeros(3)]).int().cuda()
    for pos in (None, torch.randint(-99, 200000, (T + 3,), generator=g).int().cuda()):
        L.readme_kv_append(KT[kt], k, v, off, lens, table, *caches[0], freqs, pos, layout, 1.25)
        turned = L.readme_rotary(k.float(), at if pos is None else pos, freqs, D, layout, 1.25)
        L.readme_kv_write(KT[kt], turned, v.float(), off, lens, table, *caches[1])
        torch.cuda.synchronize()
        assert torch.equal(caches[0][0], caches[1][0])
        assert torch.equal(caches[0][1].view(torch.int32), caches[1][1].view(torch.int32))
    assert not torch.equal(caches[0][0], codes)
