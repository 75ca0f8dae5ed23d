"""readme_attention_kv_tree on the GPU at sizes that choose its form: the most
requests that a call may have."""
import pytest
import torch

from tests.test_gpu_kv import _i32

pytestmark = pytest.mark.gpu


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def test_most_requests():
    """2^22 requests, the last alone with a row, at two key heads: the largest grid
    that the limits allow.  The row equals that of a call with its request alone, but
    for the order of the sums (each within 2^-8 of its value of bf16's rounding, and
    2^-10 of the largest value of the weights')."""
    L = _lib()
    R, Hk, D, mb = 1 << 22, 2, 64, 16
    g = torch.Generator(device="cuda:0").manual_seed(4)
    codes = torch.randint(1, 256, (mb, Hk, 2, 64 * D), generator=g, device="cuda:0",
                          dtype=torch.int32).to(torch.uint8)
    scales = torch.rand((mb, Hk, 2), generator=g, device="cuda:0") * 0.02 + 0.01
    q = torch.randn((1, Hk * D), generator=g, device="cuda:0").bfloat16()
    tree = torch.ones((1, 1), dtype=torch.int64, device="cuda:0")
    table = torch.full((R, mb), -1, dtype=torch.int32, device="cuda:0")
    table[-1] = torch.arange(mb, device="cuda:0")
    off = torch.zeros(R + 1, dtype=torch.int32, device="cuda:0")
    off[-1] = 1
    lens = torch.full((R,), 900, dtype=torch.int32, device="cuda:0")
    o = L.readme_attention_kv_tree(0, q, off, lens, table, codes, scales, Hk, tree)
    one = L.readme_attention_kv_tree(0, q, _i32([0, 1]), lens[:1], table[-1:], codes, scales, Hk, tree)
    torch.cuda.synchronize()
    most = 127 * float(scales[..., 1].max())
    assert ((o.double() - one.double()).abs() <= 2.0 ** -7 * one.double().abs() + 2.0 ** -10 * most).all()
    assert one.abs().max() > 0
