"""readme_rotary on the GPU against its 64-bit oracle, and what has to hold between
its calls: in place, back again, slices, graphs, far offsets."""
import numpy as np
import pytest
import torch

from oracle import drafts as od

pytestmark = pytest.mark.gpu

LAYOUT = {"half": 0, "pairs": 1}


def _lib():
    from paper_2410_19123_amd import _lib
    return _lib


def bound(x, freqs, layout, amplitude, ref, dtype):
    """2^-21 A (|a| + |b|) for the turned dims, half a step of the type for each."""
    rot = 2 * len(freqs)
    a = np.abs(x[..., :rot])
    if layout == "half":
        pair = np.concatenate([a[..., rot // 2:], a[..., :rot // 2]], -1)
    else:
        pair = a.reshape(*a.shape[:-1], -1, 2)[..., ::-1].reshape(a.shape)
    tol = np.zeros_like(x)
    tol[..., :rot] = 2.0 ** -21 * abs(amplitude) * (a + pair)
    return tol + torch.finfo(dtype).eps / 2 * np.abs(ref)


def check(x, pos, freqs, D, layout, amplitude, inverse, y):
    T = x.shape[0]
    x64 = x.double().cpu().numpy().reshape(T, -1, D)
    ref = od.rotary(x64, pos.cpu().numpy(), freqs.cpu().numpy(), layout, amplitude, inverse)
    got = y.double().cpu().numpy().reshape(T, -1, D)
    tol = bound(x64, freqs, layout, float(np.float32(amplitude)), ref, x.dtype)
    worst = (np.abs(got - ref) - tol).max()
    assert worst <= 0, worst


def make(T, H, D, dtype, seed, span=5000):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    x = torch.randn((T, H * D), generator=g, device="cuda:0").to(dtype)
    pos = torch.randint(-span, span, (T,), generator=g, device="cuda:0", dtype=torch.int32)
    return x, pos


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 16, 16), (1, 8, 128, 128), (5, 3, 80, 32),
                                       (67, 12, 64, 48), (130, 71, 96, 96), (3, 2, 512, 512),
                                       (1025, 5, 256, 64), (9000, 1, 32, 16)])
def test_rotary(T, H, D, rot, layout, dtype):
    L = _lib()
    x, pos = make(T, H, D, dtype, T + D)
    freqs = L.readme_rotary_freqs(rot, device="cuda:0")
    for amplitude, inverse in ((1.0, False), (-0.7, True)):
        y = L.readme_rotary(x, pos, freqs, D, LAYOUT[layout], amplitude, inverse)
        check(x, pos, freqs, D, layout, amplitude, inverse, y)


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_far_positions(layout):
    """Positions over all of int32, and frequencies above 1."""
    L = _lib()
    x, _ = make(64, 2, 64, torch.float32, 1)
    at = [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1] + [int(v) for v in np.geomspace(2, 2e9, 58)]
    pos = torch.tensor(at, dtype=torch.int32, device="cuda:0")
    for freqs in (L.readme_rotary_freqs(64, 5e5), L.readme_rotary_freqs(64) * 3000.0,
                  torch.zeros(32, dtype=torch.float64)):
        freqs = freqs.cuda()
        check(x, pos, freqs, 64, layout, 1.0, False, L.readme_rotary(x, pos, freqs, 64, LAYOUT[layout]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slices_in_place_and_back(dtype):
    """A slice of wider rows turned in place is the call beside it bit for bit and
    leaves the columns around it; turning back undoes it."""
    L = _lib()
    T, H, D = 37, 3, 96
    wide = torch.randn(T, (H + 4) * D, device="cuda:0").to(dtype)
    was = wide.clone()
    pos = torch.arange(100, 100 + T, dtype=torch.int32, device="cuda:0")
    freqs = L.readme_rotary_freqs(64, device="cuda:0")
    part = wide[:, 2 * D:(2 + H) * D]
    y = L.readme_rotary(part, pos, freqs, D)
    assert L.readme_rotary(part, pos, freqs, D, y=part) is part
    assert torch.equal(part, y)
    assert torch.equal(wide[:, :2 * D], was[:, :2 * D]) and torch.equal(wide[:, 5 * D:], was[:, 5 * D:])
    L.readme_rotary(part, pos, freqs, D, inverse=True, y=part)
    big = was.float().abs().max()
    assert ((wide.float() - was.float()).abs() <= 4 * torch.finfo(dtype).eps * big).all()


def test_dims_that_do_not_turn_are_copied():
    """Infinities and NaN among them, and only there."""
    L = _lib()
    x, pos = make(9, 2, 64, torch.bfloat16, 3)
    x.view(9, 2, 64)[..., 40] = float("nan")
    x.view(9, 2, 64)[..., 63] = float("-inf")
    freqs = L.readme_rotary_freqs(32, device="cuda:0")
    y = L.readme_rotary(x, pos, freqs, 64).view(9, 2, 64)
    assert torch.equal(y[..., 32:].view(torch.int16), x.view(9, 2, 64)[..., 32:].view(torch.int16))
    assert torch.isfinite(y[..., :32]).all()


def test_as_readme_rope():
    """The case that readme_rope has: its fp64 result, rounded, up to this call's
    bound and one more rounding."""
    L = _lib()
    x, _ = make(300, 4, 128, torch.bfloat16, 4)
    pos = torch.arange(300, dtype=torch.int32, device="cuda:0") * 13
    y = L.readme_rotary(x, pos, L.readme_rotary_freqs(128, device="cuda:0"), 128)
    ref = L.readme_rope(x.clone(), pos, 4)
    ab = 2.0 ** -21 * 2 * x.float().abs().max()
    assert ((y.float() - ref.float()).abs() <= ab + 2.0 ** -7 * ref.float().abs()).all()
    assert (y == ref).float().mean() > 0.999


@pytest.mark.parametrize("layout", ["half", "pairs"])
def test_gradient(layout):
    """Against differences of the call itself, which is linear: <g, R(x + h) - R(x -
    h)> for steps h of one element, and the formula's gradient."""
    L = _lib()
    T, H, D, rot = 3, 2, 32, 16
    x, pos = make(T, H, D, torch.float32, 5)
    g, _ = make(T, H, D, torch.float32, 6)
    freqs = L.readme_rotary_freqs(rot, device="cuda:0")
    grad = L.readme_rotary(g, pos, freqs, D, LAYOUT[layout], 1.5, True)
    check(g, pos, freqs, D, layout, 1.5, True, grad)
    call = lambda z: L.readme_rotary(z, pos, freqs, D, LAYOUT[layout], 1.5).double()  # noqa: E731
    for i in range(0, x.numel(), 7):
        h = torch.zeros_like(x)
        h.view(-1)[i] = 0.5
        d = ((call(x + h) - call(x - h)) * g.double()).sum()
        # x +- h and both results round: a few 2^-24 of the row's values each
        assert abs(float(d) - float(grad.view(-1)[i])) <= 2.0 ** -18 * 1.5 * float(g.abs().max())


def test_rows_past_32_bit_offsets():
    L = _lib()
    ld = (1 << 31) // 2 + 64
    base = torch.empty(2 * ld + 256, dtype=torch.bfloat16, device="cuda:0")
    x = torch.as_strided(base, (3, 128), (ld, 1))
    x.copy_(torch.randn(3, 128, device="cuda:0"))
    pos = torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda:0")
    freqs = L.readme_rotary_freqs(64, device="cuda:0")
    ref = L.readme_rotary(x.contiguous(), pos, freqs, 64)
    L.readme_rotary(x, pos, freqs, 64, y=x)
    assert torch.equal(x, ref)


def test_captured_on_another_stream():
    L = _lib()
    x, pos = make(50, 4, 128, torch.bfloat16, 7)
    freqs, y = L.readme_rotary_freqs(128, device="cuda:0"), torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.readme_rotary(x, pos, freqs, 128, y=y)
    for seed in (8, 9, 10):
        a, b = make(50, 4, 128, torch.bfloat16, seed)
        x.copy_(a)
        pos.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            ref = L.readme_rotary(x, pos, freqs, 128)
        s.synchronize()
        assert torch.equal(y, ref)


def test_no_rows_and_refusals():
    L = _lib()
    freqs = L.readme_rotary_freqs(32, device="cuda:0")
    x = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda:0")
    assert L.readme_rotary(x, torch.empty(0, dtype=torch.int32, device="cuda:0"), freqs, 64).shape == (0, 128)
    x, pos = make(4, 2, 64, torch.bfloat16, 11)
    for call in (lambda: L.readme_rotary(x, pos[:3], freqs, 64), lambda: L.readme_rotary(x, pos.long(), freqs, 64),
                 lambda: L.readme_rotary(x, pos, freqs.float(), 64), lambda: L.readme_rotary(x, pos, freqs.cpu(), 64),
                 lambda: L.readme_rotary(x, pos, freqs, 48), lambda: L.readme_rotary(x.half(), pos, freqs, 64),
                 lambda: L.readme_rotary(x, pos, freqs, 64, y=x.float()),
                 lambda: L.readme_rotary(x, pos, freqs, 64, y=x[:3]),
                 lambda: L.readme_rotary(x[:, ::2], pos, freqs, 64)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(L.ReadmeError):  # rows that do not begin at 16 bytes
        L.readme_rotary(torch.randn(4, 129, device="cuda:0")[:, 1:], pos, freqs, 64)
