"""readme_attention_kv_tree under a window that hides tokens and still leaves more
blocks than a workgroup takes by itself: the work is dealt in shares, from a block
other than a request's first on."""
import numpy as np
import pytest
import torch

from oracle import drafts as od
from tests.kv_forms import Size
from tests.test_gpu_kv import KT, _i32, _offsets, _poison_unused, _random_cache
from tests.test_gpu_kv_tree import _masks, form

pytestmark = pytest.mark.gpu

_LENS = [7000, 5230, 300, 6401]
# Named after the form that each takes; a request of no rows, and one that the window
# hides nothing of
SIZES = {
    ("16/0", 128): Size([8, 3, 0, 5], _LENS, 2, 2, 110), ("16/0", 64): Size([5, 0, 7, 1], _LENS, 2, 3, 110),
    ("16/0", 256): Size([8, 3, 0, 5], _LENS, 1, 2, 110), ("32/0", 128): Size([24, 30, 0, 20], _LENS, 1, 2, 110),
    ("32/0", 64): Size([40, 0, 33, 64], _LENS, 2, 1, 110), ("128/0", 128): Size([40, 30, 0, 65], _LENS, 1, 3, 110),
    ("128/0", 64): Size([70, 1, 33, 0], _LENS, 1, 5, 110), ("128/0", 256): Size([24, 0, 9, 40], _LENS, 1, 2, 110),
}


@pytest.mark.parametrize("window", [4500, 6000])
@pytest.mark.parametrize("name,D", SIZES)
def test_sizes_take_the_form_they_are_named_after(name, D, window):
    assert form(SIZES[name, D], D, window) == name


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("window", [4500, 6000])
@pytest.mark.parametrize("name,D", SIZES)
def test_shares_under_a_window(name, D, window, given):
    """Positions of the stored rows, and given ones: near the first row, thousands past
    it, and beyond every other."""
    from paper_2410_19123_amd import _lib as L
    s = SIZES[name, D]
    c = s.cache(_random_cache, "e4m3" if D == 128 else "i8", D, 190 + window)
    _poison_unused(c, s.lens)
    off, T, H = _offsets(s.new), sum(s.new), s.Hk * s.G
    pos = None
    if given:
        first = np.concatenate([np.full(n, ln - n) for n, ln in zip(s.new, s.lens)])
        pos = first + c.rng.integers(-9, 60, T) + (c.rng.random(T) < 0.5) * c.rng.integers(0, 5000, T)
        pos[::17] = 2 ** 31 - 1
        pos[5::19] = -2 ** 31
    masks, words = _masks(c.rng, s.new), 2
    q = torch.from_numpy(c.rng.standard_normal((T, H, D)) * 1.5).bfloat16()
    o = L.readme_attention_kv_tree(KT[c.kt], q.reshape(T, -1).cuda(), _i32(off), _i32(s.lens), *c.args(), H,
                                   torch.from_numpy(od.words(masks, words)).cuda(),
                                   None if pos is None else _i32(pos), window=window)
    got = o.cpu().double().numpy().reshape(T, H, D)
    ref, vmax, zabs = od.attention_tree(c.ref, q.double().numpy(), off, s.lens, c.table, masks,
                                        float(np.float32(D ** -0.5)), pos, window, words)
    # As for shorter calls (tests.test_gpu_kv), and the running sums of as many blocks
    delta = (D + 8) * 2.0 ** -24 * zabs + 2.0 ** -18 + 2.0 ** -24 * (64 + max(s.lens) / 64)
    tol = 2.0 ** -8 * np.abs(ref) + ((2.0 ** -11 + 2 * delta) * vmax)[..., None]
    assert np.isfinite(got).all()
    assert (np.abs(got - ref) <= tol).all(), (np.abs(got - ref) - tol).max()
