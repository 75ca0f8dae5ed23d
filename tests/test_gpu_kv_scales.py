"""Attention over the 8-bit cache where blocks' value scales lie far apart: the
stated bound is of the largest |v| that a row sees, whatever the scales of
blocks that it does not see, or of which it sees only small codes."""
import numpy as np
import pytest
import torch

from oracle import kv_cache as ok
from tests.test_gpu_kv import KT, Cache, _i32, _lib, _offsets, _random_cache

pytestmark = pytest.mark.gpu

# Sizes at which the launch takes each form: new rows and tokens of a request,
# requests, key heads, query heads a key head, blocks of the table, a window
# that the first rows of a request still reach block 0 through and the last do
# not.  Several blocks of a request go to one wave in all of them.
FORMS = {
    "rows/1": (32, 80, 256, 4, 1, 2, 16),
    "rows/8": (16, 592, 2, 2, 1, 10, 520),
    "rows/0": (16, 4076, 3, 2, 1, 66, 4000),
    "tiles/0": (40, 4090, 3, 2, 1, 67, 4000),
    "tiles/1": (80, 150, 30, 3, 4, 6, 16),
}


def _set(c, scales=None, codes=None):
    if codes is not None:
        c.ref["codes"] = codes
        c.codes.copy_(torch.from_numpy(ok.to_bytes(c.kt, codes)))
    if scales is not None:
        c.ref["scales"] = scales
        c.scales.copy_(torch.from_numpy(scales))


def _check(c, new, lens, H, window=0, scale=None, causal=True, q_scale=1.0):
    """The bound of the header: bf16's half step of the result; of max |v|, fp16's
    half step of every weight, 2^-24 for each weight below its normal numbers, and
    twice the relative error of the weights and their sum (fp32 scores of D
    products, exp2)."""
    off, T, D = _offsets(new), int(sum(new)), c.D
    q = torch.from_numpy(c.rng.standard_normal((T, H, D)) * q_scale).bfloat16()
    scale = D ** -0.5 if scale is None else scale
    o = _lib().readme_attention_kv(KT[c.kt], q.reshape(T, -1).cuda(), _i32(off), _i32(lens), *c.args(),
                                   H=H, scale=scale, causal=causal, window=window)
    ref, vmax, zabs = ok.attention(c.ref, q.double().numpy(), off, lens, c.table,
                                   float(np.float32(scale)), causal, window)
    got = o.cpu().double().numpy().reshape(T, H, D)
    assert np.isfinite(got).all()
    delta = (D + 8) * 2.0 ** -24 * zabs + 2.0 ** -18
    tol = 2.0 ** -8 * np.abs(ref) + ((2.0 ** -11 + max(lens) * 2.0 ** -24 + 2 * delta) * vmax)[..., None]
    err = np.abs(got - ref)
    bad = err > tol
    assert not bad.any(), f"{bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: " \
                          f"{got[bad][0]} for {ref[bad][0]}"


def _of_form(form, kt, D):
    new, ln, R, Hk, G, mb, window = FORMS[form]
    c = _random_cache(kt, R, Hk, D, mb, seed=70)
    return c, [new] * R, [ln] * R, Hk * G, window


TYPES = [("i8", 64), ("e4m3", 128)]


@pytest.mark.parametrize("kt,D", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_a_block_past_the_window(form, kt, D):
    """Block 0 holds values 2^36 times the others'; the window hides it from the
    last rows and shows it, in part or whole, to the first of the same tile."""
    c, new, lens, H, window = _of_form(form, kt, D)
    sc = c.ref["scales"].copy()
    sc[c.table[:, 0], :, 1] *= np.float32(2.0 ** 36)
    _set(c, sc)
    _check(c, new, lens, H, window)


@pytest.mark.parametrize("kt,D", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_large_scales_of_small_codes(form, kt, D):
    """Every third block has a value scale 2^36 times its neighbours' and codes
    that are all zero (what a rejected draft of large values leaves)."""
    c, new, lens, H, _ = _of_form(form, kt, D)
    sc, codes = c.ref["scales"].copy(), c.ref["codes"].copy()
    R, mb = c.table.shape
    quiet = c.table[(np.arange(R)[:, None] + np.arange(mb)) % 3 == 0]
    sc[quiet, :, 1] *= np.float32(2.0 ** 36)
    codes[quiet, :, 1] = 0.0
    _set(c, sc, codes)
    _check(c, new, lens, H)


@pytest.mark.parametrize("kt,D", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_scales_at_both_ends(form, kt, D):
    """Value scales 2^-90 and 2^85 in turn: rows that see only the small ones
    share a tile with rows that see both."""
    c, new, lens, H, window = _of_form(form, kt, D)
    sc = c.ref["scales"].copy()
    sc[c.table[:, 0::2].reshape(-1), :, 1] *= np.float32(2.0 ** -90)
    sc[c.table[:, 1::2].reshape(-1), :, 1] *= np.float32(2.0 ** 85)
    _set(c, sc)
    _check(c, new, lens, H)
    _check(c, new, lens, H, window)


@pytest.mark.parametrize("kt,D", TYPES)
@pytest.mark.parametrize("form", ["rows/0", "tiles/0"])
def test_scales_that_fall_and_rise(form, kt, D):
    """Value scales from 2^20 down to 2^-20 and back along each request, half of
    the codes of the larger ones zero."""
    c, new, lens, H, window = _of_form(form, kt, D)
    sc, codes = c.ref["scales"].copy(), c.ref["codes"].copy()
    mb = c.table.shape[1]
    for j in range(mb):
        sc[c.table[:, j], :, 1] *= np.float32(2.0 ** (40 * abs(j / (mb - 1) - 0.5) * 2 - 20))
        if j % 3:
            codes[c.table[:, j], :, 1, :, ::2] = 0.0
    _set(c, sc, codes)
    _check(c, new, lens, H)
    _check(c, new, lens, H, 70)


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
@pytest.mark.parametrize("new", [1, 6])
def test_a_rejected_outlier(kt, new):
    """A drafted token of 2^30 is written, rejected and overwritten: its block
    keeps the scale, the later ones have their own."""
    c = Cache(kt, 2, 1, 64, 6, seed=71)
    big = torch.full((2, 1, 64), 2.0 ** 30).bfloat16()
    c.write([40, 40], [40, 40], torch.bfloat16)
    c.write([1, 1], [41, 41], torch.bfloat16, big, big)
    c.write([300, 220 + new], [340, 260 + new], torch.bfloat16)
    _check(c, [new] * 2, [340, 260 + new], 2, scale=2.0 ** -40)


@pytest.mark.parametrize("kt,D", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_values_near_the_largest(form, kt, D):
    """Values up to 2^126: the rows are finite, though their sums before the
    division by the weights' are not."""
    c, new, lens, H, window = _of_form(form, kt, D)
    sc = c.ref["scales"].copy()
    sc[..., 1] *= np.float32(2.0 ** 118)
    _set(c, sc)
    _check(c, new, lens, H)
    _check(c, new, lens, H, window)


@pytest.mark.parametrize("small", [0.0, 1e-40, 2.0 ** -120])
@pytest.mark.parametrize("form", FORMS)
def test_scales_under_the_writes(form, small):
    """Value scales below those that readme_kv_write gives (2^-100), zero and a
    subnormal among them, beside its smallest."""
    c, new, lens, H, _ = _of_form(form, "i8", 64)
    sc = c.ref["scales"].copy()
    sc[..., 1] = np.float32(2.0 ** -100)
    sc[c.table[:, 1::3].reshape(-1), :, 1] = np.float32(small)
    _set(c, sc)
    _check(c, new, lens, H)


@pytest.mark.parametrize("qe,scale,ke", [(-38, 2.0 ** -60, 94), (60, 2.0 ** -40, -24), (-95, 1.0, 92)])
@pytest.mark.parametrize("form", ["rows/8", "tiles/1"])
def test_scores_of_far_apart_factors(form, qe, scale, ke):
    """Queries, keys and the softmax scale far from one, their scores of order one:
    the largest element of a row, and that times scale, from 2^-100 on."""
    c, new, lens, H, _ = _of_form(form, "i8", 64)
    sc = c.ref["scales"].copy()
    sc[..., 0] *= np.float32(2.0 ** ke)
    _set(c, sc)
    _check(c, new, lens, H, scale=scale, q_scale=2.0 ** qe)
