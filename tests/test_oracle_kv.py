"""Pins of the 8-bit cache's oracle: closed forms, torch's own conversions and
brute force, on the CPU."""
import math

import numpy as np
import pytest
import torch

from oracle import kv_cache as ok


def test_e4m3_values_are_torchs():
    b = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ok.e4m3_values(), b)


def test_nearest_e4m3_is_torchs_conversion():
    rng = np.random.default_rng(0)
    x = np.float32(rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 8, 20000)).clip(-448, 448)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(ok.nearest("e4m3", x.astype(np.float64)), ref)


def test_nearest_ties_and_limits():
    q = np.array([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, 127.4, 300.0])
    np.testing.assert_array_equal(ok.nearest("i8", q), [0, 2, 2, 0, -2, 126, 127, 127])
    # Between 16 (mantissa 0) and 18 (mantissa 1), between 18 and 20, the
    # smallest step's half, and past the largest
    q = np.array([17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, 500.0, -17.0])
    np.testing.assert_array_equal(ok.nearest("e4m3", q),
                                  [16, 20, 0, 2.0 ** -8, 448, -16])


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
@pytest.mark.parametrize("D", [64, 128])
def test_byte_layout_round_trip(kt, D):
    rng = np.random.default_rng(1)
    raw = rng.integers(0, 127, (2, 3, 2, 64 * D)).astype(np.uint8)
    codes = ok.from_bytes(kt, raw, D)
    np.testing.assert_array_equal(ok.to_bytes(kt, codes), raw)
    # The stated byte of one key and one value
    n, h, t, d = 1, 2, 45, 37
    kb = ((t // 32) * (D // 16) + d // 16) * 512 + (t % 32) * 16 + d % 16
    vb = ((t // 32) * D + d) * 32 + t % 32
    val = (lambda b: float(b) - 128) if kt == "i8" else (lambda b: ok.e4m3_values()[b])
    assert codes[n, h, 0, t, d] == val(raw[n, h, 0, kb])
    assert codes[n, h, 1, t, d] == val(raw[n, h, 1, vb])


def _one(kt, rows, steps):
    """Writes rows [n][D] of one request in pieces of the given sizes."""
    c = ok.new_cache(1, 1, rows.shape[1])
    at = 0
    for n in steps:
        x = rows[at:at + n][:, None]
        at += n
        ok.write(kt, c, x, x, np.array([0, n]), np.array([at]), np.array([[0]]))
    return c


def test_growth_by_hand():
    """Scale 1 (row of 127), then 200 (doubling: need 200/127 <= 2), then 20
    (no growth): codes 127 -> 63.5 -> tie to 64, 3 -> 1.5 -> 2, 5 -> 2.5 -> 2."""
    rows = np.zeros((3, 64))
    rows[0, :3] = [127, 3, 5]
    rows[1, :2] = [200, 7]
    rows[2, 0] = 21
    c = _one("i8", rows, [1, 1, 1])
    assert c["scales"][0, 0, 0] == 2.0
    np.testing.assert_array_equal(c["codes"][0, 0, 0, :3, :3],
                                  [[64, 2, 2], [100, 4, 0], [10, 0, 0]])


@pytest.mark.parametrize("kt", ["i8", "e4m3"])
def test_a_value_never_drifts_a_whole_step(kt):
    """Rows growing by 5% each, one at a time: every earlier value stays within
    one step of the final scale (I8), and E4M3 within its own relative half step
    and half the smallest step."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((64, 64)) * 1.05 ** np.arange(64)[:, None]
    c = _one(kt, x, [1] * 64)
    s = float(c["scales"][0, 0, 0])
    err = np.abs(c["codes"][0, 0, 0] * s - x)
    if kt == "i8":
        assert err.max() < s
    else:
        assert (err <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -9 * s)).all()


def test_whole_block_is_the_tight_scale():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((64, 64))
    c = _one("i8", x, [64])
    s = np.float32(np.abs(x).max() / 127)
    assert c["scales"][0, 0, 0] == s
    np.testing.assert_allclose(c["codes"][0, 0, 1] * float(s), x, atol=float(s) / 2 * (1 + 1e-6))


def test_writing_again_changes_nothing():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((40, 64)) * np.linspace(1, 9, 40)[:, None]
    c = _one("e4m3", x, [13, 27])
    before = {k: v.copy() for k, v in c.items()}
    y = x[13:][:, None]
    ok.write("e4m3", c, y, y, np.array([0, 27]), np.array([40]), np.array([[0]]))
    for k in c:
        np.testing.assert_array_equal(c[k], before[k])


def test_attention_closed_forms():
    """Equal keys give the mean of the values seen; a row before the cache's
    first token, or with every block absent, is zeros; torch's softmax agrees."""
    rng = np.random.default_rng(5)
    D, ln = 64, 70
    c = ok.new_cache(2, 1, D)
    c["scales"][:] = 0.5
    c["codes"][:, :, 1] = rng.integers(-127, 128, (2, 1, 64, D))
    table = np.array([[1, 0]])
    v = np.concatenate([c["codes"][1, 0, 1], c["codes"][0, 0, 1]])[:ln] * 0.5
    q = rng.standard_normal((3, 1, D))
    o, _, _ = ok.attention(c, q, np.array([0, 3]), np.array([ln]), table, 0.1)
    for i in range(3):
        np.testing.assert_allclose(o[i, 0], v[:ln - 2 + i].mean(0), rtol=1e-12)
    o, _, _ = ok.attention(c, q, np.array([0, 3]), np.array([ln]), table, 0.1, window=4)
    np.testing.assert_allclose(o[2, 0], v[-4:].mean(0), rtol=1e-12)
    o, _, _ = ok.attention(c, q, np.array([0, 3]), np.array([1]), table, 0.1)
    assert (o[:2] == 0).all()
    np.testing.assert_allclose(o[2, 0], v[0], rtol=1e-12)
    o, _, _ = ok.attention(c, q, np.array([0, 3]), np.array([ln]), np.array([[-1, 2]]), 0.1)
    assert (o == 0).all()
    c["codes"][:, :, 0] = rng.integers(-127, 128, (2, 1, 64, D))
    k = np.concatenate([c["codes"][1, 0, 0], c["codes"][0, 0, 0]])[:ln] * 0.5
    o, _, _ = ok.attention(c, q, np.array([0, 3]), np.array([ln]), table, 0.02, causal=False)
    z = torch.softmax(torch.from_numpy(q[:, 0] @ k.T * 0.02), 1) @ torch.from_numpy(v)
    np.testing.assert_allclose(o[:, 0], z.numpy(), rtol=1e-10, atol=1e-12)


def test_read_of_absent_positions():
    c = ok.new_cache(1, 2, 64)
    c["codes"][:] = 3.0
    c["scales"][:] = 2.0
    k, v = ok.read(c, 6, np.array([0, 2, 5]), np.array([1, 66]), np.array([[0, -1], [0, 0]]), 7.0)
    assert (k[0] == 0).all() and (k[1] == 6).all()      # position -1, then 0
    assert (v[2:5] == 6).all() and (v[5] == 7).all()    # row 5 belongs to no request
    assert math.isclose(k[2, 0, 0], 6.0)
