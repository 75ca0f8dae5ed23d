"""The 64-bit form of a drafted step (oracle/drafts.py) against what has to hold of
it whatever the code: turns keep lengths and depend on differences of positions, a
chain's bits are causal attention, and verified drafts leave the target's own
distribution."""
import itertools

import numpy as np
import pytest

from oracle import drafts as od
from oracle import kv_cache as ok


@pytest.mark.parametrize("layout", ["half", "pairs"])
@pytest.mark.parametrize("D,rot", [(16, 16), (80, 32)])
def test_turns(layout, D, rot):
    rng = np.random.default_rng(D)
    f = od.rotary_freqs(rot)
    x = rng.standard_normal((6, 3, D))
    pos = np.array([0, 1, -1, 7, 4095, 131071])
    y = od.rotary(x, pos, f, layout)
    np.testing.assert_array_equal(y[0], x[0])
    np.testing.assert_array_equal(y[..., rot:], x[..., rot:])
    np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-12)
    np.testing.assert_allclose(od.rotary(y, pos, f, layout, inverse=True), x, atol=1e-12)
    # <turned q, turned k> depends on the difference of positions alone
    q, k = x[:1], x[1:2]
    at = lambda a, b: float((od.rotary(q, [a], f, layout) * od.rotary(k, [b], f, layout)).sum())  # noqa: E731
    assert at(5, 3) == pytest.approx(at(105, 103), abs=1e-9)
    # The pair of a layout: dim 0 of position 1 turns towards its partner
    e = np.zeros((1, 1, D))
    e[..., 0] = 1.0
    t = od.rotary(e, [1], f, layout)[0, 0]
    assert t[0] == pytest.approx(np.cos(1.0)) and t[rot // 2 if layout == "half" else 1] == \
        pytest.approx(np.sin(1.0))


def test_turn_gradient_is_the_inverse():
    rng = np.random.default_rng(1)
    f, x, g = od.rotary_freqs(16), rng.standard_normal((2, 1, 32)), rng.standard_normal((2, 1, 32))
    pos = [3, 50]
    value = lambda z: float((g * od.rotary(z, pos, f, "pairs", 1.3)).sum())  # noqa: E731
    grad = od.rotary(g, pos, f, "pairs", 1.3, inverse=True)
    # The unturned dims carry no amplitude
    for i in np.ndindex(x.shape):
        h = np.zeros_like(x)
        h[i] = 0.5
        assert value(x + h) - value(x - h) == pytest.approx(grad[i], abs=1e-12)


def test_frequencies():
    plain = od.rotary_freqs(64, 1e4)
    np.testing.assert_allclose(od.rotary_freqs(64, 1e4, "linear", 8.0) * 8, plain)
    banded = od.rotary_freqs(64, 1e4, "banded", 8.0, 4096.0, 1.0, 32.0)
    turns = 4096 * plain / (2 * np.pi)
    np.testing.assert_allclose(banded[turns >= 32], plain[turns >= 32])
    np.testing.assert_allclose(banded[turns <= 1] * 8, plain[turns <= 1])
    assert (np.diff(banded) < 0).all()


def test_host_frequencies():
    from paper_2410_19123_amd import _lib as L
    for kw, kind in ((dict(), "plain"), (dict(factor=4.0), "linear"),
                     (dict(factor=32.0, trained_len=8192.0, low=1.0, high=4.0), "banded")):
        got = L.readme_rotary_freqs(96, 5e5, {"plain": 0, "linear": 1, "banded": 2}[kind], **kw)
        np.testing.assert_allclose(got.numpy(), od.rotary_freqs(96, 5e5, kind, **kw), rtol=1e-14)


def test_a_chains_bits_are_causal_attention():
    rng = np.random.default_rng(2)
    cache = ok.new_cache(8, 2, 64)
    cache["codes"][:] = rng.integers(-127, 128, cache["codes"].shape)
    cache["scales"][:] = 0.01
    table = rng.permutation(8).reshape(2, 4).astype(np.int32)
    new, lens = [9, 70], [200, 70]
    off = np.array([0, 9, 79])
    q = rng.standard_normal((79, 4, 64))
    masks = od.bits([i - 1 for i in range(9)]) + od.bits([i - 1 for i in range(70)])
    for window in (0, 30):
        a = od.attention_tree(cache, q, off, lens, table, masks, 0.1, window=window, n_words=2)[0]
        b = ok.attention(cache, q, off, lens, table, 0.1, True, window)[0]
        rows = slice(0, 79) if window == 0 else slice(0, 9)  # own rows know no window
        np.testing.assert_allclose(a[rows], b[rows], rtol=1e-12, atol=1e-14)


def _marginal(p, q, kind, steps=40):
    """Distribution of the first token that comes out where two drafts below the
    root are drawn from q (`kind`: with or without replacement, or always the
    same two), the random numbers on a grid of midpoints."""
    V = len(p)
    out = np.zeros(V)
    grid = (np.arange(steps) + 0.5) / steps
    for x in itertools.product(range(V), repeat=2):
        if kind == "given":
            weight = q[x[0]] * q[x[1]]
        elif kind == "distinct":
            weight = 0.0 if x[0] == x[1] else q[x[0]] * q[x[1]] / (1 - q[x[0]])
        else:
            weight = float(x == (0, 2))
        if weight == 0.0:
            continue
        rows = np.stack([p, p, p])
        for u1, u2 in itertools.product(grid, repeat=2):
            for u0 in grid:
                _, acc, tok, _ = od.verify([0, 3], [0, x[0], x[1]], [0, 0, 0], rows,
                                           None if kind == "certain" else np.stack([q] * 3),
                                           [u0, u1, u2], kind == "distinct")
                if acc[0]:  # the draft itself comes out
                    first = x[0] if u1 * (1.0 if kind == "certain" else q[x[0]]) < p[x[0]] else x[1]
                    out[first] += weight / steps ** 2
                    break
                out[tok[0]] += weight / steps ** 3
    return out


@pytest.mark.parametrize("kind", ["given", "distinct", "certain"])
def test_what_comes_out_follows_the_target(kind):
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.25, 0.5, 0.25])
    # Each of three comparisons lies within half a step of its border's place
    np.testing.assert_allclose(_marginal(p, q, kind, 20), p, atol=3 * 0.5 / 20)


def test_verify_by_hand():
    p = np.array([[0.5, 0.5, 0, 0], [0, 0, 0.25, 0.75], [1.0, 0, 0, 0]])
    q = np.array([[0.25, 0.25, 0.5, 0], [0, 0, 0.5, 0.5], [0.25] * 4])
    tokens, parent = [0, 1, 2], [0, 0, 1]
    # Row 1 (token 1) taken as 0.9 * 0.25 < 0.5; row 2 (token 2): 0.6 * 0.5 >= 0.25
    # refused, left max(p - q, 0) = (0, 0, 0, 0.25): token 3
    path, acc, tok, _ = od.verify([0, 3], tokens, parent, p, q, [0.1, 0.9, 0.6])
    assert path.tolist() == [0, 1, -1] and acc[0] == 1 and tok[0] == 3
    # 0.4 * 0.5 < 0.25: both taken, then token 0 for certain
    path, acc, tok, _ = od.verify([0, 3], tokens, parent, p, q, [0.99, 0.9, 0.4])
    assert path.tolist() == [0, 1, 2] and acc[0] == 2 and tok[0] == 0
    # A border that the sum meets exactly belongs to the entry after it
    path, acc, tok, _ = od.verify([0, 1], [0], [0], p[:1], None, [0.5])
    assert acc[0] == 0 and tok[0] == 1
