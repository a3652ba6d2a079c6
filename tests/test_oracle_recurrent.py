"""The float64 definitions of the recurrent block's operators: closed forms, invariants
and finite differences."""
import numpy as np
import pytest

from oracle import recurrent as Q

RNG = np.random.default_rng
GATES = [None, "sigmoid", "silu"]


def _diff(f, x, g, h=1e-6, picks=10, seed=0):
    """Central differences of f at some entries of x against the gradient g."""
    for i in RNG(seed).choice(x.size, min(picks, x.size), replace=False):
        old = x.flat[i]
        x.flat[i] = old + h
        up = f()
        x.flat[i] = old - h
        down = f()
        x.flat[i] = old
        assert (up - down) / (2 * h) == pytest.approx(g.flat[i], rel=2e-5, abs=1e-7)


def test_norm_closed_forms():
    x = np.full((1, 4, 3), 3.0)
    np.testing.assert_allclose(Q.pre_norm(x, np.arange(4.0), None, 7.0),
                               np.arange(4.0)[None, :, None] * 0.75 * np.ones((1, 4, 3)))
    y, u = Q.post_norm(x, 2 * x, np.zeros_like(x), "sigmoid", np.full(4, 2.0), np.full(4, 5.0),
                       np.ones(4), None, 0.0)
    np.testing.assert_allclose(y, 8.0)  # 3 + 5 * 1/2 * 2 * 1
    np.testing.assert_allclose(u, 1.0)
    # a norm's gradient is at right angles to its input where eps is 0
    r = RNG(0)
    x, du = r.standard_normal((2, 2, 5, 7))
    dx, _ = Q.pre_norm_bwd(du, x, None, None, 0.0)
    np.testing.assert_allclose((dx * x).sum(1), 0.0, atol=1e-13)


@pytest.mark.parametrize("kind", GATES)
@pytest.mark.parametrize("nxt", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_post_norm_differences(kind, nxt, masked):
    r = RNG(3)
    n, c, v, eps = 2, 5, 4, 1e-3
    x, z, g, dy, du = r.standard_normal((5, n, c, v))
    gamma, scale, gn = 1 + 0.3 * r.standard_normal((3, c))
    mask = (r.random((n, v)) < 0.6).astype(np.uint8) if masked else None
    if masked:
        mask[1] = 0
    gn = gn if nxt else None

    def value():
        y, u = Q.post_norm(x, z, g, kind, gamma, scale, gn, mask, eps)
        return float((y * dy).sum() + ((u * du).sum() if nxt else 0.0))

    y, _ = Q.post_norm(x, z, g, kind, gamma, scale, gn, mask, eps)
    d = Q.post_norm_bwd(dy, du, y, z, g, kind, gamma, scale, gn, mask, eps)
    for t, name in ((x, "dx"), (z, "dz"), (gamma, "dgamma"), (scale, "dscale")):
        _diff(value, t, d[name])
    if kind:
        _diff(value, g, d["dg"])
    if nxt:
        _diff(value, gn, d["dgamma_next"])


def test_pre_norm_differences():
    r = RNG(4)
    x, du = r.standard_normal((2, 2, 6, 5))
    gamma = 1 + 0.3 * r.standard_normal(6)
    mask = np.array([[1, 0, 1, 1, 0], [0, 0, 0, 0, 1]], np.uint8)
    f = lambda: float((Q.pre_norm(x, gamma, mask, 1e-3) * du).sum())  # noqa: E731
    dx, dg = Q.pre_norm_bwd(du, x, gamma, mask, 1e-3)
    _diff(f, x, dx)
    _diff(f, gamma, dg)
    assert np.all(dx[0, :, 1] == 0)


def test_recurrence_closed_forms():
    one = np.ones((1, 2, 6))
    # an open gate that forgets everything: h = sigmoid(i) x
    lam = np.full(2, 100.0)
    y, last, _ = Q.recurrence(50 * one, 0 * one, 3 * one, lam, None, None, 8.0, False)
    np.testing.assert_allclose(y, 1.5)
    # a shut gate keeps the state
    h0 = np.array([[2.0, -1.0]])
    y, last, past = Q.recurrence(-800 * one, 0 * one, 3 * one, lam, None, h0, 8.0, False)
    np.testing.assert_allclose(last, h0)
    np.testing.assert_allclose(past, h0[..., None] * one)
    # equal steps: a geometric sum
    lam, r = np.zeros(2), 0 * one
    a = np.exp(-0.5 * np.log(2.0))
    b = np.sqrt(1 - a * a) * 0.5
    y, last, _ = Q.recurrence(r, 0 * one, one, lam, None, None, 1.0, False)
    np.testing.assert_allclose(y[0, 0], b * (1 - a ** np.arange(1, 7)) / (1 - a))
    # inputs of unit variance leave the state's variance at sigmoid(0)^2 in the long run
    x = RNG(0).standard_normal((1, 2, 20000))
    y, _, _ = Q.recurrence(0 * x, 0 * x, x, lam, None, None, 1.0, False)
    assert y[..., 100:].var() == pytest.approx(0.25, rel=0.05)
    # the other direction is the same walk on the turned map
    s = RNG(1).standard_normal((3, 2, 2, 9))
    m = (RNG(2).random((2, 9)) < 0.5).astype(np.uint8)
    y, last, _ = Q.recurrence(*s, lam, m, None, 2.0, True)
    z, last2, _ = Q.recurrence(*(t[..., ::-1] for t in s), lam, m[:, ::-1], None, 2.0, False)
    np.testing.assert_array_equal(y, z[..., ::-1])
    np.testing.assert_array_equal(last, last2)


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("masked", [False, True])
def test_recurrence_differences(reverse, masked):
    q = RNG(7)
    n, c, v, rate = 2, 3, 6, 1.5
    r, i, x, dy = q.standard_normal((4, n, c, v))
    lam, (h0, dh) = q.standard_normal(c), q.standard_normal((2, n, c))
    mask = np.array([[1, 0, 1, 1, 0, 1], [0] * 6], np.uint8) if masked else None

    def value():
        y, last, _ = Q.recurrence(r, i, x, lam, mask, h0, rate, reverse)
        return float((y * dy).sum() + (last * dh).sum())

    past = Q.recurrence(r, i, x, lam, mask, h0, rate, reverse)[2]
    d = Q.recurrence_bwd(dy, dh, r, i, x, lam, mask, past, rate, reverse)
    for t, name in ((r, "dr"), (i, "di"), (x, "dx"), (lam, "dlam"), (h0, "dh0")):
        _diff(value, t, d[name])
