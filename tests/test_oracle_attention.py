"""The float64 definitions of the voxel self-attention operators: closed forms,
published values, invariants and finite differences."""
import numpy as np
import pytest

from oracle import attention as A

RNG = np.random.default_rng


def test_philox_published_vectors():
    """The known-answer values of Philox4x32-10."""
    assert A.philox((0, 0, 0, 0), (0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    f = 0xffffffff
    assert A.philox((f, f, f, f), (f, f)) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert A.philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) \
        == [0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


def test_dropout_rate_and_units():
    keep, scale = A.keeps(20000, 0.3, 7, 1)
    assert abs(keep.mean() - 0.7) < 5 * np.sqrt(0.21 / 20000)
    assert scale == pytest.approx(1 / 0.7, rel=2e-5)
    assert not np.array_equal(keep, A.keeps(20000, 0.3, 7, 2)[0])
    assert not np.array_equal(keep, A.keeps(20000, 0.3, 8, 1)[0])
    y = A.dropout(np.ones((4, 6)), 6, 0.5, 3, 0)
    assert all(len(set(r)) == 1 for r in y)
    assert np.all(A.dropout(np.ones(9), 1, 1.0, 3, 0) == 0)
    assert np.all(A.dropout(np.ones(9), 1, 0.0, 3, 0) == 1)


def test_rotation_is_orthogonal_and_relative():
    """Turning is orthogonal, and scores depend on the difference of places."""
    t = A.rotation(14, (3, 4, 5), (4, 4, 4), (0, 0, 0), 100.0)
    np.testing.assert_allclose(np.matmul(t, t.swapaxes(1, 2)), np.broadcast_to(np.eye(14), t.shape),
                               atol=1e-14)
    far = A.rotation(14, (3, 4, 5), (4, 4, 4), (50, 7, 900), 100.0)
    q, k = RNG(0).standard_normal((2, 14))
    s = np.einsum("vab,b,wac,c->vw", t, q, t, k)
    np.testing.assert_allclose(s, np.einsum("vab,b,wac,c->vw", far, q, far, k), atol=1e-11)
    # the pair (0, 2) of the first axis at place 2: an angle of 2
    z = A.qk_fwd(np.eye(14)[0].reshape(1, 14, 1).repeat(60, 2), 1, None, t, 0.0)
    np.testing.assert_allclose(z[0, [0, 2], 59], [np.cos(2), np.sin(2)], atol=1e-15)


def _diff(f, x, g, h=1e-6, picks=12, seed=0):
    """Central differences of f at some entries of x against the gradient g."""
    for i in RNG(seed).choice(x.size, min(picks, x.size), replace=False):
        old = x.flat[i]
        x.flat[i] = old + h
        up = f()
        x.flat[i] = old - h
        down = f()
        x.flat[i] = old
        assert (up - down) / (2 * h) == pytest.approx(g.flat[i], rel=1e-5, abs=1e-7)


def test_qk_gradient_differences():
    r = RNG(1)
    turn = A.rotation(9, (2, 2, 3), (2, 4, 2), (1, 0, 5), 50.0)
    x, dy, g = r.standard_normal((2, 18, 12)), r.standard_normal((2, 18, 12)), r.standard_normal(9)
    dx, dg = A.qk_bwd(dy, x, 2, g, turn, 1e-3)
    f = lambda: float((A.qk_fwd(x, 2, g, turn, 1e-3) * dy).sum())  # noqa: E731
    _diff(f, x, dx)
    _diff(f, g, dg)


def test_attention_closed_forms():
    r = RNG(2)
    v = r.standard_normal((2, 6, 11))
    # equal scores: the mean of the live values
    mask = np.ones((2, 11), np.uint8)
    mask[0, 3:7] = 0
    mask[1] = 0
    o, lse, _ = A.attention(np.zeros((2, 6, 4)), r.standard_normal((2, 6, 11)), v, 2, 2, mask, 1.0)
    live = np.flatnonzero(mask[0])
    np.testing.assert_allclose(o[0], np.repeat(v[0][:, live].mean(1)[:, None], 4, 1), atol=1e-15)
    assert np.all(o[1] == 0) and np.all(np.isneginf(lse[1]))
    np.testing.assert_allclose(lse[0], np.log(7.0))
    # one key: its value, whatever the score
    o, lse, p = A.attention(r.standard_normal((1, 3, 5)), np.ones((1, 3, 1)), v[:1, :3, :1], 1, 1,
                            None, 0.7)
    np.testing.assert_allclose(o[0], np.repeat(v[0, :3, :1], 5, 1))
    assert np.all(p == 1)


def test_attention_ignores_masked_values():
    r = RNG(3)
    q, k, v = r.standard_normal((1, 4, 3)), r.standard_normal((1, 4, 6)), r.standard_normal((1, 4, 6))
    mask = np.array([[1, 0, 1, 1, 0, 1]], np.uint8)
    a = A.attention(q, k, v, 2, 1 * 2, mask, 0.5)[0]
    k[0, :, 1], v[0, :, 4] = np.nan, np.inf
    np.testing.assert_array_equal(a, A.attention(q, k, v, 2, 2, mask, 0.5)[0])


def test_attention_gradient_differences():
    r = RNG(4)
    q, k, v = (r.standard_normal((2, c * 5, t)) for c, t in ((4, 7), (2, 9), (2, 9)))
    do = r.standard_normal(q.shape)
    mask = (r.random((2, 9)) < 0.7).astype(np.uint8)
    mask[:, 0] = 1
    p = A.attention(q, k, v, 4, 2, mask, 0.6)[2]
    grads = A.attention_bwd(do, q, k, v, 4, 2, mask, 0.6, p)
    f = lambda: float((A.attention(q, k, v, 4, 2, mask, 0.6)[0] * do).sum())  # noqa: E731
    for x, g in zip((q, k, v), grads):
        _diff(f, x, g)
    assert np.all(grads[1].transpose(0, 2, 1)[mask == 0] == 0)


def test_attention_against_autograd():
    torch = pytest.importorskip("torch")
    r = RNG(5)
    q, k, v = (torch.from_numpy(r.standard_normal((1, 3 * 4, t))).requires_grad_() for t in (6, 8, 8))
    hs = [t.view(1, 3, 4, -1).transpose(2, 3) for t in (q, k, v)]
    o = (torch.softmax(hs[0] @ hs[1].transpose(2, 3) * 0.4, -1) @ hs[2]).transpose(2, 3).reshape(1, 12, 6)
    do = torch.from_numpy(r.standard_normal((1, 12, 6)))
    o.backward(do)
    a = [t.detach().numpy() for t in (q, k, v)]
    mine, _, p = A.attention(*a, 3, 3, None, 0.4)
    np.testing.assert_allclose(mine, o.detach().numpy(), atol=1e-13)
    for g, t in zip(A.attention_bwd(do.numpy(), *a, 3, 3, None, 0.4, p), (q, k, v)):
        np.testing.assert_allclose(g, t.grad.numpy(), atol=1e-13)
