"""Float64 definitions of the recurrent block's operators: the norms of a voxel's
channels before and behind a block, and the gated linear recurrence along the voxels.
Everything is written from the formulas, in numpy; maps are [n][c][v].
"""
import numpy as np


def sigmoid(x):
    """1 / (1 + exp(-x)) without overflow."""
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def gate(g, kind):
    """(phi, its derivative); kind: None, "sigmoid" or "silu"."""
    if kind is None:
        return 1.0, None
    s, rest = sigmoid(g), sigmoid(-g)
    if kind == "sigmoid":
        return s, s * rest
    return g * s, s * (1.0 + g * rest)


def _live(mask, *maps):
    """The maps with zeros at masked voxels."""
    if mask is None:
        return maps
    on = (mask != 0)[:, None, :]
    return tuple(None if m is None else np.where(on, m, 0.0) for m in maps)


def _col(v):
    return 1.0 if v is None else v[:, None]


def inv_rms(x, eps):
    return 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)


def pre_norm(x, gamma, mask, eps):
    x, = _live(mask, x)
    return x * inv_rms(x, eps) * _col(gamma)


def pre_norm_bwd(du, x, gamma, mask, eps):
    """(dx without the residual's, dgamma)"""
    du, x = _live(mask, du, x)
    r = inv_rms(x, eps)
    e = du * _col(gamma)
    return r * (e - x * r * r * (e * x).mean(1, keepdims=True)), (du * x * r).sum((0, 2))


def post_norm(x, z, g, kind, gamma, scale, gamma_next, mask, eps):
    """(y, u or None)"""
    z, g = _live(mask, z, g)
    branch = _col(scale) * gate(g, kind)[0] * _col(gamma) * z * inv_rms(z, eps)
    y = x + _live(mask, branch)[0]
    return y, None if gamma_next is None else pre_norm(y, gamma_next, mask, eps)


def post_norm_bwd(dy, du, y, z, g, kind, gamma, scale, gamma_next, mask, eps):
    """{dx, dz, dg, dgamma, dscale, dgamma_next}, the last and dg only where they exist"""
    out = {}
    if gamma_next is not None:
        more, out["dgamma_next"] = pre_norm_bwd(du, y, gamma_next, mask, eps)
        dy = dy + more
    out["dx"] = dy
    d, z, g = _live(mask, dy, z, g)
    phi, slope = gate(g, kind)
    zr = z * inv_rms(z, eps)
    out["dgamma"] = (d * _col(scale) * phi * zr).sum((0, 2))
    out["dscale"] = (d * _col(gamma) * phi * zr).sum((0, 2))
    e = d * _col(scale) * _col(gamma)
    if kind is not None:
        out["dg"] = e * zr * slope
    out["dz"] = pre_norm_bwd(e * phi, z, None, mask, eps)[0]
    return out


def _steps(r, i, x, lam, mask, rate):
    """Decay, input and its factors of every voxel; masked ones hand the state on."""
    r, i, x = _live(mask, r, i, x)
    w = rate * np.logaddexp(0.0, lam)[:, None]
    la, = _live(mask, -w * sigmoid(r))
    beta = np.sqrt(-np.expm1(2 * la))  # 0 where masked
    return la, np.exp(la), beta, sigmoid(i), x


def walk(a, b, h, order):
    """h = a_t h + b_t over the voxels t in `order`: the states behind and before each
    step, and the last."""
    a, b = (np.ascontiguousarray(np.moveaxis(t, 2, 0)) for t in (a, b))
    after, before = np.empty_like(a), np.empty_like(a)
    for t in order:
        before[t] = h
        h = a[t] * h + b[t]
        after[t] = h
    return np.moveaxis(after, 0, 2), np.moveaxis(before, 0, 2), h


def order_of(v, reverse):
    return range(v - 1, -1, -1) if reverse else range(v)


def recurrence(r, i, x, lam, mask, h0, rate, reverse):
    """(y, state behind the walk, the states before each voxel's step)"""
    n, c, v = r.shape
    _, a, beta, si, x = _steps(r, i, x, lam, mask, rate)
    h, past, last = walk(a, beta * si * x, np.zeros((n, c)) if h0 is None else h0,
                         order_of(v, reverse))
    return _live(mask, h)[0], last, past


def recurrence_bwd(dy, dh, r, i, x, lam, mask, past, rate, reverse):
    """{dr, di, dx, dlam, dh0, state: the gradient of each voxel's state}"""
    n, c, v = r.shape
    dy, = _live(mask, dy)
    la, a, beta, si, xl = _steps(r, i, x, lam, mask, rate)
    # what reaches a state from behind: back_t = a_t (dy_t + back_{t+1})
    _, behind, dh0 = walk(a, a * dy, np.zeros((n, c)) if dh is None else dh,
                          order_of(v, not reverse))
    d = dy + behind
    with np.errstate(divide="ignore", invalid="ignore"):
        dbeta = np.where(beta > 0, -a * a / beta, 0.0)  # by la; a shut gate passes nothing on
    r, i = _live(mask, r, i)
    soft = np.logaddexp(0.0, lam)[:, None]
    dla, = _live(mask, d * (past * a + si * xl * dbeta))
    out = dict(dr=dla * -rate * soft * sigmoid(r) * sigmoid(-r),
               dlam=(dla * -rate * sigmoid(r) * sigmoid(lam)[:, None]).sum((0, 2)),
               di=d * beta * xl * si * sigmoid(-i), dx=d * beta * si, dh0=dh0)
    out["state"] = d
    return out
