"""Float64 references and element-wise bounds of the recurrent block's tests.

u is the largest relative error of one rounding to the storage type (half a step:
2^-8 bfloat16, 2^-24 float32), f = 2^-24 that of float32.  The bounds count every
rounding of the computation once, at its largest:
  a sum of K float32 terms                K f times the sum of magnitudes
  1/sqrt(mean of c squares + eps)         k = (c + 16) f relative, halved by the root and
                                          taken whole for the products with it
  sigmoid(v), and 1 - sigmoid(v) formed as exp(-v) sigmoid(v)
                                          (2 |v| + 10) f relative: exp's argument is
                                          rounded twice, exp, sum and quotient once to
                                          two units each
  an error e of a factor or a term        carried to the result by its derivative; 1.05
                                          covers products of errors
and one rounding to the storage type.  The recurrence's bound is itself a recurrence:
with M the state that magnitudes would give (M_t = a M_{t-1} + |b|), the state's error
is a times the old one's, plus a M_{t-1} times (the decay's relative error + 2 f for the
step), plus |b| times the input's relative error; the tree of joins over a block (eight
steps in a lane, six over the lanes, up to sixteen over waves, up to thirty between)
adds at most 64 f M.
"""
import numpy as np

from oracle import recurrent as Q
from tests import attn_util as AU

F, U, TINY = AU.F, AU.U, AU.TINY
# beta below 2^-63 may come out as p 2^63 (p = beta^2), and 1/beta is at most 2^63; a
# sigmoid below 2^-126 may come out as 0, and beta^2 is at most 2^10 times that
SHUT = 2.0 ** -58
within = AU.within


def _eps_sig(v):
    return (2 * np.abs(v) + 10) * F


def _stored(value, err, dt):
    return value, 1.05 * err + U[dt] * (np.abs(value) + 1.05 * err) + TINY


def _norm_bwd(du, x, gamma, mask, eps, edu=0.0):
    """Gradient through a norm and its error; du may carry the error edu."""
    du, x = Q._live(mask, du, x)
    k = (x.shape[1] + 16) * F
    r, g = Q.inv_rms(x, eps), np.abs(Q._col(gamma))
    dx, dg = Q.pre_norm_bwd(du, x, gamma, mask, eps)

    def mag(d):
        return r * (g * d + np.abs(x) * r * r * (g * d * np.abs(x)).mean(1, keepdims=True))

    terms = np.abs(du * x * r)
    # gains: up to 2^10 additions in a row in float32 (a thread's tokens, its tiles, the
    # tree over the lanes), the rest in float64
    return dx, 4 * k * mag(np.abs(du)) + mag(edu * np.ones_like(x)), dg, \
        ((k + 1024 * F) * terms).sum((0, 2)) + TINY


def pre_norm_refs(x, gamma, mask, eps, dt, du=None, dres=None):
    k = (x.shape[1] + 16) * F
    u = Q.pre_norm(x, gamma, mask, eps)
    out = dict(u=_stored(u, k * np.abs(u), dt))
    if du is not None:
        dx, e, dg, eg = _norm_bwd(du, x, gamma, mask, eps)
        res = 0.0 if dres is None else dres
        out["dx"] = _stored(dx + res, e + 2 * F * (np.abs(dx) + np.abs(res)), dt)
        out["dgamma"] = (dg, eg)
    return out


def post_norm_refs(x, z, g, kind, gamma, scale, gamma_next, mask, eps, dt):
    k = (z.shape[1] + 16) * F
    y, u = Q.post_norm(x, z, g, kind, gamma, scale, gamma_next, mask, eps)
    eg = 0.0 if kind is None else 2 * _eps_sig(Q._live(mask, g)[0])
    branch = np.abs(y - x)
    ey = branch * (k + eg + 8 * F) + 2 * F * (np.abs(x) + branch)
    out = dict(y=_stored(y, ey, dt))
    if u is not None:
        yl, eyl = Q._live(mask, y, ey)
        r = Q.inv_rms(yl, eps)
        er = r * r * (np.abs(yl) * eyl).mean(1, keepdims=True) + k
        out["u"] = _stored(u, np.abs(Q._col(gamma_next)) * r * (eyl + np.abs(yl) * er), dt)
    return out


def post_norm_bwd_refs(dy, du, y, z, g, kind, gamma, scale, gamma_next, mask, eps, dt):
    k = (z.shape[1] + 16) * F
    want = Q.post_norm_bwd(dy, du, y, z, g, kind, gamma, scale, gamma_next, mask, eps)
    out, eD = {}, np.zeros_like(dy)
    if gamma_next is not None:
        more, e, dg, eg = _norm_bwd(du, y, gamma_next, mask, eps)
        eD = e + 2 * F * (np.abs(dy) + np.abs(more))
        out["dgamma_next"] = (dg, eg)
    out["dx"] = _stored(want["dx"], eD, dt)
    d, e, zl, gl = Q._live(mask, want["dx"], eD, z, g)
    d = np.abs(d)
    phi, slope = Q.gate(gl, kind)
    phi = np.abs(phi)
    ephi = 0.0 if kind is None else 2 * _eps_sig(gl)
    zr = np.abs(zl * Q.inv_rms(zl, eps))
    v = np.abs(Q._col(scale) * Q._col(gamma))
    total = (e * phi * zr + d * phi * zr * (k + ephi + 1024 * F)).sum((0, 2)) + TINY
    one = np.ones(z.shape[1])
    out["dgamma"] = (want["dgamma"], 1.05 * total * np.abs(one if scale is None else scale))
    out["dscale"] = (want["dscale"], 1.05 * total * np.abs(gamma))
    if kind is not None:
        s, rest = Q.sigmoid(gl), Q.sigmoid(-gl)
        size = s * rest if kind == "sigmoid" else s + np.abs(gl) * s * rest
        es = 2 * _eps_sig(gl) * size
        out["dg"] = _stored(want["dg"], v * zr * (e * np.abs(slope) + d * (es + size * (k + 8 * F))),
                            dt)
    ee = v * (e * phi + d * phi * (ephi + 8 * F))
    signed = Q._live(mask, want["dx"])[0] * Q._col(scale) * Q._col(gamma) * Q.gate(gl, kind)[0]
    _, ez, _, _ = _norm_bwd(signed, zl, None, mask, eps, ee)
    out["dz"] = _stored(want["dz"], ez, dt)
    return out


def recurrence_refs(r, i, x, lam, mask, h0, rate, reverse, dt, dy=None, dh=None):
    """{name: (value, bound)} for y, h_last and, with dy, dr, di, dx, dlam, dh0."""
    y, last, past = Q.recurrence(r, i, x, lam, mask, h0, rate, reverse)
    n, c, v = r.shape
    rl, il, xl = Q._live(mask, r, i, x)
    on = np.ones((n, 1, v)) if mask is None else (mask != 0)[:, None, :].astype(np.float64)
    w = rate * np.logaddexp(0.0, lam)[:, None]
    la = -w * Q.sigmoid(rl) * on
    a, p = np.exp(la), -np.expm1(2 * la)
    beta = np.sqrt(p)
    e_la = _eps_sig(rl) + 18 * F
    e_a = np.abs(la) * (e_la + 2 * F) + 4 * F
    with np.errstate(divide="ignore", invalid="ignore"):
        steep = np.where(p > 0, 2 * np.abs(la) * a * a / p, 1.0)
        inv = np.where(p > 0, 1.0 / beta, 0.0)
    e_p = steep * (e_la + 2 * F) + 48 * F
    b = np.abs(Q.sigmoid(il) * xl) * on  # without beta
    e_b = e_p / 2 + _eps_sig(il) + 12 * F
    order, back = Q.order_of(v, reverse), Q.order_of(v, not reverse)
    zero = np.zeros((n, c))
    m, mp, ml = Q.walk(a, beta * b, zero if h0 is None else np.abs(h0), order)
    e, ep, el = Q.walk(a, a * mp * (e_a + 2 * F) + b * (beta * e_b + SHUT), zero, order)
    out = dict(y=_stored(y, (e + 64 * F * m) * on, dt),
               h_last=(last, 1.05 * (el + 64 * F * ml) + TINY))
    if dy is None:
        return out
    want = Q.recurrence_bwd(dy, dh, r, i, x, lam, mask, past, rate, reverse)
    dyl = np.abs(Q._live(mask, dy)[0])
    _, mb, ml = Q.walk(a, a * dyl, zero if dh is None else np.abs(dh), back)
    md = dyl + mb
    _, eb, el = Q.walk(a, a * md * (e_a + 4 * F), zero, back)
    ed = eb + 64 * F * md
    D = np.abs(want["state"])
    ep = ep + 64 * F * mp
    t1, t2 = np.abs(la) * a * np.abs(past), b * a * a * np.abs(la) * inv
    eK = ed * (t1 + t2 + b * SHUT) + D * (
        np.abs(la) * a * ep + t1 * (e_la + e_a + 6 * F) +
        t2 * (_eps_sig(il) + 2 * e_a + e_la + e_p / 2 + 16 * F) + b * SHUT)
    eK *= on
    K = D * (t1 + t2) * on
    rest = Q.sigmoid(-rl)
    out["dr"] = _stored(want["dr"], (eK + K * (_eps_sig(rl) + 4 * F)) * rest, dt)
    si, ri = Q.sigmoid(il), Q.sigmoid(-il)
    for name, size in (("dx", si * on), ("di", b * ri)):
        out[name] = _stored(want[name], size * (
            beta * (ed + D * (e_p / 2 + 2 * _eps_sig(il) + 16 * F)) + (D + ed) * SHUT), dt)
    soft = np.logaddexp(0.0, lam)
    ratio = np.where(soft > 0, Q.sigmoid(lam) / np.where(soft > 0, soft, 1.0), 1.0)
    out["dlam"] = (want["dlam"], 1.05 * ratio * (eK + 1024 * F * K).sum((0, 2)) + TINY)
    out["dh0"] = (want["dh0"], 1.05 * (el + 64 * F * ml) + TINY)
    return out
