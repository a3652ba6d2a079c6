"""Float64 references and element-wise bounds of the voxel self-attention tests.

u is the largest relative error of one rounding to the storage type (half a step:
2^-8 bfloat16, 2^-24 float32), f = 2^-24 that of float32.  The bounds count every
rounding of the computation once, at its largest, and sums of K float32 terms
with K f times the sum of magnitudes:
  score s = scale q.k:      es = (D + 4) f scale |q|.|k| + 8 f (|s| + max |s|)
     (products, the scale, and the exponent's argument, formed in log 2 units)
  probability p:            relative error ep = 2 max es + 16 f
     (the exponential is off by a few units; its error and that of the sum both
     count), and u where it is rounded for the matrix product
  o = sum p v:              (u + ep + T f) sum p|v| + u |o|
  D_i = do . o (stored o):  (D + 2) f |do|.|o| + |do| . (bound of o)
  ds = p (do.v - D_i):      p ((D + 2) f |do|.|v| + bound of D_i) + (u + ep) |ds|
                            + p ep |D_i|... (p's own error times the bracket)
  sums over ds and p:       as for o, with the bound of ds carried through.
The sums l over T probabilities are float32: T f relative, in ep.
Probabilities below 2^-126, the smallest normal float32, may come out as 0: an
absolute error of 2^-126 each, so a sum over them is off by 2^-126 times the sum of
the other factors' magnitudes (400 scores 80 apart and factors near 10: 400 * 10 *
2^-126 = 5e-35), however small the result.
"""
import numpy as np

from oracle import attention as A

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
F = 2.0 ** -24
TINY = 2.0 ** -120  # results below the normal range may be flushed
GONE = 2.0 ** -126  # a probability that comes out as 0


def attention_refs(q, k, v, heads, kv, mask, scale, dt, do=None):
    """{name: (value, bound)} for o, lse and, with do, dq, dk, dv."""
    u, hd, grp = U[dt], q.shape[1] // heads, heads // kv
    tq, tk = q.shape[2], k.shape[2]
    if mask is not None:
        live = (mask != 0)[:, None, :]
        k, v = np.where(live, k, 0.0), np.where(live, v, 0.0)
    o, lse, p = A.attention(q, k, v, heads, kv, mask, scale)
    qh = A._heads(q, heads)
    kh, vh = (np.repeat(A._heads(t, kv), grp, axis=1) for t in (k, v))
    mag = np.matmul(np.abs(qh), np.abs(kh).swapaxes(2, 3)) * scale
    if mask is not None:
        mag = np.where((mask != 0)[:, None, None, :], mag, 0.0)
    es = (hd + 4) * F * mag + 8 * F * (mag + mag.max(-1, keepdims=True))
    ep = 2 * es.max(-1, keepdims=True) + (16 + tk) * F
    to = A._flat((u + ep + tk * F) * np.matmul(p, np.abs(vh)) +
                 GONE * np.abs(vh).sum(2, keepdims=True)) + u * np.abs(o) + TINY
    out = dict(o=(o, to))
    with np.errstate(invalid="ignore"):
        out["lse"] = (lse, ep[..., 0] + 8 * F * (np.abs(lse) + 1))
    if do is None:
        return out
    doh, oh, toh = (A._heads(t, heads) for t in (do, o, to))
    grads = A.attention_bwd(do, q, k, v, heads, kv, mask, scale, p)
    dp = np.matmul(doh, vh.swapaxes(2, 3))
    dlt = (doh * oh).sum(-1, keepdims=True)
    tdp = (hd + 2) * F * np.matmul(np.abs(doh), np.abs(vh).swapaxes(2, 3))
    tdl = ((hd + 2) * F * np.abs(doh * oh) + np.abs(doh) * toh).sum(-1, keepdims=True)
    ads = p * np.abs(dp - dlt)
    tds = p * (tdp + tdl) + (u + ep) * ads + GONE * (np.abs(dp - dlt) + tdp + tdl)

    def join(t):
        return A._flat(t.reshape((t.shape[0], kv, grp) + t.shape[2:]).sum(2))

    n = max(tq * grp, tk)
    # 4 f: the scale and the multiplications themselves
    tdq = A._flat(np.matmul(tds + (n + 4) * F * (ads + tds), np.abs(kh))) * scale
    tdk = join(np.matmul((tds + (n + 4) * F * (ads + tds)).swapaxes(2, 3), np.abs(qh))) * scale
    tdv = join(np.matmul((p * (u + ep + (n + 4) * F) + GONE).swapaxes(2, 3), np.abs(doh)))
    for name, g, t in zip(("dq", "dk", "dv"), grads, (tdq, tdk, tdv)):
        out[name] = (g, t + u * (np.abs(g) + t) + TINY)
    return out


def within(got, ref, what):
    """Every element within its bound; infinities equal."""
    want, bound = ref
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), "%s: infinities differ" % what
    d, b = np.abs(got[~inf] - want[~inf]), np.broadcast_to(bound, want.shape)[~inf]
    assert np.all(np.isfinite(d)), "%s: not finite" % what
    if d.size:
        i = int(np.argmax(d - b))
        assert d[i] <= b[i], "%s: %d of %d beyond the bound, worst got %.6e want %.6e off %.3e " \
            "bound %.3e" % (what, int((d > b).sum()), d.size, got[~inf][i], want[~inf][i], d[i], b[i])
