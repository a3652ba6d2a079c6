"""Float64 definitions of the voxel self-attention operators: head norm with
rotation by the voxel's place, attention with a key mask and grouped heads, and
dropout from a counter.  Everything is written from the formulas, in numpy.
"""
import numpy as np


# ------------------------------------------------------------------ norm and rotation
def rotation(head_dim, grid, rot, origin, base):
    """[v][head_dim][head_dim]: the matrix that turns a head's vector at each voxel."""
    at = np.stack(np.meshgrid(*(np.arange(s, dtype=np.float64) + o
                                for s, o in zip(grid, origin)), indexing="ij")).reshape(3, -1)
    m = np.broadcast_to(np.eye(head_dim), (at.shape[1], head_dim, head_dim)).copy()
    first = 0
    for axis in range(3):
        for i in range(rot[axis] // 2):
            t = at[axis] * base ** (-2.0 * i / rot[axis])
            a, b = first + i, first + rot[axis] // 2 + i
            m[:, a, a], m[:, a, b] = np.cos(t), -np.sin(t)
            m[:, b, a], m[:, b, b] = np.sin(t), np.cos(t)
        first += rot[axis]
    return m


def _heads(x, heads):
    """[n][heads * hd][v] -> [n][heads][v][hd]"""
    n, c, v = x.shape
    return x.reshape(n, heads, c // heads, v).transpose(0, 1, 3, 2)


def _flat(x):
    n, h, v, d = x.shape
    return x.transpose(0, 1, 3, 2).reshape(n, h * d, v)


def qk_fwd(x, heads, gamma, turn, eps):
    """gamma None: rotation alone."""
    t = _heads(x, heads)
    if gamma is not None:
        t = t / np.sqrt((t * t).mean(-1, keepdims=True) + eps) * gamma
    return _flat(np.einsum("vab,nhvb->nhva", turn, t))


def qk_bwd(dy, x, heads, gamma, turn, eps):
    """(dx, dgamma)"""
    dz = np.einsum("vab,nhva->nhvb", turn, _heads(dy, heads))
    if gamma is None:
        return _flat(dz), None
    t = _heads(x, heads)
    r = 1.0 / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    dg = (dz * t * r).sum((0, 1, 2))
    u = dz * gamma
    return _flat(r * (u - t * r * r * (u * t).mean(-1, keepdims=True))), dg


# ------------------------------------------------------------------ attention
def attention(q, k, v, heads, kv, mask, scale):
    """(o, lse [n][heads][tq], p [n][heads][tq][tk]); masked keys are not read."""
    n = q.shape[0]
    tq, tk = q.shape[2], k.shape[2]
    if mask is not None:
        live = (mask != 0)[:, None, :]
        k, v = np.where(live, k, 0.0), np.where(live, v, 0.0)
    qh = _heads(q, heads)
    kh, vh = (np.repeat(_heads(t, kv), heads // kv, axis=1) for t in (k, v))
    s = np.matmul(qh, kh.swapaxes(2, 3)) * scale
    if mask is not None:
        s = np.where((mask != 0)[:, None, None, :], s, -np.inf)
    m = s.max(-1, keepdims=True)
    m = np.where(np.isneginf(m), 0.0, m)
    e = np.exp(s - m)
    total = e.sum(-1, keepdims=True)
    p = e / np.where(total == 0, 1.0, total)
    with np.errstate(divide="ignore"):
        lse = (np.log(total) + m)[..., 0]
    assert p.shape == (n, heads, tq, tk)
    return _flat(np.matmul(p, vh)), lse, p


def attention_bwd(do, q, k, v, heads, kv, mask, scale, p):
    """(dq, dk, dv)"""
    n, grp = q.shape[0], heads // kv
    if mask is not None:
        live = (mask != 0)[:, None, :]
        k, v = np.where(live, k, 0.0), np.where(live, v, 0.0)
    qh, doh = _heads(q, heads), _heads(do, heads)
    kh, vh = (np.repeat(_heads(t, kv), grp, axis=1) for t in (k, v))
    dp = np.matmul(doh, vh.swapaxes(2, 3))
    ds = p * (dp - (p * dp).sum(-1, keepdims=True)) * scale

    def join(t):  # sum over the query heads of a group
        return _flat(t.reshape((n, kv, grp) + t.shape[2:]).sum(2))

    return (_flat(np.matmul(ds, kh)), join(np.matmul(ds.swapaxes(2, 3), qh)),
            join(np.matmul(p.swapaxes(2, 3), doh)))


# ------------------------------------------------------------------ dropout
def philox(ctr, key, rounds=10):
    """Philox4x32 (Salmon et al. 2011) on plain integers: four words from four
    counter words and two key words."""
    c, k = list(ctr), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xffffffff, (a >> 32) ^ c[3] ^ k[1], a & 0xffffffff]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def keeps(units, p, seed, step):
    """bool [units]: which decisions keep, and the scale of what is kept."""
    at = int(round(p * 65536))
    out = []
    for b in range((units + 7) // 8):
        w = philox((b & 0xffffffff, b >> 32, step & 0xffffffff, step >> 32),
                   (seed & 0xffffffff, seed >> 32))
        for x in w:
            out += [x & 0xffff, x >> 16]
    return np.array(out[:units]) >= at, (65536.0 / (65536 - at) if at < 65536 else 0.0)


def dropout(x, unit, p, seed, step, residual=None):
    flat = x.reshape(-1)
    units = (flat.size + unit - 1) // unit
    keep, scale = keeps(units, p, seed, step)
    keep = np.repeat(keep, unit)[:flat.size]
    y = np.where(keep, flat * scale, 0.0).reshape(x.shape)
    return y if residual is None else y + residual
