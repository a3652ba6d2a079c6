"""rat3d_qk_norm_rope_*, rat3d_rope_table and rat3d_dropout_* against their float64
definitions, and a whole voxel self-attention block."""
import zlib

import numpy as np
import pytest

from oracle import attention as A
from tests import attn_util as AU
from tests import gpu_util as U

pytestmark = pytest.mark.gpu

F = 2.0 ** -24


def _rng(case):
    return np.random.default_rng(zlib.crc32(repr(case).encode()))


def _ws(nbytes):
    torch = U.torch_mod()
    return torch.full((max(int(nbytes), 16),), 0xFF, dtype=torch.uint8, device="cuda:0")


# n, heads, kv, hd, grid, rot, origin, norm
QK = [
    (1, 1, 1, 6, (1, 1, 1), (2, 2, 2), (0, 0, 0), True),
    (2, 2, 1, 16, (3, 5, 7), (4, 6, 4), (0, 0, 0), True),
    (1, 3, 3, 40, (5, 4, 11), (12, 12, 12), (91, 0, 7), True),
    (2, 4, 2, 32, (6, 7, 6), (10, 10, 10), (0, 0, 0), True),
    (1, 2, 2, 64, (4, 8, 8), (20, 20, 20), (0, 0, 0), True),
    (1, 1, 1, 128, (3, 9, 5), (42, 42, 42), (0, 0, 0), True),
    (1, 1, 2, 96, (2, 13, 5), (32, 32, 32), (-5, 1 << 20, -(1 << 24)), True),
    (3, 2, 1, 33, (2, 3, 43), (6, 0, 8), (0, 0, 0), True),
    (1, 2, 1, 1, (2, 5, 13), (0, 0, 0), (0, 0, 0), True),
    (1, 2, 1, 17, (2, 5, 13), (0, 16, 0), (0, 3, 0), False),
    (2, 3, 0, 24, (4, 5, 13), (8, 8, 8), (0, 0, 0), True),
    (2, 0, 2, 24, (4, 5, 13), (8, 8, 8), (0, 0, 0), False),
    (1, 70, 30, 8, (2, 2, 40), (2, 2, 2), (0, 0, 0), True),
    (40, 9, 3, 20, (5, 6, 7), (6, 6, 6), (0, 0, 0), True),
    # tiles enough for eight tokens a thread in bfloat16
    (1030, 1, 1, 16, (3, 5, 3), (4, 6, 4), (0, 0, 0), True),
    (520, 1, 1, 40, (5, 6, 9), (12, 12, 12), (0, 0, 0), True),
    (1030, 1, 0, 64, (2, 4, 5), (20, 20, 20), (3, 0, 0), True),
    (520, 1, 1, 72, (1, 2, 130), (24, 24, 24), (0, 0, 0), True),
    (1030, 1, 1, 96, (1, 3, 11), (32, 32, 32), (0, 0, 7), False),
]


def _qk_bounds(dt, x, heads, gamma, turn, eps, dy=None):
    """(value, bound) of the forward, or of dx and dgamma.  Roundings in float32: the
    mean square (D + 4 terms), the root and quotient, the gain, two products and a
    sum of the turn, and cos and sin, each once rounded: (D + 16) f of the turned
    magnitudes; then one rounding to the storage type."""
    u, hd = AU.U[dt], x.shape[1] // heads
    at = np.abs(turn)
    k = (hd + 16) * F
    if dy is None:
        y = A.qk_fwd(x, heads, gamma, turn, eps)
        t = A._heads(x, heads)
        z = np.abs(t if gamma is None else t / np.sqrt((t * t).mean(-1, keepdims=True) + eps) * gamma)
        return y, k * A._flat(np.einsum("vab,nhvb->nhva", at, z)) + u * np.abs(y) + AU.TINY
    dx, dg = A.qk_bwd(dy, x, heads, gamma, turn, eps)
    dz = np.einsum("vab,nhva->nhvb", at, np.abs(A._heads(dy, heads)))
    if gamma is None:
        return (dx, k * A._flat(dz) + u * np.abs(dx) + AU.TINY), None
    t = A._heads(x, heads)
    r = 1.0 / np.sqrt((t * t).mean(-1, keepdims=True) + eps)
    w = np.abs(gamma) * dz
    mag = r * (w + np.abs(t) * r * r * (w * np.abs(t)).mean(-1, keepdims=True))
    terms = (dz * np.abs(t) * r).sum((0, 1, 2))
    # sums over volumes, heads and voxels: a thread adds the four tokens of each of
    # its heads, 32 threads join in a tree, and 256 threads the parts: fewer than
    # 2^10 additions in a row at these sizes
    return (dx, 4 * k * A._flat(mag) + u * np.abs(dx) + AU.TINY), (dg, (k + 1024 * F) * terms + AU.TINY)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", QK, ids=lambda c: "n%d_h%d_%d_d%d_%s" % (
    c[0], c[1], c[2], c[3], "x".join(map(str, c[4]))))
def test_qk_norm_rope(case, dt):
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, grid, rot, origin, norm = case
    rng = _rng((case, dt))
    v, base, eps = int(np.prod(grid)), 100.0, 1e-5
    desc = R.qk_desc(n, heads, kv, hd, *grid, U.code(dt), rot=rot, origin=origin, base=base,
                     eps=eps, norm=norm)
    size = R.rat3d_rope_table_size(desc)
    table = _ws(size) if size else None
    if size:
        R.rat3d_rope_table(desc, table)
    turn = A.rotation(hd, grid, rot, origin, base)
    side = {}
    for s, many in (("q", heads), ("k", kv)):
        if not many:
            side[s] = None
            continue
        x, xr = U.dev_input(rng.standard_normal((n, many * hd, v)) * 2, dt)
        if v > 2:
            x[0, :, 1] = 0  # a token of zeros: eps keeps the norm finite
            xr[0, :, 1] = 0
        dy, dyr = U.dev_input(rng.standard_normal((n, many * hd, v)), dt)
        g, gr = U.dev_input(1 + 0.3 * rng.standard_normal(hd), "f32")
        init, initr = U.dev_input(rng.standard_normal(hd), "f32")
        side[s] = dict(x=x, xr=xr, dy=dy, dyr=dyr, g=g, gr=gr if norm else None, many=many,
                       y=U.guarded((n, many * hd, v), dt), dx=U.guarded((n, many * hd, v), dt),
                       dg=U.guarded((hd,), "f32"), init=init, initr=initr)
    get = lambda s, f: None if side[s] is None else side[s][f] if not isinstance(  # noqa: E731
        side[s][f], tuple) else side[s][f][0]
    print("qk", case, dt, flush=True)
    R.rat3d_qk_norm_rope_fwd(desc, get("q", "x"), get("k", "x"), get("q", "g"), get("k", "g"),
                             table, get("q", "y"), get("k", "y"))
    need = R.rat3d_qk_norm_rope_workspace_size(desc)
    assert (need > 0) == norm

    def bwd(acc):
        R.rat3d_qk_norm_rope_bwd(desc, get("q", "dy"), get("k", "dy"), get("q", "x"),
                                 get("k", "x"), get("q", "g"), get("k", "g"), table,
                                 get("q", "dx"), get("k", "dx"), get("q", "dg"), get("k", "dg"),
                                 acc, _ws(need), need)
    bwd(0)
    U.sync()
    for s in "qk":
        if side[s] is None:
            continue
        d = side[s]
        want = _qk_bounds(dt, d["xr"], d["many"], d["gr"], turn, eps)
        AU.within(U.f64(d["y"][0]), want, "y " + s)
        dx, dg = _qk_bounds(dt, d["xr"], d["many"], d["gr"], turn, eps, d["dyr"])
        AU.within(U.f64(d["dx"][0]), dx, "dx " + s)
        if norm:
            AU.within(U.f64(d["dg"][0]), dg, "dgamma " + s)
            d["dg0"] = d["dg"][0].clone()
            d["dg"][0].copy_(d["init"])
        for o in ("y", "dx", "dg"):
            U.guard_intact(d[o][1], o)
    if norm:
        bwd(1)
        U.sync()
        for s in "qk":
            if side[s] is not None:
                assert torch.equal(side[s]["dg"][0], side[s]["init"] + side[s]["dg0"])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_qk_ranges_in_place(dt):
    """Channel ranges of one tensor at odd elements, and the results over the inputs."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, grid, rot = 2, 3, 1, 20, (3, 5, 9), (6, 6, 6)
    v = 135
    wide = (heads + 2 * kv) * hd * v + 5
    rng = _rng(("ranges", dt))
    x, xr = U.dev_input(rng.standard_normal(n * wide + 32), dt)
    g, gr = U.dev_input(1 + 0.3 * rng.standard_normal(hd), "f32")
    desc = R.qk_desc(n, heads, kv, hd, *grid, U.code(dt), rot=rot, q_stride=wide, k_stride=wide,
                     oq_stride=wide, ok_stride=wide)
    table = _ws(R.rat3d_rope_table_size(desc))
    R.rat3d_rope_table(desc, table)
    es = x.element_size()
    qp, kp = x.data_ptr() + es, x.data_ptr() + (heads * hd * v + 2) * es
    R.rat3d_qk_norm_rope_fwd(desc, qp, kp, g, g, table, qp, kp)
    U.sync()
    turn = A.rotation(hd, grid, rot, (0, 0, 0), 100.0)
    got = U.f64(x)
    rest = np.ones(got.size, bool)
    for at, many in ((1, heads), (heads * hd * v + 2, kv)):
        sl = [slice(at + i * wide, at + i * wide + many * hd * v) for i in range(n)]
        view = lambda a: np.stack([a[s] for s in sl]).reshape(n, many * hd, v)  # noqa: E731
        AU.within(view(got), _qk_bounds(dt, view(xr), many, gr, turn, 1e-6), "in place")
        for s in sl:
            rest[s] = False
    np.testing.assert_array_equal(got[rest], xr[rest])
    del torch


def test_qk_offsets_beyond_32_bits():
    """Volumes more than 2^31 elements apart."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, grid, v, wide = 2, 2, 1, 16, (3, 5, 9), 135, (1 << 31) + 4097
    rng = _rng("far")
    x, xr = U.dev_input(rng.standard_normal((n, (heads + kv) * hd, v)), "bf16")
    g, gr = U.dev_input(1 + 0.3 * rng.standard_normal(hd), "f32")
    big = torch.empty(wide + x[0].numel() + 64, dtype=torch.bfloat16, device="cuda:0")
    rows = [big[i * wide + 5:i * wide + 5 + x[0].numel()].view(-1, v) for i in range(n)]
    for i in range(n):
        rows[i].copy_(x[i])
    desc = R.qk_desc(n, heads, kv, hd, *grid, R.BF16, rot=(4, 4, 4), q_stride=wide, k_stride=wide)
    table = _ws(R.rat3d_rope_table_size(desc))
    R.rat3d_rope_table(desc, table)
    y, z = U.empty((n, heads * hd, v), "bf16"), U.empty((n, kv * hd, v), "bf16")
    p = big.data_ptr() + 10
    R.rat3d_qk_norm_rope_fwd(desc, p, p + 2 * heads * hd * v, g, g, table, y, z)
    U.sync()
    turn = A.rotation(hd, grid, (4, 4, 4), (0, 0, 0), 100.0)
    AU.within(U.f64(y), _qk_bounds("bf16", xr[:, :heads * hd], heads, gr, turn, 1e-6), "q")
    AU.within(U.f64(z), _qk_bounds("bf16", xr[:, heads * hd:], kv, gr, turn, 1e-6), "k")


# ------------------------------------------------------------------ dropout
DROP = [(1, 1, 0.5), (7, 1, 0.3), (8, 1, 0.1), (9, 1, 0.9), (4099, 1, 0.25), (4100, 3, 0.5),
        (4100, 7, 0.5), (4103, 8, 0.5), (6000, 75, 0.4), (6001, 75, 0.4), (9000, 3000, 0.5),
        (513, 1 << 40, 0.5), (100, 1, 0.0), (100, 1, 1.0), (100, 10, 1.0), (100, 1, 1e-9)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("count,unit,p", DROP)
def test_dropout(count, unit, p, dt):
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    rng = _rng((count, unit, p, dt))
    seed, step = int(rng.integers(1 << 63)) * 2 + 1, int(rng.integers(1 << 63))
    x, xr = U.dev_input(rng.standard_normal(count), dt)
    res, rr = U.dev_input(rng.standard_normal(count), dt)
    dy, dyr = U.dev_input(rng.standard_normal(count), dt)
    keep, scale = A.keeps((count + unit - 1) // unit, p, seed, step)
    keep = np.repeat(keep, min(unit, count))[:count]
    x[torch.from_numpy(~keep).to("cuda:0")] = float("nan")  # dropped values leave nothing
    desc = R.dropout_desc(count, p, U.code(dt), seed=seed, unit=unit)
    u = AU.U[dt]
    for r, rv in ((None, 0.0), (res, rr)):
        y, buf = U.guarded((count,), dt)
        R.rat3d_dropout_fwd(desc, step, None, x, r, y)
        U.sync()
        U.guard_intact(buf, "y")
        want = np.where(keep, xr * scale, 0.0) + rv
        # the scale and the product round in float32, the sum once to the type
        AU.within(U.f64(y), (want, 4 * F * (np.abs(xr) * scale + np.abs(rv)) + u * np.abs(want)
                             + AU.TINY), "y")
    dx, buf = U.guarded((count,), dt)
    R.rat3d_dropout_bwd(desc, step, None, dy, dx, 0)
    U.sync()
    want = np.where(keep, dyr * scale, 0.0)
    AU.within(U.f64(dx), (want, 4 * F * np.abs(want) + u * np.abs(want) + AU.TINY), "dx")
    first = U.f64(dx)
    R.rat3d_dropout_bwd(desc, step, None, dy, dx, 1)
    U.sync()
    want = want + first
    AU.within(U.f64(dx), (want, 4 * F * (np.abs(want) + np.abs(first)) + u * np.abs(want) + AU.TINY),
              "dx added")
    U.guard_intact(buf, "dx")
    # in place, and the step taken from the device
    half = torch.tensor([step - step // 2], dtype=torch.int64, device="cuda:0")
    z = dy.clone()
    R.rat3d_dropout_fwd(desc, step // 2, half, z, None, z)
    U.sync()
    np.testing.assert_array_equal(U.f64(z), first)


def test_dropout_graph_draws_new_masks():
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    count = 5000
    x = torch.ones(count, device="cuda:0")
    y = torch.empty_like(x)
    step = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    desc = R.dropout_desc(count, 0.5, R.F32, seed=11)
    R.rat3d_dropout_fwd(desc, 3, step, x, None, y)
    U.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        R.rat3d_dropout_fwd(desc, 3, step, x, None, y)
    for i in range(3):
        step.fill_(i * 5)
        U.sync()
        graph.replay()
        U.sync()
        keep, scale = A.keeps(count, 0.5, 11, 3 + 5 * i)
        np.testing.assert_array_equal(U.f64(y), np.where(keep, scale, 0.0))


# ------------------------------------------------------------------ the block
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_self_attention_block(dt):
    """y = x + dropout(conv(attention(norm_rope(conv(x))))) as a program runs it, in
    one tensor for q, k and v, forward and backward, against float64 and, in
    float32, against differences of the float64 block."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, c, heads, kv, hd, grid = 2, 48, 4, 2, 24, (4, 5, 6)
    v, rot, p, seed, step, eps = 120, (8, 8, 8), 0.2, 5, 9, 1e-5
    wide, co = (heads + 2 * kv) * hd, heads * hd
    rng = _rng(("block", dt))
    x, xr = U.dev_input(rng.standard_normal((n, c, v)), dt)
    w1, w1r = U.dev_input(rng.standard_normal((wide, c)) / np.sqrt(c), dt)
    w2, w2r = U.dev_input(rng.standard_normal((c, co)) / np.sqrt(co), dt)
    gq, gqr = U.dev_input(1 + 0.2 * rng.standard_normal(hd), "f32")
    gk, gkr = U.dev_input(1 + 0.2 * rng.standard_normal(hd), "f32")
    dy, dyr = U.dev_input(rng.standard_normal((n, c, v)), dt)
    mask = (rng.random((n, v)) < 0.7).astype(np.uint8)
    m = torch.from_numpy(mask).to("cuda:0")
    code = U.code(dt)
    c1 = R.conv_desc(n, c, wide, *grid, 1, 1, 0, False, code)
    c2 = R.conv_desc(n, co, c, *grid, 1, 1, 0, False, code)
    qd = R.qk_desc(n, heads, kv, hd, *grid, code, rot=rot, eps=eps, q_stride=wide * v,
                   k_stride=wide * v)
    ad = R.attention_desc(n, heads, kv, hd, v, v, code, v_stride=wide * v)
    dd = R.dropout_desc(n * c * v, p, code, seed=seed, unit=1)
    table = _ws(R.rat3d_rope_table_size(qd))
    R.rat3d_rope_table(qd, table)
    need = max([R.rat3d_conv3d_workspace_size(d, i) for d in (c1, c2) for i in range(3)] +
               [R.rat3d_attention_workspace_size(ad, i) for i in (0, 1)] +
               [R.rat3d_qk_norm_rope_workspace_size(qd)])
    ws = _ws(need)
    E = lambda ch: U.empty((n, ch, v), dt)  # noqa: E731
    qkv, q, k, o, z, y = E(wide), E(co), E(kv * hd), E(co), E(c), E(c)
    lse = U.zeros_f32((n, heads, v))
    kin, vin = qkv[:, co:co + kv * hd], qkv[:, co + kv * hd:]
    R.rat3d_conv3d_fwd(c1, x, w1, None, qkv, ws, need)
    R.rat3d_qk_norm_rope_fwd(qd, qkv, kin, gq, gk, table, q, k)
    R.rat3d_attention_fwd(ad, q, k, vin, m, o, lse, ws, need)
    R.rat3d_conv3d_fwd(c2, o, w2, None, z, ws, need)
    R.rat3d_dropout_fwd(dd, step, None, z, x, y)
    dz, do, dq, dk, dqkv, dx = E(c), E(co), E(co), E(kv * hd), E(wide), dy.clone()
    dgq, dgk = U.zeros_f32(hd), U.zeros_f32(hd)
    dw1, dw2 = U.zeros_f32((wide, c)), U.zeros_f32((c, co))
    R.rat3d_dropout_bwd(dd, step, None, dy, dz, 0)
    R.rat3d_conv3d_wgrad(c2, o, dz, dw2, None, 0, ws, need)
    R.rat3d_conv3d_dgrad(c2, dz, w2, do, 0, ws, need)
    dvin = dqkv[:, co + kv * hd:]
    R.rat3d_attention_bwd(ad, do, q, k, vin, m, o, lse, dq, dk, dvin, ws, need)
    R.rat3d_qk_norm_rope_bwd(qd, dq, dk, qkv, kin, gq, gk, table, dqkv, dqkv[:, co:co + kv * hd],
                             dgq, dgk, 0, ws, need)
    R.rat3d_conv3d_wgrad(c1, x, dqkv, dw1, None, 0, ws, need)
    R.rat3d_conv3d_dgrad(c1, dqkv, w1, dx, 1, ws, need)
    U.sync()

    turn = A.rotation(hd, grid, rot, (0, 0, 0), 100.0)
    drop = A.dropout(np.ones((n, c, v)), 1, p, seed, step)

    def forward(xr, w1r, w2r, gqr, gkr):
        t = np.matmul(w1r, xr)
        qs, ks = A.qk_fwd(t[:, :co], heads, gqr, turn, eps), \
            A.qk_fwd(t[:, co:co + kv * hd], kv, gkr, turn, eps)
        vs = t[:, co + kv * hd:]
        os, _, ps = A.attention(qs, ks, vs, heads, kv, mask, hd ** -0.5)
        return t, qs, ks, vs, os, ps, xr + drop * np.matmul(w2r, os)

    t, qs, ks, vs, os, ps, ys = forward(xr, w1r, w2r, gqr, gkr)
    dzr = drop * dyr
    dor = np.matmul(w2r.T, dzr)
    dqr, dkr, dvr = A.attention_bwd(dor, qs, ks, vs, heads, kv, mask, hd ** -0.5, ps)
    a, dgqr = A.qk_bwd(dqr, t[:, :co], heads, gqr, turn, eps)
    b, dgkr = A.qk_bwd(dkr, t[:, co:co + kv * hd], kv, gkr, turn, eps)
    dt_ = np.concatenate([a, b, dvr], axis=1)
    want = dict(y=ys, dx=dyr + np.matmul(w1r.T, dt_), dw1=np.matmul(dt_, xr.swapaxes(1, 2)).sum(0),
                dw2=np.matmul(dzr, os.swapaxes(1, 2)).sum(0), dgq=dgqr, dgk=dgkr)
    got = dict(y=y, dx=dx, dw1=dw1, dw2=dw2, dgq=dgq, dgk=dgk)
    for name in want:
        r = U.rel(U.f64(got[name]), want[name])
        print(name, r, flush=True)
        # the stated tolerances of the composites: 1e-4 in float32, 2e-2 in bfloat16
        assert r <= U.TOL[dt], (name, r)
    if dt == "f32":
        f = lambda *s: float((forward(*s)[-1] * dyr).sum())  # noqa: E731
        args, h = [xr, w1r, w2r, gqr, gkr], 1e-5
        for i, name in ((0, "dx"), (1, "dw1"), (2, "dw2"), (3, "dgq"), (4, "dgk")):
            e = tuple(np.unravel_index(int(np.argmax(np.abs(want[name]))), want[name].shape))
            s = [z.copy() for z in args]
            s[i][e] += h
            up = f(*s)
            s[i][e] -= 2 * h
            diff = (up - f(*s)) / (2 * h)
            assert float(U.f64(got[name])[e]) == pytest.approx(diff, rel=1e-3), name


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_qk_smallest_eps_and_no_rotation(dt):
    """At the smallest eps a token of zeros stays zero and its gradient finite; without
    rotation a table that is given all the same changes nothing."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    hd, v = 24, 10
    desc = R.qk_desc(1, 1, 0, hd, 1, 2, 5, U.code(dt), rot=(0, 0, 0), eps=2.0 ** -126, norm=True)
    x, xr = U.dev_input(_rng(("eps", dt)).standard_normal((1, hd, v)), dt)
    x[0, :, 3] = 0
    xr[0, :, 3] = 0
    dy, _ = U.dev_input(np.ones((1, hd, v)), dt)
    g, gr = U.dev_input(np.ones(hd), "f32")
    table = torch.full((2,), float("nan"), device="cuda:0")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    dg = torch.empty(hd, device="cuda:0")
    need = R.rat3d_qk_norm_rope_workspace_size(desc)
    R.rat3d_qk_norm_rope_fwd(desc, x, None, g, None, table, y, None)
    R.rat3d_qk_norm_rope_bwd(desc, dy, None, x, None, g, None, table, dx, None, dg, None, 0,
                             _ws(need), need)
    U.sync()
    want = _qk_bounds(dt, xr, 1, gr, A.rotation(hd, (1, 2, 5), (0, 0, 0), (0, 0, 0), 100.0),
                      2.0 ** -126)
    AU.within(U.f64(y), want, "y")
    assert bool((y[0, :, 3] == 0).all())
    # r = 2^63 there: dx = dy r, a power of two
    assert bool((dx[0, :, 3].float() == 2.0 ** 63).all())
    assert bool(torch.isfinite(dg).all())
