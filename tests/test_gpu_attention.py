"""rat3d_attention_* against its float64 definition, element by element: head
sizes, token counts around the tiles, grouped heads, masks, strides, splits."""
import zlib

import numpy as np
import pytest

from tests import attn_util as AU
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def _rng(case):
    return np.random.default_rng(zlib.crc32(repr(case).encode()))


def _mask(kind, n, tk, rng):
    if kind is None:
        return None
    m = np.zeros((n, tk), np.uint8)
    if kind == "half":
        m[:] = rng.random((n, tk)) < 0.5
    elif kind == "one":  # a single live key, another in each volume
        for i in range(n):
            m[i, rng.integers(tk)] = 255
    elif kind == "first_none":  # the first volume has no key at all
        m[1:] = rng.random((n - 1, tk)) < 0.6
        m[1:, -1] = 1
    elif kind == "all":
        m[:] = 2
    elif kind == "first65":
        m[:, :65] = 1
    elif kind == "run":  # a run of masked keys longer than a tile, inside
        m[:] = 1
        m[:, tk // 4:tk // 2 + 70] = 0
    return m


def _dev(a, dt, guard=0):
    """Device tensor of a [n][c][t] and its exact values."""
    return U.dev_input(a, dt)


def _tensors(case):
    n, heads, kv, hd, tq, tk, mk, dt = case
    rng = _rng(case)
    mask = _mask(mk, n, tk, rng)
    q, qr = U.dev_input(rng.standard_normal((n, heads * hd, tq)) * 1.5, dt)
    k, kr = U.dev_input(rng.standard_normal((n, kv * hd, tk)), dt)
    v, vr = U.dev_input(rng.standard_normal((n, kv * hd, tk)), dt)
    do, dor = U.dev_input(rng.standard_normal((n, heads * hd, tq)), dt)
    m = None
    if mask is not None:
        torch = U.torch_mod()
        m = torch.from_numpy(mask).to("cuda:0")
        # what masked voxels hold must not matter
        dead = (m == 0)[:, None, :]
        k.masked_fill_(dead, float("nan"))
        v.masked_fill_(dead, float("inf"))
    return (q, k, v, do, m), (qr, kr, vr, dor, mask)


def _ws(nbytes):
    torch = U.torch_mod()
    return torch.full((max(int(nbytes), 16),), 0xFF, dtype=torch.uint8, device="cuda:0")


def _both(R, desc, case, dev, lse=True):
    """Forward and backward into guarded outputs."""
    n, heads, kv, hd, tq, tk, mk, dt = case
    q, k, v, do, m = dev
    outs = {}
    for name, shape in (("o", q.shape), ("dq", q.shape), ("dk", k.shape), ("dv", k.shape)):
        outs[name] = U.guarded(tuple(shape), dt)
    outs["lse"] = U.guarded((n, heads, tq), "f32")
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    print("attention", case, "workspace", need, flush=True)
    R.rat3d_attention_fwd(desc, q, k, v, m, outs["o"][0], outs["lse"][0], _ws(need[0]), need[0])
    U.sync()
    R.rat3d_attention_bwd(desc, do, q, k, v, m, outs["o"][0], outs["lse"][0], outs["dq"][0],
                          outs["dk"][0], outs["dv"][0], _ws(need[1]), need[1])
    U.sync()
    for name, (_, buf) in outs.items():
        U.guard_intact(buf, name)
    return {name: t for name, (t, _) in outs.items()}


def _check(case):
    from paper_2104_05035_amd import rat3d as R
    n, heads, kv, hd, tq, tk, mk, dt = case
    dev, ref = _tensors(case)
    desc = R.attention_desc(n, heads, kv, hd, tq, tk, U.code(dt))
    got = _both(R, desc, case, dev)
    q, k, v, do, mask = ref
    want = AU.attention_refs(q, k, v, heads, kv, mask, hd ** -0.5, dt, do)
    for name in ("o", "lse", "dq", "dk", "dv"):
        AU.within(U.f64(got[name]), want[name], "%s %s" % (name, case))
    again = _both(R, desc, case, dev)
    torch = U.torch_mod()
    for name in got:
        assert torch.equal(got[name], again[name]), "%s differs from run to run" % name


#            n heads kv hd  tq   tk   mask
HEAD_DIMS = [(1, 1, 1, hd, 37, 70, None) for hd in (1, 2, 8, 15, 16, 17, 24, 31, 32, 33, 40, 48,
                                                  63, 64, 65, 80, 96, 97, 100, 127, 128)]
TOKENS = [(1, 2, 1, 20, tq, tk, None) for tq, tk in (
    (1, 1), (1, 2), (2, 1), (1, 31), (1, 700), (3, 33), (31, 32), (32, 31), (33, 64), (63, 65),
    (64, 63), (65, 129), (127, 128), (128, 127), (129, 96), (257, 191), (192, 255), (1000, 5),
    (5, 1000))]
HEADS = [(2, 3, 3, 16, 40, 50, None), (2, 4, 2, 32, 40, 50, None), (3, 6, 1, 8, 70, 33, None),
         (1, 5, 5, 64, 252, 252, None), (2, 8, 2, 40, 252, 252, "half")]
MASKS = [(2, 2, 1, 24, 50, tk, mk) for tk, mk in (
    (1, "all"), (1, "one"), (40, "half"), (64, "one"), (130, "half"), (130, "first_none"),
    (130, "all"), (130, "first65"), (300, "run"), (700, "half"), (700, "one"), (65, "first_none"),
    (5000, "half"), (4097, "one"))]
# workgroups enough for the kernels with two column blocks a wave
WIDE = [(64, 4, 4, 64, 77, 130, None), (64, 8, 4, 40, 130, 77, "half"), (64, 4, 4, 32, 33, 256, None),
        (128, 2, 2, 64, 257, 300, "run"), (32, 8, 8, 24, 300, 290, "half"),
        (90, 6, 3, 48, 1, 65, "first_none"), (256, 1, 1, 50, 97, 31, "one"),
        (256, 1, 1, 33, 1, 1, None), (256, 2, 1, 17, 65, 2, None), (90, 3, 3, 64, 64, 96, "all")]
# few query rows: pieces of the keys, in both widths
FEW = [(1, 1, 1, 1, 1, 1, None), (2, 2, 1, 33, 1, 513, "half"), (1, 4, 1, 40, 1, 2049, None),
       (2, 2, 2, 128, 3, 700, "run"), (2, 3, 3, 64, 4, 1025, "first_none"), (1, 4, 2, 24, 2, 3000, "one"),
       (40, 4, 2, 8, 1, 16400, "half"), (40, 2, 2, 9, 4, 13313, None), (60, 3, 3, 5, 3, 6145, "run"),
       (1, 1, 1, 17, 5, 600, None), (2, 6, 2, 32, 4, 1030, "half"), (1, 8, 1, 64, 2, 900, "first65"),
       (2, 4, 2, 40, 7, 520, "first_none"), (40, 2, 2, 6, 13, 13000, "half"), (1, 1, 1, 16, 17, 300, None)]
# around the length up to which the packing itself finds the live keys
LISTS = [(2, 2, 2, 16, 40, tk, mk) for tk, mk in (
    (2047, "half"), (2048, "run"), (2049, "half"), (1001, "first65"), (9, "half"), (7, "half"))]
ALL = [c + (dt,) for c in HEAD_DIMS + TOKENS + HEADS + MASKS + WIDE + FEW + LISTS for dt in ("bf16", "f32")]


@pytest.mark.parametrize("case", ALL, ids=lambda c: "n%d_h%d_%d_d%d_q%d_k%d_%s_%s" % c)
def test_attention(case):
    _check(case)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("odd", [0, 1])
def test_channel_ranges_of_one_tensor(dt, odd):
    """q, k, v and their gradients as ranges of wider tensors, at odd elements; what
    lies between them stays as it was."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, t = 2, 4, 2, 24, 75
    rng = _rng(("ranges", dt, odd))
    wide = (heads + 2 * kv) * hd * t + 3 * t + odd  # elements a volume, an odd rest
    buf = rng.standard_normal(n * wide + 64)
    x, xr = U.dev_input(buf, dt)
    at = dict(q=odd, k=odd + heads * hd * t + 7, v=odd + (heads + kv) * hd * t + 11)
    c = dict(q=heads * hd, k=kv * hd, v=kv * hd)

    def view(a, name):
        return np.stack([a[at[name] + i * wide:at[name] + i * wide + c[name] * t]
                         for i in range(n)]).reshape(n, c[name], t)

    q, k, v = (view(xr, s) for s in "qkv")
    do, dor = U.dev_input(rng.standard_normal((n, heads * hd, t)), dt)
    want = AU.attention_refs(q, k, v, heads, kv, None, 0.3, dt, dor)
    desc = R.attention_desc(n, heads, kv, hd, t, t, U.code(dt), scale=0.3, q_stride=wide,
                            k_stride=wide, v_stride=wide)
    o, lse = U.empty((n, heads * hd, t), dt), U.zeros_f32((n, heads, t))
    es = x.element_size()
    g = torch.full_like(x, 77.0)
    ptr = {s: x.data_ptr() + at[s] * es for s in "qkv"}
    gp = {s: g.data_ptr() + at[s] * es for s in "qkv"}
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    R.rat3d_attention_fwd(desc, ptr["q"], ptr["k"], ptr["v"], None, o, lse, _ws(need[0]), need[0])
    R.rat3d_attention_bwd(desc, do, ptr["q"], ptr["k"], ptr["v"], None, o, lse, gp["q"], gp["k"],
                          gp["v"], _ws(need[1]), need[1])
    U.sync()
    AU.within(U.f64(o), want["o"], "o")
    AU.within(U.f64(lse), want["lse"], "lse")
    gr = U.f64(g)
    untouched = np.ones(gr.size, bool)
    for s in "qkv":
        AU.within(view(gr, s), want["d" + s], "d" + s)
        for i in range(n):
            untouched[at[s] + i * wide:at[s] + i * wide + c[s] * t] = False
    assert np.all(gr[untouched] == 77.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_large_and_small_scores(dt):
    """Scores of +-hundreds: the running maximum moves by more than any float32
    exponent in both directions along the keys."""
    from paper_2104_05035_amd import rat3d as R
    n, hd, t = 1, 16, 400
    rng = _rng(("scores", dt))
    q, qr = U.dev_input(np.ones((n, hd, t)) * np.sign(rng.standard_normal((n, 1, t))), dt)
    ramp = np.linspace(-40, 40, t)[None, None, :] * np.ones((n, hd, 1))
    k, kr = U.dev_input(ramp, dt)
    v, vr = U.dev_input(rng.standard_normal((n, hd, t)), dt)
    do, dor = U.dev_input(rng.standard_normal((n, hd, t)), dt)
    desc = R.attention_desc(n, 1, 1, hd, t, t, U.code(dt), scale=1.0)
    got = _both(R, desc, (n, 1, 1, hd, t, t, None, dt), (q, k, v, do, None))
    want = AU.attention_refs(qr, kr, vr, 1, 1, None, 1.0, dt, dor)
    for name in want:
        AU.within(U.f64(got[name]), want[name], name)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_values_that_are_not_finite(dt):
    """A NaN or infinite value at a live key reaches every query's result, one in a
    query that query's alone."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, hd, t = 1, 32, 100
    rng = _rng(("nan", dt))
    q, k, v = (U.dev_input(rng.standard_normal((n, hd, t)), dt)[0] for _ in range(3))
    v[0, 3, 70] = float("nan")
    v[0, 5, 10] = float("inf")
    q[0, 0, 41] = float("nan")
    desc = R.attention_desc(n, 1, 1, hd, t, t, U.code(dt))
    o = U.empty((n, hd, t), dt)
    need = R.rat3d_attention_workspace_size(desc, 0)
    R.rat3d_attention_fwd(desc, q, k, v, None, o, None, _ws(need), need)
    U.sync()
    o = o.float()
    assert torch.isnan(o[0, :, 41]).all() and torch.isnan(o[0, 3]).all()
    rest = [i for i in range(t) if i != 41]
    assert torch.isposinf(o[0, 5, rest]).all()
    assert torch.isfinite(o[0, 6][rest]).all()


def test_two_calls_at_once_and_another_stream():
    """Calls on two streams, each with a workspace of its own, and a call on a
    stream that the tensors were not made on."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    cases = [(2, 4, 2, 32, 500, 700, "half", "bf16"), (1, 3, 3, 40, 300, 650, None, "f32")]
    todo = []
    for c in cases:
        dev, _ = _tensors(c)
        n, heads, kv, hd, tq, tk, mk, dt = c
        desc = R.attention_desc(n, heads, kv, hd, tq, tk, U.code(dt))
        todo.append((c, dev, desc, _both(R, desc, c, dev)))
    U.sync()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for (c, dev, desc, _), st in zip(todo, streams):
        st.wait_stream(torch.cuda.current_stream())
        q, k, v, do, m = dev
        need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
        ws = _ws(max(need))
        o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, k))
        lse = U.zeros_f32((c[0], c[1], c[4]))
        U.sync()
        outs.append((need, ws, o, lse, dq, dk, dv))
    for (c, dev, desc, _), st, (need, ws, o, lse, dq, dk, dv) in zip(todo, streams, outs):
        q, k, v, do, m = dev
        R.rat3d_attention_fwd(desc, q, k, v, m, o, lse, ws, need[0], stream=st.cuda_stream)
        R.rat3d_attention_bwd(desc, do, q, k, v, m, o, lse, dq, dk, dv, ws, need[1],
                              stream=st.cuda_stream)
    U.sync()
    for (_, _, _, want), (_, _, o, lse, dq, dk, dv) in zip(todo, outs):
        for name, t in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert torch.equal(t, want[name]), name


@pytest.mark.parametrize("tq", [0, 1])
def test_captured_and_replayed(tq):
    """Forward and backward in a HIP graph, replayed on new inputs and masks, with
    eager work between the replays."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, tk = 2, 4, 2, 32, 600
    case = (n, heads, kv, hd, tq or tk, tk, "half", "bf16")
    dev, _ = _tensors(case)
    q, k, v, do, m = dev
    desc = R.attention_desc(n, heads, kv, hd, tq or tk, tk, R.BF16)
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    ws = _ws(max(need))
    o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, k))
    lse = U.zeros_f32((n, heads, tq or tk))

    def both():
        R.rat3d_attention_fwd(desc, q, k, v, m, o, lse, ws, need[0])
        R.rat3d_attention_bwd(desc, do, q, k, v, m, o, lse, dq, dk, dv, ws, need[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    U.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        g = torch.Generator(device="cuda:0").manual_seed(100 + i)
        for t in (q, k, v, do):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda:0"))
        m.copy_((torch.rand(m.shape, generator=g, device="cuda:0") < 0.2 + 0.3 * i).to(m.dtype))
        ws.fill_(0xFF)
        U.sync()
        graph.replay()
        U.sync()
        got = [t.clone() for t in (o, lse, dq, dk, dv)]
        for t in (o, lse, dq, dk, dv):
            t.fill_(55.0)
        both()
        U.sync()
        for a, b in zip(got, (o, lse, dq, dk, dv)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt,heads,hd,tq,tk", [("bf16", 2, 64, 3000, 16128), ("f32", 1, 32, 1500, 9001)])
def test_long_rows(dt, heads, hd, tq, tk):
    """Long rows against float64 on the device (the bounds' sums of magnitudes too),
    norm-wise: the stated tolerances, with room."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    g = torch.Generator(device="cuda:0").manual_seed(5)
    tdt = U.tdtype(dt)
    q, do = (torch.randn((1, heads * hd, tq), generator=g, device="cuda:0").to(tdt) for _ in range(2))
    k, v = (torch.randn((1, heads * hd, tk), generator=g, device="cuda:0").to(tdt) for _ in range(2))
    desc = R.attention_desc(1, heads, heads, hd, tq, tk, U.code(dt))
    got = _both(R, desc, (1, heads, heads, hd, tq, tk, None, dt), (q, k, v, do, None))
    for h in range(heads):
        c = slice(h * hd, (h + 1) * hd)
        qd, kd, vd, dd = (t[0, c].double().t().contiguous() for t in (q, k, v, do))
        s = torch.mm(qd, kd.t().contiguous()) * hd ** -0.5
        p = torch.softmax(s, 1)
        dp = torch.mm(dd, vd.t().contiguous())
        ds = p * (dp - (p * dp).sum(1, keepdim=True)) * hd ** -0.5
        refs = dict(o=torch.mm(p, vd), dq=torch.mm(ds, kd), dk=torch.mm(ds.t().contiguous(), qd),
                    dv=torch.mm(p.t().contiguous(), dd))
        # three roundings to the storage type on the way, each at most u
        tol = 3 * AU.U[dt] + (1e-5 if dt == "f32" else 0.0)
        for name, r in refs.items():
            x = got[name][0, c].double().t()
            off = float((x - r).norm() / r.norm())
            print(name, off, flush=True)
            assert off <= tol, (name, off)
        assert float((got["lse"][0, h].double() - torch.logsumexp(s, 1)).abs().max()) <= 1e-5


def test_offsets_beyond_32_bits():
    """Volumes more than 2^31 elements apart, forward and backward, and their gradients
    in the same places."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, t = 2, 4, 2, 32, 200
    wide = (1 << 31) + 4097
    case = (n, heads, kv, hd, t, t, "half", "bf16")
    (q, k, v, do, m), _ = _tensors(case)
    packed = R.attention_desc(n, heads, kv, hd, t, t, R.BF16)
    want = _both(R, packed, case, (q, k, v, do, m))
    big, grads = (torch.empty(wide + 8 * heads * hd * t, dtype=torch.bfloat16, device="cuda:0")
                  for _ in range(2))
    at, view = {}, {}
    end = 0
    for name, x in (("q", q), ("k", k), ("v", v)):
        c = x.shape[1] * t
        at[name] = end
        end += c + 3
        for buf in (big, grads):
            view[name, buf is big] = [buf[i * wide + at[name]:i * wide + at[name] + c].view(-1, t)
                                      for i in range(n)]
        for i in range(n):
            view[name, True][i].copy_(x[i])
    desc = R.attention_desc(n, heads, kv, hd, t, t, R.BF16, q_stride=wide, k_stride=wide,
                            v_stride=wide)
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    o, lse = torch.empty_like(q), U.zeros_f32((n, heads, t))
    p = {s: big.data_ptr() + 2 * at[s] for s in "qkv"}
    g = {s: grads.data_ptr() + 2 * at[s] for s in "qkv"}
    R.rat3d_attention_fwd(desc, p["q"], p["k"], p["v"], m, o, lse, _ws(need[0]), need[0])
    R.rat3d_attention_bwd(desc, do, p["q"], p["k"], p["v"], m, o, lse, g["q"], g["k"], g["v"],
                          _ws(need[1]), need[1])
    U.sync()
    assert torch.equal(o, want["o"]) and torch.equal(lse, want["lse"])
    for s in "qkv":
        for i in range(n):
            assert torch.equal(view[s, False][i], want["d" + s][i]), s


def test_read_out_of_a_very_long_row():
    """One query over 20 million keys of 128 channels: a channel's row begins more than
    2^31 elements behind the first."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    hd, tk = 128, 20_000_003
    g = torch.Generator(device="cuda:0").manual_seed(3)
    q = torch.randn((1, hd, 1), generator=g, device="cuda:0").to(torch.bfloat16)
    k, v = (torch.empty((1, hd, tk), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    for x in (k, v):
        for c in range(hd):
            x[0, c] = torch.randn(tk, generator=g, device="cuda:0").to(torch.bfloat16)
    desc = R.attention_desc(1, 1, 1, hd, 1, tk, R.BF16)
    need = R.rat3d_attention_workspace_size(desc, 0)
    o, lse = torch.empty_like(q), U.zeros_f32((1, 1, 1))
    R.rat3d_attention_fwd(desc, q, k, v, None, o, lse, _ws(need), need)
    U.sync()
    s = torch.zeros(tk, dtype=torch.float64, device="cuda:0")
    for c in range(hd):
        s += q[0, c, 0].double() * k[0, c].double()
    s *= hd ** -0.5
    want = torch.stack([(torch.softmax(s, 0) * v[0, c].double()).sum() for c in range(hd)])
    # probabilities and sums are float32: errors of 2^-24 a term, of random sign over
    # 2 * 10^7 of them, against a mean whose own terms have random signs too; the
    # rounding of the result is 2^-8 at most
    off = float((o[0, :, 0].double() - want).norm() / want.norm())
    assert off <= 2.0 ** -8 + 1e-4, off
    assert abs(float(lse) - float(torch.logsumexp(s, 0))) <= 1e-4


def test_calls_follow_the_current_stream():
    """Without a stream argument a call goes to the stream that is current then."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    other = torch.cuda.Stream()
    assert R._stream(None) == torch.cuda.current_stream().cuda_stream
    with torch.cuda.stream(other):
        assert R._stream(None) == other.cuda_stream
        # a call that waits for work of that stream only if it is enqueued there
        x = torch.ones(1 << 24, device="cuda:0")
        for _ in range(20):
            x.mul_(1.5).div_(1.5)
        y = torch.empty_like(x)
        R.rat3d_dropout_fwd(R.dropout_desc(x.numel(), 0.0, R.F32), 0, None, x, None, y)
    other.synchronize()
    assert torch.equal(x, y)
    assert R._stream(None) == torch.cuda.current_stream().cuda_stream != other.cuda_stream
    assert R._stream(123) == 123
