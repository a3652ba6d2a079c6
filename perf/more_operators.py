"""A recurrent block over the voxels of a volume, as timed cases: the norm of a
voxel's channels before the block, the gated linear recurrence along the voxels,
and the norm behind it with its gate, residual scale and residual.

Tensors are channel-first like every map of the library: a map [n][c][d][h][w]
holds one token a voxel, in memory order.  A 1^3 convolution behind the first norm
gives the recurrence's two gates, its values and the block's gate, side by side:

    u = norm(x);  r, i, v, g = conv(u);  h = recurrence(r, i, v);  z = conv(h);
    y = x + scale gate(g) norm(z),  and the next block's u = norm(y)

Sizes are those of the residual attention network's maps: 48 x 56 x 48 (stem of 32
and first partition of 64 channels), 24 x 28 x 24, 12 x 14 x 12 and 6 x 7 x 6 (the
stages of 64, 128 and 256 channels), and the first stage of 91 x 109 x 91 scans,
whose maps are odd.  Masks are the voxels of an ellipsoid, as a scan's brain mask is.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS, RATE = 1e-6, 8.0


def listed():
    return [
        # the norm before a block on the deepest map of one scan: a small call
        dict(name="pre_small_f32", op="pre", n=1, c=256, d=6, h=7, w=6, mask=False, dtype="f32"),
        # its gradient at the first stage's maps, with the residual's gradient added
        dict(name="pre_grad_bf16", op="pre_grad", n=8, c=64, d=24, h=28, w=24, mask=False,
             dtype="bf16"),
        # the norm behind a block for one read-out token a scan: latency counts
        dict(name="post_readout_bf16", op="post", n=8, c=256, d=1, h=1, w=1, gate="silu",
             next=True, mask=False, dtype="bf16"),
        # the same over the first partition's maps, one micro-batch of 16 scans: the largest
        dict(name="post_partition_bf16", op="post", n=16, c=64, d=48, h=56, w=48, gate="silu",
             next=True, mask=False, dtype="bf16"),
        # its gradients at the second stage's maps, all five inputs
        dict(name="post_grad_bf16", op="post_grad", n=16, c=128, d=12, h=14, w=12, gate="silu",
             next=True, mask=False, dtype="bf16"),
        # gradients on 91 x 109 x 91 scans' first stage inside the brain, the network's last block
        dict(name="post_grad_odd_f32", op="post_grad", n=2, c=64, d=23, h=28, w=23,
             gate="sigmoid", next=False, mask=True, dtype="f32"),
        # one more token of a sequence from the kept state, serving: the smallest call
        dict(name="scan_step_bf16", op="scan", n=8, c=256, d=1, h=1, w=1, reverse=False,
             mask=False, dtype="bf16"),
        # recurrence over the deepest map, one scan inside the brain
        dict(name="scan_small_f32", op="scan", n=1, c=256, d=6, h=7, w=6, reverse=False,
             mask=True, dtype="f32"),
        # over the first stage's maps from the last voxel on, inference
        dict(name="scan_bf16", op="scan", n=8, c=64, d=24, h=28, w=24, reverse=True, mask=False,
             dtype="bf16"),
        # a training pass on 91 x 109 x 91 scans' first stage inside the brain
        dict(name="scan_train_odd_f32", op="scan_train", n=2, c=64, d=23, h=28, w=23,
             reverse=True, mask=True, dtype="f32"),
        # a training pass over one scan's stem: few rows, long ones
        dict(name="scan_train_long_bf16", op="scan_train", n=1, c=32, d=48, h=56, w=48,
             reverse=False, mask=False, dtype="bf16"),
        # over the first partition's maps, one micro-batch of 16 scans: the largest
        dict(name="scan_train_bf16", op="scan_train", n=16, c=64, d=48, h=56, w=48,
             reverse=False, mask=False, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["pre", "pre_grad", "post", "post", "post_grad", "post_grad", "scan", "scan",
                     "scan_train", "scan_train"])
    if rng.random() < 0.15:  # a few tokens
        d, h, w = 1, 1, rng.randint(1, 9)
    else:
        base = _log(rng, 3, 50)
        d, h, w = (max(2, int(round(base * rng.uniform(0.85, 1.15)))) for _ in range(3))
    v = d * h * w
    c = _log(rng, 3, 300) if rng.random() < 0.5 else rng.choice([16, 32, 64, 64, 128, 256, 512])
    most = 1.2e8 if rng.random() < 0.5 else 2e7
    c = max(1, min(c, int(most / v)))
    n = _log(rng, 1, max(1, min(16, int(most / (v * c)))))
    case = dict(op=op, n=n, c=c, d=d, h=h, w=w, mask=v > 9 and rng.random() < 0.4,
                dtype="bf16" if rng.random() < 0.6 else "f32")
    if op in ("post", "post_grad"):
        case.update(gate=rng.choice(["none", "sigmoid", "silu"]), next=rng.random() < 0.5)
    if op in ("scan", "scan_train"):
        case["reverse"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _voxels(case):
    return case["d"] * case["h"] * case["w"]


def _brain(case, g):
    """uint8 [n][v]: 1 inside an ellipsoid whose centre varies a little."""
    n = case["n"]
    at = torch.rand((n, 3), generator=g, device=DEV) - 0.5
    far = 0.0
    for i, a in enumerate(("d", "h", "w")):
        x = torch.arange(case[a], device=DEV, dtype=torch.float32) - (case[a] - 1) / 2
        shape = [1, 1, 1, 1]
        shape[i + 1] = case[a]
        far = far + ((x.view(shape) - at[:, i].view(n, 1, 1, 1)) / (0.45 * case[a])) ** 2
    return (far <= 1.0).to(torch.uint8).view(n, -1).contiguous()


def _inputs(case, seed):
    """The inputs alone, the same for every form."""
    g, t = torch.Generator(device=DEV).manual_seed(int(seed) * 7907 + 13), _type(case)
    n, c, v, op = case["n"], case["c"], _voxels(case), case["op"]

    def randn(channels, scale=1.0):
        return (torch.randn((n, channels, v), generator=g, device=DEV) * scale).to(t)

    def gain(mean):
        return mean * (1.0 + 0.1 * torch.randn(c, generator=g, device=DEV))

    s = dict(mask=_brain(case, g) if case["mask"] else None)
    if op in ("pre", "pre_grad"):
        s.update(x=randn(c, 1.5), gamma=gain(1.0))
        if op == "pre_grad":
            s.update(du=randn(c, 1.0 / 64), dres=randn(c, 1.0 / 64))
        return s
    # the convolution's output holds the recurrence's gates and values, then the block's gate
    if op in ("post", "post_grad"):
        s.update(z=randn(c), gamma=gain(1.0), scale=gain(0.3),
                 wide=randn(4 * c) if case["gate"] != "none" else None,
                 gamma_next=gain(1.0) if case["next"] else None)
        if op == "post":
            s["x"] = randn(c, 1.5)
        else:
            s.update(y=randn(c, 1.5), dy=randn(c, 1.0 / 64),
                     du=randn(c, 1.0 / 64) if case["next"] else None)
        return s
    # decays of a closed gate up to an open one: u^(rate sigma(r)), u in 0.9 .. 0.999
    u = 0.9 + 0.099 * torch.rand(c, generator=g, device=DEV)
    s.update(wide=randn(4 * c), lam=torch.log(torch.expm1(-torch.log(u))),
             h0=torch.randn((n, c), generator=g, device=DEV))
    if op == "scan_train":
        s.update(dy=randn(c, 1.0 / 64),
                 dh=torch.randn((n, c), generator=g, device=DEV) / 64)
    return s


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    return state


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    e = float(case["n"]) * case["c"] * _voxels(case)
    op = case["op"]
    if op == "pre":
        tensors, flops = 2, 5
    elif op == "pre_grad":
        tensors, flops = 4, 12
    elif op == "post":
        tensors, flops = 3 + (case["gate"] != "none") + case["next"], 14
    elif op == "post_grad":
        tensors, flops = 3 + 2 * (case["gate"] != "none") + (3 if case["next"] else 0), 28
    elif op == "scan":
        tensors, flops = 4, 20
    else:
        tensors, flops = 8, 60
    return {"bytes": e * es * tensors + (case["n"] * _voxels(case) if case["mask"] else 0),
            "flops": flops * e}


# ------------------------------------------------------------------ plain forms
def _live(s):
    return None if s["mask"] is None else (s["mask"] != 0)[:, None, :]


def _only(t, live):
    return t if live is None else torch.where(live, t, torch.zeros((), device=DEV))


def _inv(t):
    return torch.rsqrt((t * t).mean(1, keepdim=True) + EPS)


def _norm_bwd(dz, x, gain, live):
    """Gradients of gain x / rms(x): of x, and of the gain."""
    dz, x = _only(dz.float(), live), _only(x.float(), live)
    inv = _inv(x)
    dg = (dz * x * inv).double().sum((0, 2)).float()
    u = dz * gain[:, None]
    return inv * (u - x * (inv * inv) * (u * x).mean(1, keepdim=True)), dg


def _phi(s):
    """The gate's value and slope."""
    case = s["case"]
    if case["gate"] == "none":
        return 1.0, None
    g = _only(s["wide"][:, 3 * case["c"]:].float(), _live(s))
    sg = torch.sigmoid(g)
    if case["gate"] == "sigmoid":
        return sg, sg * (1.0 - sg)
    return g * sg, sg * (1.0 + g * (1.0 - sg))


def _run_pre(s):
    live, x, gain = _live(s), s["x"], s["gamma"]
    if s["case"]["op"] == "pre":
        t = _only(x.float(), live)
        return dict(u=(t * _inv(t) * gain[:, None]).to(x.dtype))
    dx, dg = _norm_bwd(s["du"], x, gain, live)
    return dict(dx=(dx + s["dres"].float()).to(x.dtype), dgamma=dg)


def _run_post(s):
    case, live, to = s["case"], _live(s), s["z"].dtype
    gain, scale, nxt = s["gamma"][:, None], s["scale"][:, None], s["gamma_next"]
    z = _only(s["z"].float(), live)
    inv = _inv(z)
    phi, slope = _phi(s)
    if case["op"] == "post":
        y = s["x"].float() + _only(scale * phi * (gain * z * inv), live)
        out = dict(y=y.to(to))
        if nxt is not None:
            t = _only(y, live)
            out["u"] = (t * _inv(t) * nxt[:, None]).to(to)
        return out
    dy, out = s["dy"].float(), {}
    if nxt is not None:
        more, out["dgamma_next"] = _norm_bwd(s["du"], s["y"], nxt, live)
        dy = dy + more
        out["dx"] = dy.to(to)
    dy = _only(dy, live)
    total = (dy * phi * z * inv).double().sum((0, 2))
    out["dgamma"] = (s["scale"].double() * total).float()
    out["dscale"] = (s["gamma"].double() * total).float()
    if slope is not None:
        out["dg"] = (dy * scale * gain * z * inv * slope).to(to)
    e = dy * scale * gain * phi
    out["dz"] = (inv * (e - z * (inv * inv) * (e * z).mean(1, keepdim=True))).to(to)
    return out


def _scan(a, b, h0, reverse):
    """h_t = a_t h_{t-1} + b_t: steps joined in pairs, then pairs of pairs (a and b are
    overwritten)."""
    t = a.shape[-1]
    first = t - 1 if reverse else 0
    b[..., first] += a[..., first] * h0
    step = 1
    while step < t:
        here, there = slice(step, None), slice(None, t - step)  # a token, and its past
        if reverse:
            here, there = there, here
        b[..., here] = b[..., here] + a[..., here] * b[..., there]
        a[..., here] = a[..., here] * a[..., there]
        step *= 2
    return b


def _shift(t, edge, reverse):
    """Every token gets what the token before it has, the first one `edge`."""
    if reverse:
        return torch.cat([t[..., 1:], edge[..., None]], dim=-1)
    return torch.cat([edge[..., None], t[..., :-1]], dim=-1)


def _run_scan(s):
    case, live, c, rev = s["case"], _live(s), s["case"]["c"], s["case"]["reverse"]
    r, i, x = (_only(s["wide"][:, k * c:(k + 1) * c].float(), live) for k in range(3))
    to = s["wide"].dtype
    soft = torch.nn.functional.softplus(s["lam"].double()).float()
    sr, si = torch.sigmoid(r), torch.sigmoid(i)
    la = _only(-RATE * soft[:, None] * sr, live)
    a = torch.exp(la)
    beta = torch.sqrt(-torch.expm1(2.0 * la))
    b = beta * si * x
    h = _scan(a.clone(), b, s["h0"], rev)
    out = dict(y=_only(h, live).to(to), h_last=h[..., 0 if rev else -1].clone())
    if case["op"] == "scan":
        return out
    # e_t = a_t (dy_t + e_{t+1}) is what a token hands on to the one before it
    dy = _only(s["dy"].float(), live)
    e = _scan(a.clone(), a * dy, s["dh"], not rev)
    out["dh0"] = e[..., -1 if rev else 0].clone()
    d = dy + _shift(e, s["dh"], not rev)
    del e
    past = _shift(h, s["h0"], rev)
    k = d * la * a * past - d * si * x * a * a * torch.where(
        beta > 0, la / torch.where(beta > 0, beta, torch.ones_like(beta)), torch.zeros_like(beta))
    out["dr"] = _only(k * torch.sigmoid(-r), live).to(to)
    ratio = torch.sigmoid(s["lam"].double()) / torch.nn.functional.softplus(s["lam"].double())
    out["dlam"] = (ratio * k.double().sum((0, 2))).float()
    out["di"] = _only(d * beta * x * si * torch.sigmoid(-i), live).to(to)
    out["dx"] = _only(d * beta * si, live).to(to)
    return out


# ------------------------------------------------------------------ the library's calls
GATES = {"none": 0, "sigmoid": 1, "silu": 2}


def _own_norm(s):
    from paper_2104_05035_amd import rat3d as R
    case, op = s["case"], s["case"]["op"]
    n, c, v = case["n"], case["c"], _voxels(case)
    if "plan" not in s:  # descriptor, workspace and buffers: kept by a program
        t = s["x"] if "x" in s else s["z"]
        gate = case.get("gate", "none")
        desc = R.norm_desc(n, c, v, R.dtype_code(t.dtype), gate=GATES[gate], eps=EPS,
                           g_stride=4 * c * v if gate != "none" else 0)
        need = R.rat3d_norm_workspace_size(desc) if op.endswith("grad") else 0
        b = s["plan"] = dict(desc=desc, need=need,
                             ws=torch.empty(max(need, 16), dtype=torch.uint8, device=DEV))
        nxt = case.get("next", False)
        if op in ("pre", "post"):
            b.update(y=torch.empty_like(t), u=torch.empty_like(t) if op == "pre" or nxt else None)
        else:
            b.update(dx=torch.empty_like(t) if op == "pre_grad" or nxt else None,
                     dz=torch.empty_like(t),
                     **{k: torch.empty(c, device=DEV) for k in ("dgamma", "dscale")})
            b["dgamma_next"] = torch.empty(c, device=DEV) if nxt else None
        b["g"] = b["dg"] = None
        if gate != "none":
            b["g"] = s["wide"][:, 3 * c:]
            if op == "post_grad":  # it lies where the convolution before wants it
                b["dg"] = torch.zeros_like(s["wide"])[:, 3 * c:]
    b = s["plan"]
    if op == "pre":
        R.rat3d_pre_norm_fwd(b["desc"], s["x"], s["gamma"], s["mask"], b["u"])
        return dict(u=b["u"])
    if op == "pre_grad":
        R.rat3d_pre_norm_bwd(b["desc"], s["du"], s["x"], s["gamma"], s["mask"], s["dres"], b["dx"],
                             b["dgamma"], 0, b["ws"], b["need"])
        return dict(dx=b["dx"], dgamma=b["dgamma"])
    if op == "post":
        R.rat3d_post_norm_fwd(b["desc"], s["x"], s["z"], b["g"], s["gamma"], s["scale"],
                              s["gamma_next"], s["mask"], b["y"], b["u"])
        return dict(y=b["y"], **({"u": b["u"]} if case["next"] else {}))
    R.rat3d_post_norm_bwd(b["desc"], s["dy"], s["du"], s["y"], s["z"], b["g"], s["gamma"],
                          s["scale"], s["gamma_next"], s["mask"], b["dx"], b["dz"], b["dg"],
                          b["dgamma"], b["dscale"], b["dgamma_next"], 0, b["ws"], b["need"])
    return {k: b[k] for k in _post_grads(case)}


def _post_grads(case):
    return ((("dgamma_next", "dx") if case["next"] else ()) + ("dgamma", "dscale") +
            (("dg",) if case["gate"] != "none" else ()) + ("dz",))


def _own_scan(s):
    from paper_2104_05035_amd import rat3d as R
    case, train = s["case"], s["case"]["op"] == "scan_train"
    n, c, v, x = case["n"], case["c"], _voxels(case), s["wide"]
    if "plan" not in s:
        wide = 4 * c * v
        desc = R.recurrence_desc(n, c, v, R.dtype_code(x.dtype), reverse=case["reverse"],
                                 rate=RATE, r_stride=wide, i_stride=wide, x_stride=wide)
        need = max(R.rat3d_recurrence_workspace_size(desc, p) for p in range(1 + train))
        b = s["plan"] = dict(desc=desc, need=need, r=x[:, :c], i=x[:, c:2 * c], x=x[:, 2 * c:3 * c],
                             ws=torch.empty(max(need, 16), dtype=torch.uint8, device=DEV),
                             y=torch.empty((n, c, v), dtype=x.dtype, device=DEV),
                             h_last=torch.empty((n, c), device=DEV), carry=None)
        if train:  # the gradients lie side by side as r, i and x do
            dx = torch.zeros_like(x)
            b.update(dr=dx[:, :c], di=dx[:, c:2 * c], dx=dx[:, 2 * c:3 * c],
                     dlam=torch.empty(c, device=DEV), dh0=torch.empty((n, c), device=DEV),
                     carry=torch.empty(max(R.rat3d_recurrence_carry_size(desc), 16),
                                       dtype=torch.uint8, device=DEV))
    b = s["plan"]
    R.rat3d_recurrence_fwd(b["desc"], b["r"], b["i"], b["x"], s["lam"], s["mask"], s["h0"], b["y"],
                           b["h_last"], b["carry"], b["ws"], b["need"])
    if not train:
        return dict(y=b["y"], h_last=b["h_last"])
    R.rat3d_recurrence_bwd(b["desc"], s["dy"], s["dh"], b["r"], b["i"], b["x"], s["lam"],
                           s["mask"], b["carry"], b["dr"], b["di"], b["dx"], b["dlam"], b["dh0"],
                           0, b["ws"], b["need"])
    return {k: b[k] for k in ("y", "h_last", "dh0", "dr", "dlam", "di", "dx")}


def run(state):
    op = state["case"]["op"]
    if own:
        return _own_scan(state) if op.startswith("scan") else _own_norm(state)
    return (_run_scan if op.startswith("scan") else
            _run_pre if op.startswith("pre") else _run_post)(state)


# ------------------------------------------------------------------ definitions in 64 bits
def _exact_norm(x, gain):
    """Gain times x over its root mean square, for tokens as rows."""
    return x / torch.sqrt(torch.sum(x ** 2, 1, keepdim=True) / x.shape[1] + EPS) * gain


def _rows(t, live):
    """[n][c][v] to the live tokens as rows, float64."""
    t = t.double().permute(0, 2, 1)
    return t[live] if live is not None else t.reshape(-1, t.shape[2])


def _maps(rows, like, live, rest=None):
    """Back to [n][c][v]; masked tokens hold `rest` or zeros."""
    n, c, v = like.shape
    t = torch.zeros((n, v, c), dtype=torch.float64, device=DEV) if rest is None else \
        rest.double().permute(0, 2, 1).clone()
    if live is None:
        t.copy_(rows.reshape(n, v, c))
    else:
        t[live] = rows
    return t.permute(0, 2, 1)


def _exact_norms(case, s):
    live = None if s["mask"] is None else s["mask"] != 0
    op, gamma = case["op"], s["gamma"].double()
    if op == "pre":
        return dict(u=_maps(_exact_norm(_rows(s["x"], live), gamma), s["x"], live))
    if op == "pre_grad":
        x = _rows(s["x"], live).requires_grad_()
        gamma.requires_grad_()
        dx, dg = torch.autograd.grad(_exact_norm(x, gamma), (x, gamma), _rows(s["du"], live))
        return dict(dx=_maps(dx + _rows(s["dres"], live), s["x"], live, s["dres"]), dgamma=dg)
    z, scale = _rows(s["z"], live), s["scale"].double()
    nxt = s["gamma_next"].double() if case["next"] else None
    gated = case["gate"] != "none"
    wide = s["wide"][:, 3 * case["c"]:] if gated else None
    g = _rows(wide, live) if gated else None

    def branch():
        t = scale * _exact_norm(z, gamma)
        if gated:
            t = t / (1.0 + torch.exp(-g))
        return t * g if case["gate"] == "silu" else t

    if op == "post":
        y = _rows(s["x"], live) + branch()
        out = dict(y=_maps(y, s["x"], live, s["x"]))
        if case["next"]:
            out["u"] = _maps(_exact_norm(y, nxt), s["x"], live)
        return out
    dy, out = _rows(s["dy"], live), {}
    if case["next"]:
        y = _rows(s["y"], live).requires_grad_()
        nxt.requires_grad_()
        more, out["dgamma_next"] = torch.autograd.grad(_exact_norm(y, nxt), (y, nxt),
                                                       _rows(s["du"], live))
        dy = dy + more
        out["dx"] = _maps(dy, s["y"], live, s["dy"])
    leaves = dict(dgamma=gamma, dscale=scale, dg=g, dz=z)
    leaves = {k: t.requires_grad_() for k, t in leaves.items() if t is not None}
    out.update(zip(leaves, torch.autograd.grad(branch(), tuple(leaves.values()), dy)))
    for k in ("dg", "dz"):
        if k in out:
            out[k] = _maps(out[k], s["z"], live)
    return out


def _exact_line(a, b, h0):
    """h_t = a_t h_{t-1} + b_t along the last axis, float64: the tokens in blocks, whose
    tokens are taken one after another for all blocks at once, then block after block."""
    t = a.shape[-1]
    size = max(1, int(math.sqrt(t)))
    blocks = -(-t // size)
    lead = a.shape[:-1]
    pad = blocks * size - t

    def cut(x, fill):  # [size][lead][blocks]
        x = torch.cat([x, torch.full(lead + (pad,), fill, dtype=x.dtype, device=DEV)], dim=-1)
        return x.view(lead + (blocks, size)).movedim(-1, 0).contiguous()

    a, b = cut(a, 1.0), cut(b, 0.0)
    for j in range(1, size):
        b[j] += a[j] * b[j - 1]
        a[j] *= a[j - 1]
    state = h0.double()
    start = torch.empty(lead + (blocks,), dtype=torch.float64, device=DEV)
    for k in range(blocks):
        start[..., k] = state
        state = a[-1, ..., k] * state + b[-1, ..., k]
    h = b + a * start
    return h.movedim(0, -1).reshape(lead + (-1,))[..., :t], state


def _exact_scan(case, s):
    c, rev = case["c"], case["reverse"]
    turn = (lambda t: t.flip(-1)) if rev else (lambda t: t)
    r, i, x = (turn(s["wide"][:, k * c:(k + 1) * c]).double() for k in range(3))
    lam = s["lam"].double()[:, None]
    soft = torch.log1p(torch.exp(lam))
    open_r, open_i = 1.0 / (1.0 + torch.exp(-r)), 1.0 / (1.0 + torch.exp(-i))
    log_a = -RATE * soft * open_r
    live = None if s["mask"] is None else turn(s["mask"] != 0)[:, None, :].expand_as(r)
    if live is not None:
        log_a = torch.where(live, log_a, 0.0)
    a = torch.exp(log_a)
    beta = torch.sqrt(-torch.expm1(2 * log_a))  # 0 where masked
    h, last = _exact_line(a, beta * open_i * x, s["h0"])
    shown = h if live is None else torch.where(live, h, 0.0)
    out = dict(y=turn(shown), h_last=last)
    if case["op"] == "scan":
        return out
    dy = turn(s["dy"]).double()
    if live is not None:
        dy = torch.where(live, dy, 0.0)
    # the state's gradient, from the end: dh_t = dy_t + a_{t+1} dh_{t+1}
    back = torch.cat([a[..., 1:], torch.ones_like(a[..., :1])], dim=-1).flip(-1)
    dh = _exact_line(back, dy.flip(-1), s["dh"])[0].flip(-1)
    out["dh0"] = dh[..., 0] * a[..., 0]
    del back
    db = dh
    past = torch.cat([s["h0"].double()[..., None], h[..., :-1]], dim=-1)
    dbeta = db * open_i * x
    dlog = dh * past * a - torch.where(beta > 0, dbeta * a * a / beta, 0.0)
    if live is not None:
        dlog = torch.where(live, dlog, 0.0)
    out["dr"] = turn(dlog * -RATE * soft * open_r * (1.0 - open_r))
    out["dlam"] = (dlog * -RATE * open_r / (1.0 + torch.exp(-lam))).sum((0, 2))
    out["di"] = turn(db * beta * x * open_i * (1.0 - open_i))
    out["dx"] = turn(db * beta * open_i)
    return out


def exact(case, seed):
    """The outputs of `run` from the operators' definitions in 64 bits."""
    s = _inputs(case, seed)
    return _exact_scan(case, s) if case["op"].startswith("scan") else _exact_norms(case, s)
