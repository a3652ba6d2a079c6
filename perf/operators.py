"""Token self-attention over the voxels of a volume, as timed cases: the head
norms with the rotation by the voxel's place, the attention itself, and the
dropout of the residual branch.

Tensors are channel-first like every map of the library: a map [n][c][d][h][w]
holds one token a voxel, its channels are heads x head_dim, and queries, keys
and values are channel ranges of the output of one 1^3 convolution.

Sizes are those of the residual attention network's maps: 48 x 56 x 48 (first
partition, 64 channels), 24 x 28 x 24, 12 x 14 x 12 and 6 x 7 x 6 (the stages
of 64, 128 and 256 channels), and the same stages of 91 x 109 x 91 scans,
whose maps are odd in every axis.  Masks are the voxels of an ellipsoid, as a
scan's brain mask is.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS, BASE = 1e-6, 100.0


def listed():
    return [
        # head norms and rotation of the deepest map, one scan: the smallest call
        dict(name="qk_small_f32", op="qk", n=1, heads=4, kv=4, hd=64, d=6, h=7, w=6, origin=0,
             dtype="f32"),
        # the first partition's maps, one micro-batch of 16 scans: the largest
        dict(name="qk_partition_bf16", op="qk", n=16, heads=2, kv=2, hd=32, d=48, h=56, w=48,
             origin=0, dtype="bf16"),
        # gradients at the first stage's maps, two query heads to a key head
        dict(name="qk_grad_bf16", op="qk_grad", n=8, heads=4, kv=2, hd=32, d=24, h=28, w=24,
             origin=0, dtype="bf16"),
        # gradients on a 91 x 109 x 91 scan's first stage, a crop of a larger volume
        dict(name="qk_grad_odd_f32", op="qk_grad", n=2, heads=3, kv=3, hd=40, d=23, h=28, w=23,
             origin=91, dtype="f32"),
        # attention over the second stage's maps inside the brain, inference
        dict(name="attn_mask_bf16", op="attn", n=8, heads=4, kv=4, hd=32, d=12, h=14, w=12,
             tq=0, mask=True, dtype="bf16"),
        # one read-out token a scan over the partition's full-resolution map
        dict(name="attn_readout_bf16", op="attn", n=8, heads=4, kv=2, hd=32, d=48, h=56, w=48,
             tq=1, mask=False, dtype="bf16"),
        # a training pass over the deepest map, float32: short rows, few tiles
        dict(name="attn_train_small_f32", op="attn_train", n=2, heads=4, kv=4, hd=64, d=6, h=7,
             w=6, tq=0, mask=False, dtype="f32"),
        # a training pass over the first stage's maps: the largest
        dict(name="attn_train_bf16", op="attn_train", n=4, heads=2, kv=2, hd=64, d=24, h=28, w=24,
             tq=0, mask=False, dtype="bf16"),
        # the same of 91 x 109 x 91 scans at the second stage: odd sizes, masked, grouped heads
        dict(name="attn_train_odd_bf16", op="attn_train", n=4, heads=6, kv=2, hd=40, d=12, h=14,
             w=11, tq=0, mask=True, dtype="bf16"),
        # and in float32, the precision of the paper's runs
        dict(name="attn_train_f32", op="attn_train", n=2, heads=4, kv=4, hd=32, d=12, h=14, w=12,
             tq=0, mask=False, dtype="f32"),
        # the residual branch's dropout over the partition's maps, forward and gradient
        dict(name="dropout_bf16", op="dropout", n=16, c=64, d=48, h=56, w=48, unit="element",
             p=0.1, residual=True, dtype="bf16"),
        # whole channels dropped, odd maps, float32
        dict(name="dropout_channel_f32", op="dropout", n=2, c=64, d=23, h=28, w=23,
             unit="channel", p=0.25, residual=False, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["qk", "qk_grad", "attn", "attn", "attn_train", "attn_train", "readout",
                     "dropout"])
    dt = "bf16" if rng.random() < 0.6 else "f32"
    kv = rng.choice([1, 1, 2, 2, 3, 4])
    heads = kv * rng.choice([1, 1, 1, 2, 3])
    hd = rng.choice([16, 24, 32, 32, 40, 48, 64, 64, 80, 96, 128])
    side = {"qk": 48, "qk_grad": 40, "attn": 25, "attn_train": 22, "readout": 48,
            "dropout": 48}[op]
    base = _log(rng, 4, side)
    d, h, w = (max(3, int(round(base * rng.uniform(0.85, 1.15)))) for _ in range(3))
    v = d * h * w
    if op == "dropout":
        c = rng.choice([3, 16, 32, 64, 64, 128, 256])
        n = _log(rng, 1, max(1, min(16, int(1.2e8 / (v * c)))))
        return dict(op=op, n=n, c=c, d=d, h=h, w=w,
                    unit=rng.choice(["element", "element", "channel", "volume"]),
                    p=rng.choice([0.05, 0.1, 0.2, 0.25, 0.5]), residual=rng.random() < 0.5,
                    dtype=dt)
    if op in ("qk", "qk_grad"):
        n = _log(rng, 1, max(1, min(16, int(6e7 / (v * heads * hd)))))
        return dict(op=op, n=n, heads=heads, kv=kv, hd=hd, d=d, h=h, w=w,
                    origin=rng.choice([0, 0, 91, rng.randint(0, 4096)]), dtype=dt)
    case = dict(op="attn" if op == "readout" else op, heads=heads, kv=kv, hd=hd, d=d, h=h, w=w,
                mask=rng.random() < 0.5, dtype=dt)
    if op == "readout":
        case["tq"] = rng.choice([1, 1, 1, 2, 4])
        case["n"] = _log(rng, 1, max(1, min(16, int(6e7 / (v * kv * hd)))))
        return case
    # mostly self-attention; else some query tokens of another map
    case["tq"] = rng.choice([0, 0, 0, _log(rng, 5, v)])
    t = case["tq"] or v
    most = (6.0e11 if op == "attn" else 1.0e12) * (1 if dt == "bf16" else 0.2)
    one = (4 if op == "attn" else 14) * heads * hd * float(t) * v
    case["n"] = _log(rng, 1, max(1, min(16, int(most / one))))
    return case


# ------------------------------------------------------------------ inputs
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 6271 + 29)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def _axes(case):
    """Semi-axes of the mask's ellipsoid, in voxels."""
    return [0.45 * case[a] for a in ("d", "h", "w")]


def _brain(case, g):
    """uint8 [n][d][h][w]: 1 inside an ellipsoid whose centre varies a little."""
    n = case["n"]
    at = torch.rand((n, 3), generator=g, device=DEV) - 0.5
    far = 0.0
    for i, (a, r) in enumerate(zip(("d", "h", "w"), _axes(case))):
        x = torch.arange(case[a], device=DEV, dtype=torch.float32) - (case[a] - 1) / 2
        shape = [1, 1, 1, 1]
        shape[i + 1] = case[a]
        far = far + ((x.view(shape) - at[:, i].view(n, 1, 1, 1)) / r) ** 2
    return (far <= 1.0).to(torch.uint8).view(n, -1).contiguous()


def _inputs(case, seed):
    """The inputs alone, the same for every form."""
    g, t = _gen(seed), _type(case)
    v = case["d"] * case["h"] * case["w"]
    n = case["n"]
    if case["op"] == "dropout":
        shape = (n, case["c"], v)
        x = _randn(g, shape, t)
        return dict(x=x, residual=_randn(g, shape, t) if case["residual"] else None,
                    dy=_randn(g, shape, t, 1.0 / 64), seed=int(seed) * 104729 + 3,
                    step=int(seed) % 1000 + 5)
    heads, kv, hd = case["heads"], case["kv"], case["hd"]
    if case["op"] in ("qk", "qk_grad"):
        # queries, keys and values come out of one 1^3 convolution, side by side
        s = dict(qkv=_randn(g, (n, (heads + 2 * kv) * hd, v), t, 1.3),
                 gq=1.0 + 0.1 * torch.randn(hd, generator=g, device=DEV),
                 gk=1.0 + 0.1 * torch.randn(hd, generator=g, device=DEV))
        if case["op"] == "qk_grad":
            s["dq"] = _randn(g, (n, heads * hd, v), t, 1.0 / 64)
            s["dk"] = _randn(g, (n, kv * hd, v), t, 1.0 / 64)
        return s
    tq = case["tq"] or v
    s = dict(q=_randn(g, (n, heads * hd, tq), t), k=_randn(g, (n, kv * hd, v), t),
             v=_randn(g, (n, kv * hd, v), t),
             mask=_brain(case, g) if case["mask"] else None)
    if case["op"] == "attn_train":
        s["do"] = _randn(g, (n, heads * hd, tq), t, 1.0 / 64)
    return s


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    return state


def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    v, n = case["d"] * case["h"] * case["w"], case["n"]
    if case["op"] == "dropout":
        e = float(n) * case["c"] * v
        return {"bytes": e * es * (4 + case["residual"]), "flops": 2.0 * e}
    heads, kv, hd = case["heads"], case["kv"], case["hd"]
    if case["op"] in ("qk", "qk_grad"):
        e = float(n) * (heads + kv) * hd * v
        grad = case["op"] == "qk_grad"
        return {"bytes": e * es * (3 if grad else 2), "flops": (16.0 if grad else 8.0) * e}
    tq = case["tq"] or v
    live = float(v)
    if case["mask"]:  # the voxels of the ellipsoid
        a, b, c = _axes(case)
        live = min(live, 4.0 / 3.0 * math.pi * a * b * c)
    q, k = float(n) * heads * hd * tq, float(n) * kv * hd * live
    train = case["op"] == "attn_train"
    whole = float(n) * kv * hd * v  # gradients of masked keys are written too
    moved = (2 * q + 2 * k) if not train else (4 * q + 2 * k + 2 * whole)
    return {"bytes": moved * es + (n * v if case["mask"] else 0),
            "flops": (14.0 if train else 4.0) * float(n) * heads * hd * tq * live}


# ------------------------------------------------------------------ plain forms
def _rot(case):
    """Channels of a head that each axis turns."""
    return 2 * (case["hd"] // 6)


def _angles(case):
    """Angles [pairs][v], in 64 bits: the three axes one after another."""
    r = _rot(case)
    f = BASE ** (-2.0 * torch.arange(r // 2, device=DEV, dtype=torch.float64) / r)
    i = torch.arange(case["d"] * case["h"] * case["w"], device=DEV)
    hw, w = case["h"] * case["w"], case["w"]
    at = torch.stack([i // hw, i // w % case["h"], i % w]) + case["origin"]
    return (at.to(torch.float64)[:, None, :] * f[None, :, None]).reshape(3 * (r // 2), -1)


def _turn(x, cos, sin, r, back=False):
    """x [..., hd, v]: channels a*r + i and a*r + r/2 + i of axis a are one pair."""
    lead, v = x.shape[:-2], x.shape[-1]
    t = x[..., :3 * r, :].reshape(lead + (3, 2, r // 2, v))
    c, s = cos.view(3, r // 2, v), sin.view(3, r // 2, v)
    s = -s if back else s
    a, b = t[..., 0, :, :], t[..., 1, :, :]
    y = torch.stack([a * c - b * s, a * s + b * c], dim=-3).reshape(lead + (3 * r, v))
    return torch.cat([y, x[..., 3 * r:, :]], dim=-2)


def _qk_fwd(x, gain, cos, sin, r, to):
    x = x.float()
    z = x * torch.rsqrt((x * x).mean(-2, keepdim=True) + EPS) * gain[:, None]
    return _turn(z, cos, sin, r).to(to)


def _qk_bwd(dy, x, gain, cos, sin, r, to):
    x, dz = x.float(), _turn(dy.float(), cos, sin, r, back=True)
    inv = torch.rsqrt((x * x).mean(-2, keepdim=True) + EPS)
    dg = (dz * x * inv).double().sum((0, 1, 3)).float()
    u = dz * gain[:, None]
    dx = inv * (u - x * inv * inv * (u * x).mean(-2, keepdim=True))
    return dx.to(to), dg


def _run_qk(s):
    case = s["case"]
    n, heads, kv, hd = case["n"], case["heads"], case["kv"], case["hd"]
    r, to = _rot(case), s["qkv"].dtype
    q = s["qkv"][:, :heads * hd].reshape(n, heads, hd, -1)
    k = s["qkv"][:, heads * hd:(heads + kv) * hd].reshape(n, kv, hd, -1)
    ang = _angles(case)
    cos, sin = ang.cos().float(), ang.sin().float()
    if case["op"] == "qk":
        y, z = _qk_fwd(q, s["gq"], cos, sin, r, to), _qk_fwd(k, s["gk"], cos, sin, r, to)
        return dict(q=y.view(n, heads * hd, -1), k=z.view(n, kv * hd, -1))
    dq, dgq = _qk_bwd(s["dq"].view(q.shape), q, s["gq"], cos, sin, r, to)
    dk, dgk = _qk_bwd(s["dk"].view(k.shape), k, s["gk"], cos, sin, r, to)
    return dict(dq=dq.reshape(n, heads * hd, -1), dk=dk.reshape(n, kv * hd, -1), dgq=dgq, dgk=dgk)


def _run_attn(s):
    case = s["case"]
    n, heads, kv, hd = case["n"], case["heads"], case["kv"], case["hd"]
    to, scale, grp = s["q"].dtype, case["hd"] ** -0.5, heads // kv
    q = s["q"].float().view(n, heads, hd, -1)
    k = s["k"].float().view(n, kv, hd, -1).repeat_interleave(grp, dim=1)
    v = s["v"].float().view(n, kv, hd, -1).repeat_interleave(grp, dim=1)
    p = torch.matmul(q.transpose(2, 3).contiguous(), k).mul_(scale)  # [n][heads][tq][tk]
    if s["mask"] is not None:
        p.masked_fill_((s["mask"] == 0)[:, None, None, :], -math.inf)
    m = p.amax(-1, keepdim=True)
    p.sub_(torch.where(m == -math.inf, torch.zeros_like(m), m)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, torch.ones_like(total), total))
    o = torch.matmul(v, p.transpose(2, 3))  # [n][heads][hd][tq]
    out = dict(o=o.to(to).reshape(n, heads * hd, -1))
    if case["op"] == "attn_train":
        do = s["do"].float().view(n, heads, hd, -1)
        dv = torch.matmul(do, p).view(n, kv, grp, hd, -1).sum(2)
        ds = torch.matmul(do.transpose(2, 3).contiguous(), v)
        ds.sub_((do * o).sum(2)[..., None]).mul_(p).mul_(scale)
        dq = torch.matmul(k, ds.transpose(2, 3))
        dk = torch.matmul(q, ds).view(n, kv, grp, hd, -1).sum(2)
        out.update(dq=dq.to(to).reshape(n, heads * hd, -1),
                   dk=dk.to(to).reshape(n, kv * hd, -1), dv=dv.to(to).reshape(n, kv * hd, -1))
    return out


def _unit(case):
    """Neighbouring elements that share one decision."""
    v = case["d"] * case["h"] * case["w"]
    return {"element": 1, "channel": v, "volume": case["c"] * v}[case["unit"]]


def _philox(blocks, step, seed):
    """Philox4x32 with ten rounds (Salmon et al. 2011): the four 32-bit words
    of counters (block, step) under the key `seed`, as int64 [4][blocks]."""
    low = 0xffffffff
    i = torch.arange(blocks, device=DEV)
    c0, c1 = i & low, i >> 32
    c2, c3 = torch.full_like(i, step & low), torch.full_like(i, step >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # modulo 2^64: the bits are the product's
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3])


def _run_dropout(s):
    case, x = s["case"], s["x"]
    unit = _unit(case)
    units = x.numel() // unit
    words = _philox((units + 7) // 8, s["step"], s["seed"])  # eight decisions of 16 bits each
    lots = torch.stack([words & 0xffff, words >> 16], dim=1).permute(2, 0, 1).reshape(-1)[:units]
    at = int(round(case["p"] * 65536))
    keep = (lots >= at).view(-1, 1).expand(-1, unit).reshape(x.shape)
    scale = 65536.0 / (65536 - at)
    zero = torch.zeros((), device=DEV)
    y = torch.where(keep, x.float() * scale, zero)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(x.dtype), dx=torch.where(keep, s["dy"].float() * scale, zero).to(x.dtype))


# ------------------------------------------------------------------ the library's calls
def _own_qk(s):
    from paper_2104_05035_amd import rat3d as R
    case, x = s["case"], s["qkv"]
    n, heads, kv, hd = case["n"], case["heads"], case["kv"], case["hd"]
    v = x.shape[2]
    if "plan" not in s:  # descriptor, table of angles and buffers: kept by a program
        dt = R.dtype_code(x.dtype)
        at = case["origin"]
        desc = R.qk_desc(n, heads, kv, hd, case["d"], case["h"], case["w"], dt,
                         rot=(_rot(case),) * 3, origin=(at,) * 3, base=BASE, eps=EPS,
                         q_stride=x.shape[1] * v, k_stride=x.shape[1] * v)
        table = torch.empty(R.rat3d_rope_table_size(desc), dtype=torch.uint8, device=DEV)
        R.rat3d_rope_table(desc, table)
        need = R.rat3d_qk_norm_rope_workspace_size(desc)
        s["plan"] = dict(
            desc=desc, table=table, q=x[:, :heads * hd], k=x[:, heads * hd:(heads + kv) * hd],
            need=need, ws=torch.empty(max(need, 16), dtype=torch.uint8, device=DEV),
            dgq=torch.empty(hd, device=DEV), dgk=torch.empty(hd, device=DEV))
        if case["op"] == "qk":
            s["plan"].update(oq=torch.empty((n, heads * hd, v), dtype=x.dtype, device=DEV),
                             ok=torch.empty((n, kv * hd, v), dtype=x.dtype, device=DEV))
        else:  # the gradients lie side by side as q and k do, for the convolution before
            dx = torch.zeros_like(x)
            s["plan"].update(dq=dx[:, :heads * hd], dk=dx[:, heads * hd:(heads + kv) * hd])
    b = s["plan"]
    if case["op"] == "qk":
        R.rat3d_qk_norm_rope_fwd(b["desc"], b["q"], b["k"], s["gq"], s["gk"], b["table"], b["oq"],
                                 b["ok"])
        return dict(q=b["oq"], k=b["ok"])
    R.rat3d_qk_norm_rope_bwd(b["desc"], s["dq"], s["dk"], b["q"], b["k"], s["gq"], s["gk"],
                             b["table"], b["dq"], b["dk"], b["dgq"], b["dgk"], 0, b["ws"],
                             b["need"])
    return dict(dq=b["dq"], dk=b["dk"], dgq=b["dgq"], dgk=b["dgk"])


def _own_attn(s):
    from paper_2104_05035_amd import rat3d as R
    case, train = s["case"], s["case"]["op"] == "attn_train"
    if "plan" not in s:
        n, heads, tq = case["n"], case["heads"], s["q"].shape[2]
        desc = R.attention_desc(n, heads, case["kv"], case["hd"], tq, s["k"].shape[2],
                                R.dtype_code(s["q"].dtype))
        need = max(R.rat3d_attention_workspace_size(desc, i) for i in range(1 + train))
        s["plan"] = dict(desc=desc, need=need, o=torch.empty_like(s["q"]),
                         ws=torch.empty(max(need, 16), dtype=torch.uint8, device=DEV),
                         lse=torch.empty((n, heads, tq), device=DEV) if train else None)
        if train:
            s["plan"].update(dq=torch.empty_like(s["q"]), dk=torch.empty_like(s["k"]),
                             dv=torch.empty_like(s["v"]))
    b = s["plan"]
    R.rat3d_attention_fwd(b["desc"], s["q"], s["k"], s["v"], s["mask"], b["o"], b["lse"], b["ws"],
                          b["need"])
    if not train:
        return dict(o=b["o"])
    R.rat3d_attention_bwd(b["desc"], s["do"], s["q"], s["k"], s["v"], s["mask"], b["o"], b["lse"],
                          b["dq"], b["dk"], b["dv"], b["ws"], b["need"])
    return dict(o=b["o"], dq=b["dq"], dk=b["dk"], dv=b["dv"])


def _own_dropout(s):
    from paper_2104_05035_amd import rat3d as R
    x = s["x"]
    if "plan" not in s:
        s["plan"] = dict(desc=R.dropout_desc(x.numel(), s["case"]["p"], R.dtype_code(x.dtype),
                                             seed=s["seed"], unit=_unit(s["case"])),
                         y=torch.empty_like(x), dx=torch.empty_like(x))
    b = s["plan"]
    R.rat3d_dropout_fwd(b["desc"], s["step"], None, x, s["residual"], b["y"])
    R.rat3d_dropout_bwd(b["desc"], s["step"], None, s["dy"], b["dx"], 0)
    return dict(y=b["y"], dx=b["dx"])


def run(state):
    op = state["case"]["op"]
    if own:
        f = _own_qk if op in ("qk", "qk_grad") else _own_dropout if op == "dropout" else _own_attn
    else:
        f = _run_qk if op in ("qk", "qk_grad") else _run_dropout if op == "dropout" else _run_attn
    return f(state)


# ------------------------------------------------------------------ definitions in 64 bits
def _rotation(case):
    """R [v][hd][hd] in float64, with z -> R z the turning of one head."""
    hd, r = case["hd"], _rot(case)
    at = np.stack(np.meshgrid(*(np.arange(case[a], dtype=np.float64) + case["origin"]
                                for a in ("d", "h", "w")), indexing="ij")).reshape(3, -1)
    m = np.zeros((at.shape[1], hd, hd))
    m[:, np.arange(hd), np.arange(hd)] = 1.0
    for axis in range(3):
        for i in range(r // 2):
            t = at[axis] * BASE ** (-2.0 * i / r)
            a, b = axis * r + i, axis * r + r // 2 + i
            m[:, a, a], m[:, a, b] = np.cos(t), -np.sin(t)
            m[:, b, a], m[:, b, b] = np.sin(t), np.cos(t)
    return torch.from_numpy(m).to(DEV)


def _exact_qk(case, s):
    n, heads, kv, hd = case["n"], case["heads"], case["kv"], case["hd"]
    turn = _rotation(case)
    x = s["qkv"].double()
    out = {}
    for name, gain, first, many in (("q", "gq", 0, heads), ("k", "gk", heads, kv)):
        # [v][hd][n * many]: a head's vector is a column
        t = x[:, first * hd:(first + many) * hd].reshape(n * many, hd, -1).permute(2, 1, 0)
        g = s[gain].double()[None, :, None]
        size = ((t ** 2).sum(1, keepdim=True) / hd + EPS).sqrt()
        if case["op"] == "qk":
            y = torch.bmm(turn, (t / size * g).contiguous())
            out[name] = y.permute(2, 1, 0).reshape(n, many * hd, -1)
            continue
        dy = s["d" + name].double().reshape(n * many, hd, -1).permute(2, 1, 0).contiguous()
        dz = torch.bmm(turn.transpose(1, 2).contiguous(), dy)
        unit = t / size
        out["d" + gain] = (dz * unit).sum((0, 2))
        dx = (dz * g - unit * (dz * g * unit).sum(1, keepdim=True) / hd) / size
        out["d" + name] = dx.permute(2, 1, 0).reshape(n, many * hd, -1)
    return {k: out[k] for k in (("q", "k") if case["op"] == "qk" else ("dq", "dk", "dgq", "dgk"))}


def _exact_attn(case, s):
    n, heads, kv, hd = case["n"], case["heads"], case["kv"], case["hd"]
    train, scale = case["op"] == "attn_train", 1.0 / math.sqrt(hd)
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    out = dict(o=o)
    if train:
        out.update(dq=torch.zeros_like(o),
                   dk=torch.zeros(s["k"].shape, dtype=torch.float64, device=DEV),
                   dv=torch.zeros(s["v"].shape, dtype=torch.float64, device=DEV))
    for b in range(n):
        live = (torch.nonzero(s["mask"][b]).flatten() if s["mask"] is not None else
                torch.arange(s["k"].shape[2], device=DEV))
        if live.numel() == 0:
            continue
        for h in range(heads):
            mine = slice(h * hd, (h + 1) * hd)
            its = slice(h // (heads // kv) * hd, (h // (heads // kv) + 1) * hd)
            q = s["q"][b, mine].double().t().contiguous()  # [tq][hd]
            k = s["k"][b, its].double()[:, live].t().contiguous()
            v = s["v"][b, its].double()[:, live].t().contiguous()
            p = torch.softmax(torch.mm(q, k.t().contiguous()) * scale, dim=1)
            o[b, mine] = torch.mm(p, v).t()
            if not train:
                continue
            do = s["do"][b, mine].double().t().contiguous()
            dp = torch.mm(do, v.t().contiguous())
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            out["dq"][b, mine] = (torch.mm(ds, k) * scale).t()
            out["dk"][b, its].index_add_(1, live, (torch.mm(ds.t().contiguous(), q) * scale).t())
            out["dv"][b, its].index_add_(1, live, torch.mm(p.t().contiguous(), do).t())
    return out


def _exact_dropout(case, s):
    unit = _unit(case)
    units = s["x"].numel() // unit
    # the generator again, in unsigned 64-bit words of numpy
    u = np.uint64
    low = u(0xffffffff)
    i = np.arange((units + 7) // 8, dtype=u)
    ctr = [i & low, i >> u(32), np.full_like(i, s["step"] & 0xffffffff),
           np.full_like(i, s["step"] >> 32)]
    key = [s["seed"] & 0xffffffff, s["seed"] >> 32]
    for _ in range(10):
        a, b = u(0xD2511F53) * ctr[0], u(0xCD9E8D57) * ctr[2]
        ctr = [(b >> u(32)) ^ ctr[1] ^ u(key[0]), b & low, (a >> u(32)) ^ ctr[3] ^ u(key[1]),
               a & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    lots = np.empty((i.size, 8), dtype=np.int32)
    for j in range(4):
        lots[:, 2 * j], lots[:, 2 * j + 1] = ctr[j] & u(0xffff), ctr[j] >> u(16)
    at = round(case["p"] * 65536)
    keep = torch.from_numpy(lots.reshape(-1)[:units] >= at).to(DEV).double()
    keep = (keep / (1.0 - at / 65536.0))[:, None].expand(units, unit).reshape(s["x"].shape)
    y = s["x"].double() * keep
    if s["residual"] is not None:
        y += s["residual"].double()
    return dict(y=y, dx=s["dy"].double() * keep)


def exact(case, seed):
    """The outputs of `run` from the operators' definitions in 64 bits."""
    s = _inputs(case, seed)
    if case["op"] == "dropout":
        return _exact_dropout(case, s)
    if case["op"] in ("qk", "qk_grad"):
        # the rotation as a matrix for each voxel
        if float(case["d"] * case["h"] * case["w"]) * case["hd"] ** 2 > 1.5e9:
            return None
        return _exact_qk(case, s)
    return _exact_attn(case, s)
