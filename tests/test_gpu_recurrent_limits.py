"""What the recurrent block's calls promise at their limits: long sums of gains, values near
the largest float, gains, states and gradients that are not finite beside masked voxels, the
longest rows."""
import itertools

import numpy as np
import pytest

from tests import gpu_util as U
from tests import recurrent_util as RU
from tests import test_gpu_block_norm as TN
from tests import test_gpu_recurrence as TR
from tests.test_gpu_any import _tags
from tests.test_gpu_block_norm import _ws
from tests.test_gpu_recurrent_kernels import _cus

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


# ------------------------------------------------------------------ sums of gains
# A gain's gradient over equal terms du x r = 2^-1/2 is the number of voxels times that.  The
# root is off by 3 f (the mean's quotient and sum rounded, halved; one unit of the root), a
# thread's up to eight terms by 7 f, the result by f; everything between is float64.
EQUAL = 16 * RU.F


def _equal_gains(R, n, c, v, dt):
    """Gains' gradients before and behind a block where every term is the same, and the names
    of the kernels; the results lie over the inputs."""
    torch = U.torch_mod()
    x = torch.ones((n, c, v), dtype=U.tdtype(dt), device="cuda:0")
    du = torch.ones_like(x)
    one = torch.ones(c, device="cuda:0")
    pre, post = torch.empty(c, device="cuda:0"), torch.empty(c, device="cuda:0")
    d = R.norm_desc(n, c, v, U.code(dt), eps=1.0)
    need = R.rat3d_norm_workspace_size(d)
    ws, buf = U.guarded((need,), torch.uint8)
    tags = _tags(lambda: (
        R.rat3d_post_norm_bwd(d, du, None, None, x, None, one, None, None, None, None, x, None,
                              post, None, None, 0, ws, need),
        x.fill_(1.0),
        R.rat3d_pre_norm_bwd(d, du, x, one, None, None, x, pre, 0, ws, need)))
    U.guard_intact(buf, "workspace")
    # dx = r - r^3 = r / 2
    far = float(x[:, :: max(1, c // 3)].float().sub_(0.5 ** 1.5).abs_().max())
    assert far <= EQUAL + RU.U[dt], far
    return tags, U.f64(pre), U.f64(post)


@pytest.mark.parametrize("c,v,dt,tag", [(300, 1, "f32", "_one"), (513, 4, "f32", "_any"),
                                        (520, 8, "bf16", "_any")])
def test_gains_of_channels_read_again(c, v, dt, tag):
    """More channels than threads hold, 862 tiles a workgroup: a float32 sum of them would
    drift by 190 f."""
    from paper_2104_05035_amd import rat3d as R
    n = 862 * 2 * _cus()
    tags, *got = _equal_gains(R, n, c, v, dt)
    assert {"pre_norm_bwd" + tag, "post_norm_bwd" + tag} <= set(tags)
    for g in got:
        np.testing.assert_allclose(g, n * v * 0.5 ** 0.5, rtol=EQUAL)


def test_gains_of_rows_beyond_2_27_voxels():
    """Float32 rows of which 32 bits reach seven: four groups of threads, eight workgroups a
    CU, 1024 tiles each."""
    from paper_2104_05035_amd import rat3d as R
    v = (1 << 27) + 131
    tags, *got = _equal_gains(R, 1, 17, v, "f32")
    assert {"pre_norm_bwd_any", "post_norm_bwd_any"} <= set(tags)
    for g in got:
        np.testing.assert_allclose(g, v * 0.5 ** 0.5, rtol=EQUAL)


# ------------------------------------------------------------------ values far out
# channels and voxels of kernels that hold whole and other tiles, and that read again
SHAPES = [(16, 3), (24, 37), (64, 128), (200, 65), (300, 65), (384, 64), (600, 33), (640, 64)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c,v", SHAPES)
@pytest.mark.parametrize("kind,nxt", [("silu", True), (None, True), ("sigmoid", False)])
def test_squares_beyond_the_largest_float(c, v, dt, kind, nxt):
    """Voxels whose sum of squares is infinite have N = 0, though their values times gains and
    gate are no float any more: as masked ones they change nothing but themselves."""
    s = TN.Norms((2, c, v, kind, nxt, None), dt)
    R, r, torch = s.R, s.ref, U.torch_mod()
    rng = np.random.default_rng(c + v)
    big = rng.random((2, v)) < 0.4
    big[0, 0] = True
    for name in ("x", "z"):  # in every channel, or in one of them
        some = rng.random((2, c, v)) < 0.5
        some[:, rng.integers(c)] = True
        far = rng.choice([-3e38, 3e38, 2.5e38], (2, c, v)) * (some | (rng.random((2, 1, v)) < 0.5))
        t, f = U.dev_input(np.where(big[:, None, :], far, r[name]), dt)
        setattr(s, name, t)
        r[name] = f
    s.g[torch.from_numpy(big).to("cuda:0")[:, None, :].expand(s.g.shape)] = 4.0
    s.gamma *= 3
    r["gamma"] = U.f64(s.gamma)
    live = (~big).astype(np.uint8)
    g, gn = s.g if kind else None, s.gnext if nxt else None
    y, u, dx, dz, dg, pre, pdx = (s.out() for _ in range(7))
    v0, v1, v2, v3 = (s.out((c,), "f32") for _ in range(4))
    R.rat3d_post_norm_fwd(s.desc, s.x, s.z, g, s.gamma, s.scale, gn, None, y, u if nxt else None)
    R.rat3d_post_norm_bwd(s.desc, s.dy, s.du if nxt else None, s.x if nxt else None, s.z, g, s.gamma,
                          s.scale, gn, None, dx if nxt else None, dz, dg if kind else None, v0, v1,
                          v2 if nxt else None, 0, _ws(s.need), s.need)
    R.rat3d_pre_norm_fwd(s.desc, s.x, s.gamma, None, pre)
    R.rat3d_pre_norm_bwd(s.desc, s.du, s.x, s.gamma, None, s.dres, pdx, v3, 0, _ws(s.need), s.need)
    U.sync()
    gnr = r["gnext"] if nxt else None
    want = RU.post_norm_refs(r["x"], r["z"], r["g"], kind, r["gamma"], r["scale"], gnr, live, TN.EPS,
                             dt)
    want.update(RU.post_norm_bwd_refs(r["dy"], r["du"], r["x"], r["z"], r["g"], kind, r["gamma"],
                                      r["scale"], gnr, live, TN.EPS, dt))
    if not nxt:
        del want["dx"]
    p = RU.pre_norm_refs(r["x"], r["gamma"], live, TN.EPS, dt, r["du"], r["dres"])
    want.update(pre=p["u"], pdx=p["dx"], v3=p["dgamma"])
    got = dict(y=y, u=u, dx=dx, dz=dz, dg=dg, dgamma=v0, dscale=v1, dgamma_next=v2, pre=pre, pdx=pdx,
               v3=v3)
    for k in want:
        RU.within(U.f64(got[k]), want[k], k)
    s.intact()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c,v", SHAPES)
def test_infinite_values_are_not_hidden(c, v, dt):
    """An infinity is NaN in its own channel; the voxel's other channels have N = 0."""
    s = TN.Norms((1, c, v, "silu", True, None), dt)
    R, torch = s.R, U.torch_mod()
    ch, at = c // 2, v // 2
    s.z[0, ch, at] = INF
    s.g[0, ch, at] = 1.0
    y, u, dz, dx, dg, pre = (s.out() for _ in range(6))
    vec = [s.out((c,), "f32") for _ in range(3)]
    R.rat3d_pre_norm_fwd(s.desc, s.z, s.gamma, None, pre)
    R.rat3d_post_norm_fwd(s.desc, s.x, s.z, s.g, s.gamma, s.scale, None, None, y, None)
    R.rat3d_post_norm_bwd(s.desc, s.dy, s.du, s.x, s.z, s.g, s.gamma, s.scale, s.gnext, None, dx, dz,
                          dg, *vec, 0, _ws(s.need), s.need)
    U.sync()
    rest = torch.arange(c, device="cuda:0") != ch
    for t in (y, dz, pre):
        assert bool(torch.isnan(t[0, ch, at]))
        assert int(torch.isnan(t).sum()) == 1
    assert torch.equal(y[0, rest, at], s.x[0, rest, at])
    assert bool((dz[0, rest, at] == 0).all()) and bool((pre[0, rest, at] == 0).all())
    assert bool(torch.isfinite(dx).all())
    s.intact()


# ------------------------------------------------------------------ beside masked voxels
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c,v", SHAPES)
@pytest.mark.parametrize("kind,nxt", [("silu", True), (None, True), ("sigmoid", False)])
def test_masked_voxels_whatever_the_gains(c, v, dt, kind, nxt):
    """u = 0, y = x, dx = dres or dy, dz = dg = 0 at masked voxels, also where a gain is
    infinite or no number."""
    s = TN.Norms((3, c, v, kind, nxt, "holes"), dt)
    R, torch = s.R, U.torch_mod()
    off = torch.from_numpy(s.mask == 0).to("cuda:0")[:, None, :].expand(s.x.shape)
    g = s.g if kind else None
    for bad in (INF, NAN):
        for name in ("gamma", "scale", "gnext"):
            kept = getattr(s, name).clone()
            getattr(s, name)[:: max(1, c // 3)] = bad
            gn = s.gnext if nxt else None
            y, u, dx, dz, dg, pre, pdx, pdx0 = (s.out() for _ in range(8))
            vec = [s.out((c,), "f32") for _ in range(4)]
            R.rat3d_post_norm_fwd(s.desc, s.x, s.z, g, s.gamma, s.scale, gn, s.dmask, y,
                                  u if nxt else None)
            R.rat3d_post_norm_bwd(s.desc, s.dy, s.du if nxt else None, s.x if nxt else None, s.z, g,
                                  s.gamma, s.scale, gn, s.dmask, dx if nxt else None, dz,
                                  dg if kind else None, vec[0], vec[1], vec[2] if nxt else None, 0,
                                  _ws(s.need), s.need)
            R.rat3d_pre_norm_fwd(s.desc, s.x, s.gamma, s.dmask, pre)
            for res, to in ((s.dres, pdx), (None, pdx0)):
                R.rat3d_pre_norm_bwd(s.desc, s.du, s.x, s.gamma, s.dmask, res, to, vec[3], 0,
                                     _ws(s.need), s.need)
            U.sync()
            zero = torch.zeros_like(s.x)
            want = dict(y=(y, s.x), dz=(dz, zero), pre=(pre, zero), pdx=(pdx, s.dres),
                        pdx0=(pdx0, zero))
            if nxt:
                want.update(u=(u, zero), dx=(dx, s.dy))
            if kind:
                want["dg"] = (dg, zero)
            for k, (got, w) in want.items():
                assert bool((got[off] == w[off]).all()), (name, bad, k)
            getattr(s, name).copy_(kept)
    s.intact()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c,v", [(3, 5), (6, 37), (4, 700), (300, 1100), (2, 9003), (1, 70000)])
@pytest.mark.parametrize("reverse", [False, True])
def test_masked_rows_give_lambda_nothing(c, v, reverse, dt):
    """A volume that is masked as a whole hands its states on whatever they are, and has no
    part in lambda's gradient."""
    torch = U.torch_mod()
    s = TR.Walk((3, c, v, reverse, "holes", 1.0, 8.0), dt)
    assert not s.mask[1].any()
    want, got = s.results(), s.results()
    s.fwd(want)
    s.bwd(want)
    s.h0[1], s.dh[1] = INF, NAN
    s.fwd(got)
    s.bwd(got)
    U.sync()
    assert bool((got["h_last"][1] == INF).all()) and bool(torch.isnan(got["dh0"][1]).all())
    got["h_last"][1], got["dh0"][1] = want["h_last"][1], want["dh0"][1]
    for k in want:
        assert torch.equal(got[k], want[k]), k
    for b in s.guards:
        U.guard_intact(b)


# ------------------------------------------------------------------ results over inputs
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c,v,mask", [(40, 203, "holes"), (64, 128, None), (300, 67, None),
                                      (600, 203, "holes"), (640, 64, None), (270, 3, "holes")])
def test_every_result_over_every_input(c, v, mask, dt):
    """Each choice of inputs that results may lie over: the bits of tensors of their own."""
    s = TN.Norms((2, c, v, "silu", True, mask), dt)
    R, torch = s.R, U.torch_mod()
    same = lambda a, b: torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))  # noqa: E731
    vec = [torch.empty(c, device="cuda:0") for _ in range(4)]
    ws = _ws(s.need)

    def forward(t, y, u):
        R.rat3d_post_norm_fwd(s.desc, t["x"], t["z"], t["g"], s.gamma, s.scale, s.gnext, s.dmask, y, u)
        return y, u

    def behind(t, dx, dz, dg):
        R.rat3d_post_norm_bwd(s.desc, t["dy"], t["du"], t["x"], t["z"], t["g"], s.gamma, s.scale,
                              s.gnext, s.dmask, dx, dz, dg, *vec[:3], 0, ws, s.need)
        return dx, dz, dg

    def before(t, dx):
        R.rat3d_pre_norm_bwd(s.desc, t["du"], t["x"], s.gamma, s.dmask, t["dres"], dx, vec[3], 0, ws,
                             s.need)
        return (dx,)

    for call, names, results in ((forward, ("x", "z", "g"), 2),
                                 (behind, ("dy", "du", "x", "z", "g"), 3),
                                 (before, ("du", "x", "dres"), 1)):
        src = {k: getattr(s, k) for k in names}
        own = call(src, *(torch.empty_like(s.x) for _ in range(results)))
        for over in itertools.permutations(names, results):
            t = {k: a.clone() for k, a in src.items()}
            for a, b in zip(own, call(t, *(t[k] for k in over))):
                assert same(a, b), (call.__name__, over)


# ------------------------------------------------------------------ the longest rows
@pytest.mark.parametrize("c,tag", [(6, ""), (17, "_any")])
def test_float32_rows_of_2_28_voxels(c, tag):
    """Rows of which 32 bits reach four: every piece of 4096 voxels has the bits of the first,
    and these are right."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    v = 1 << 28
    g = torch.Generator(device="cuda:0").manual_seed(4)
    small = torch.randn((c, 4096), generator=g, device="cuda:0")
    x = torch.empty((c, v), device="cuda:0")
    x.view(c, -1, 4096).copy_(small[:, None, :])
    gamma = 1 + 0.1 * torch.arange(c, device="cuda:0", dtype=torch.float32)
    d = R.norm_desc(1, c, v, R.F32, eps=1e-5)
    tags = _tags(lambda: R.rat3d_pre_norm_fwd(d, x, gamma, None, x))
    assert tags == ["pre_norm_fwd" + tag]
    want = RU.pre_norm_refs(U.f64(small)[None], U.f64(gamma), None, 1e-5, "f32")["u"]
    RU.within(U.f64(x[:, :4096])[None], want, "u")
    for k in range(c):
        row = x[k].view(-1, 4096)
        assert bool((row == row[:1]).all()), k


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("reverse", [False, True])
def test_joined_segments_of_several_masked_rows(reverse, dt):
    """Rows of more segments than find one another, with masks, states and results in place:
    the bits of each row alone, and a row's values in pieces."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    block = 8 * (512 if dt == "bf16" else 256)
    n, c, v = 2, 2, 2048 * block + 5
    g = torch.Generator(device="cuda:0").manual_seed(19)
    ins = [torch.randn((n, c, v), generator=g, device="cuda:0").to(U.tdtype(dt)) for _ in range(4)]
    mask = (torch.rand((n, v), generator=g, device="cuda:0") < 0.6).to(torch.uint8)
    mask[1, v // 3:v // 2] = 0  # whole segments
    lam = torch.tensor([-9.0, -3.0], device="cuda:0")
    h0 = torch.randn((n, c), generator=g, device="cuda:0")
    dh = torch.randn((n, c), generator=g, device="cuda:0")

    def run(r, i, x, dy, mask, lam, h0, dh):
        m, k, t = r.shape
        d = R.recurrence_desc(m, k, t, U.code(dt), reverse=reverse)
        need = [R.rat3d_recurrence_workspace_size(d, p) for p in (0, 1)]
        carry = _ws(R.rat3d_recurrence_carry_size(d))
        y, dlam = torch.empty_like(r), torch.empty_like(lam)
        r, i, x, last, first = r.clone(), i.clone(), x.clone(), h0.clone(), dh.clone()
        R.rat3d_recurrence_fwd(d, r, i, x, lam, mask, last, y, last, carry, _ws(need[0]), need[0])
        R.rat3d_recurrence_bwd(d, dy, first, r, i, x, lam, mask, carry, r, i, x, dlam, first, 0,
                               _ws(need[1]), need[1])
        U.sync()
        return dict(y=y, h_last=last, dr=r, di=i, dx=x, dh0=first, dlam=dlam)

    tags = []
    tags.append(_tags(lambda: tags.append(run(*ins, mask, lam, h0, dh))))
    whole, tags = tags
    assert {"recurrence_fwd_join", "recurrence_bwd_join"} <= set(tags)
    total, size = torch.zeros((2, c), dtype=torch.float64, device="cuda:0")
    for j in range(n):
        for k in range(c):
            o = run(*(t[j:j + 1, k:k + 1].contiguous() for t in ins), mask[j:j + 1], lam[k:k + 1],
                    h0[j:j + 1, k:k + 1].contiguous(), dh[j:j + 1, k:k + 1].contiguous())
            total[k] += o["dlam"][0].double()
            size[k] += o["dlam"][0].double().abs()
            for name in o:
                if name != "dlam":
                    assert torch.equal(o[name][0, 0], whole[name][j, k]), (name, j, k)
    # each row's sum is rounded once, and that of both
    assert bool(((whole["dlam"].double() - total).abs() <= 2 * RU.F * size).all())
    # the second volume with the short memory in pieces: a segment's edges lie inside them
    r, i, x, dy = (t[1:, 1:] for t in ins)
    size = -(-v // 7)
    cuts = [(a, min(a + size, v)) for a in range(0, v, size)][::-1 if reverse else 1]
    state = h0[1:, 1:].contiguous()
    for a, b in cuts:
        o = run(*(t[..., a:b].contiguous() for t in (r, i, x, dy)), mask[1:, a:b].contiguous(), lam[1:],
                state, torch.zeros_like(state))
        state = o["h_last"]
        got, want = whole["y"][1:, 1:, a:b].float(), o["y"].float()
        # decays of 0.68 at the mean: a state's error is that of some hundred steps, 64 f each,
        # of values up to 8, and both are rounded
        assert bool(((got - want).abs() <= 2 * RU.U[dt] * want.abs() + 8 * 64 * 100 * RU.F).all())


# ------------------------------------------------------------------ streams
def test_walks_on_two_streams():
    """Forward and backward on two streams at once, everything allocated and filled before: the
    bits of one after another, and nothing beside the results."""
    torch = U.torch_mod()
    s = [TR.Walk((1, 4, 50000, False, None, 1.0, 8.0), "bf16"),
         TR.Walk((2, 3, 60001, True, "holes", 1.0, 8.0), "bf16")]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]

    def run(walks):
        out = [(t, t.results(), [_ws(b) for b in t.need], st) for t, st in walks]
        U.sync()  # the fills are on the current stream
        for t, o, ws, st in out:
            p = st.cuda_stream
            t.R.rat3d_recurrence_fwd(t.desc, t.r, t.i, t.x, t.lam, t.dmask, t.h0, o["y"], o["h_last"],
                                     t.carry, ws[0], t.need[0], stream=p)
            t.R.rat3d_recurrence_bwd(t.desc, t.dy, t.dh, t.r, t.i, t.x, t.lam, t.dmask, t.carry,
                                     o["dr"], o["di"], o["dx"], o["dlam"], o["dh0"], 0, ws[1],
                                     t.need[1], stream=p)
        U.sync()
        return [o for _, o, _, _ in out]

    alone = [run([w])[0] for w in zip(s, streams)]
    for _ in range(3):
        for o, a in zip(run(list(zip(s, streams))), alone):
            assert all(torch.equal(o[k], a[k]) for k in a)
    for t in s:
        for b in t.guards:
            U.guard_intact(b)
