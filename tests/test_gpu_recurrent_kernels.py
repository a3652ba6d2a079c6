"""Which kernels of the recurrent block run, by their measurement names, and what only
large calls reach: results past the memory-side cache, offsets beyond 32 bits, rows of
more segments than find one another, long sums."""
import numpy as np
import pytest

from tests import gpu_util as U
from tests import recurrent_util as RU
from tests import test_gpu_block_norm as TN
from tests import test_gpu_recurrence as TR
from tests.test_gpu_any import _tags
from tests.test_gpu_block_norm import _rng, _ws

pytestmark = pytest.mark.gpu


def _cus():
    return U.torch_mod().cuda.get_device_properties(0).multi_processor_count


# ------------------------------------------------------------------ norms
# tokens, channels, volumes, and the names' ends in bfloat16 and float32: forward, gradient
# before a block, behind one with and without a next norm (a pair: without and with a mask)
ONE, HALF, QUARTER, ANY, FULL = (("_one",) * 4, ("_half",) * 4, ("_half",) + ("_quarter",) * 3,
                                 ("_any",) * 4, ("",) * 4)
REST = ("_half",) + ("_any",) * 3
NORMS = [
    (7, 40, "few", ONE, HALF), (3, 300, "few", ONE, ONE), (130, 24, "few", HALF, HALF),
    (90, 128, "many", FULL, FULL), (33, 100, "many", FULL, FULL), (33, 100, "few", HALF, HALF),
    (256, 64, "few", HALF, HALF), (128, 128, "few", HALF, HALF), (70, 256, "few", QUARTER, HALF),
    (64, 256, "few", QUARTER, HALF), (40, 160, "many", ("",) + ("_half",) * 3, ("", "", "_half", "")),
    (64, 256, "some", HALF, ("", "", ("", "_half"), "")),
    (64, 200, "some", HALF, ("", "", "_half", "")), (50, 257, "few", QUARTER, QUARTER),
    (128, 512, "few", QUARTER, QUARTER), (128, 384, "some", REST, REST),
    (64, 270, "some", REST, REST), (129, 300, "some", QUARTER, QUARTER),
    (129, 513, "few", ANY, ANY), (128, 640, "few", ANY, ANY)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", NORMS, ids=lambda c: "v%d_c%d_%s" % c[:3])
def test_norm_kernels(case, dt):
    v, c, volumes, *ends = case
    # of 16 bytes of tokens a thread: tiles more than two a CU, or one for two CUs
    n = dict(few=2, some=_cus() // 2 + 12, many=-(-int(2.1 * _cus()) // -(-v // 128)))[volumes]
    ends = [e if isinstance(e, tuple) else (e, e) for e in ends[dt == "f32"]]
    for k, mask in enumerate((None, "holes")):
        fwd, pre, nxt, last = (e[k] for e in ends)
        for kind, is_next, post in (("silu", True, nxt), (None, False, last)):
            tags = _tags(lambda: TN.test_post_norm((n, c, v, kind, is_next, mask), dt))
            assert set(tags) == {"post_norm_fwd" + fwd, "post_norm_bwd" + post, "norm_gain"}
        tags = _tags(lambda: TN.test_pre_norm((n, c, v, None, False, mask), dt))
        assert set(tags) == {"pre_norm_fwd" + fwd, "pre_norm_bwd" + pre, "norm_gain"}


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_results_past_the_cache(dt):
    """Results of more than 256 MB: the bits of the same voxels in smaller calls."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    c, part, parts = 32, 128 * 1100, 32 if dt == "bf16" else 16
    v = part * parts
    g = torch.Generator(device="cuda:0").manual_seed(5)
    rnd = lambda: torch.randn((1, c, v), generator=g, device="cuda:0").to(U.tdtype(dt))  # noqa: E731
    x, z, gt, dy, du = (rnd() for _ in range(5))
    vec = [1 + 0.3 * torch.randn(c, generator=g, device="cuda:0") for _ in range(3)]
    E = lambda t: torch.empty_like(t)  # noqa: E731

    def run(x, z, gt, dy, du):
        d = R.norm_desc(1, c, x.shape[2], U.code(dt), gate=R.GATE_SILU)
        need = R.rat3d_norm_workspace_size(d)
        y, u, dx, dz, dg, pu, pdx = (E(x) for _ in range(7))
        dv = [torch.empty(c, device="cuda:0") for _ in range(4)]
        R.rat3d_post_norm_fwd(d, x, z, gt, *vec, None, y, u)
        R.rat3d_post_norm_bwd(d, dy, du, x, z, gt, *vec, None, dx, dz, dg, *dv[:3], 0, _ws(need),
                              need)
        R.rat3d_pre_norm_fwd(d, x, vec[0], None, pu)
        R.rat3d_pre_norm_bwd(d, du, x, vec[0], None, dy, pdx, dv[3], 0, _ws(need), need)
        U.sync()
        return [y, u, dx, dz, dg, pu, pdx], torch.stack(dv).double()

    assert x.numel() * x.element_size() > 256e6
    whole, dv = run(x, z, gt, dy, du)
    total = torch.zeros_like(dv)
    for k in range(parts):
        cut = lambda t: t[..., k * part:(k + 1) * part].contiguous()  # noqa: E731
        small, d = run(*(cut(t) for t in (x, z, gt, dy, du)))
        total += d
        assert all(torch.equal(cut(a), b) for a, b in zip(whole, small))
    # 32 values of float32, of sums of random signs: sqrt(v) each, a float32 rounding of it
    # apart, and of each thread's sums
    assert float((dv - total).abs().max()) <= 64 * 2.0 ** -24 * float(v) ** 0.5 * 40


def test_norm_gain_of_many_voxels():
    """Equal terms of 2^27 voxels: the sum does not drift; offsets in a row beyond 32 bits
    of bytes."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    v = 1 << 27
    x = torch.ones((1, 1, v), device="cuda:0")
    gamma, dg, dx = torch.ones(1, device="cuda:0"), torch.empty(1, device="cuda:0"), torch.empty_like(x)
    d = R.norm_desc(1, 1, v, R.F32, eps=1.0)
    need = R.rat3d_norm_workspace_size(d)
    R.rat3d_pre_norm_bwd(d, x, x, gamma, None, None, dx, dg, 0, _ws(need), need)
    U.sync()
    # r once rounded in the root, the product, a thread's tokens and the tree
    assert float(dg[0]) == pytest.approx(v / 2.0 ** 0.5, rel=16 * 2.0 ** -24)
    # dx = r - r^3 = r / 2
    assert bool((dx - 0.5 / 2.0 ** 0.5).abs().max() <= 16 * 2.0 ** -24)


def test_norm_rows_of_2_28_voxels():
    """The longest rows: a group's rows are 2^32 bytes apart at most."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    c, v = 16, 1 << 28
    x = torch.empty((c, v), dtype=torch.bfloat16, device="cuda:0")
    g = torch.Generator(device="cuda:0").manual_seed(3)
    small = torch.randn((c, 4096), generator=g, device="cuda:0").to(torch.bfloat16)
    x.view(c, -1, 4096).copy_(small[:, None, :])
    gamma = torch.ones(c, device="cuda:0")
    d = R.norm_desc(1, c, v, R.BF16, eps=1e-5)
    R.rat3d_pre_norm_fwd(d, x, gamma, None, x)
    want = torch.empty_like(small)
    R.rat3d_pre_norm_fwd(R.norm_desc(1, c, 4096, R.BF16, eps=1e-5), small, gamma, None, want)
    U.sync()
    RU.within(U.f64(want)[None], RU.pre_norm_refs(U.f64(small)[None], np.ones(c), None, 1e-5, "bf16")["u"],
              "u")
    # the same voxels in every piece, as far as the kernels sum in one order
    for k in (0, 1, v // 8192, v // 4096 - 1):
        assert bool((x.view(c, -1, 4096)[:, k].float() - want.float()).abs().max() <=
                    2.0 ** -7 * want.float().abs().max())


def test_norm_of_more_workgroups_than_a_launch_holds():
    """2^26 volumes of one voxel: more than 2^32 threads, so more than one launch."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n = (1 << 26) + 77
    x = torch.arange(n, device="cuda:0").remainder_(5).sub_(2).float().view(n, 1, 1)
    u = torch.full_like(x, 9.0)
    R.rat3d_pre_norm_fwd(R.norm_desc(n, 1, 1, R.F32, eps=2.0 ** -100), x, torch.ones(1, device="cuda:0"),
                         None, u)
    U.sync()
    # x / |x|: the root of a square is exact to a unit
    assert bool(((u - x.sign()).abs() <= 4 * 2.0 ** -24).all())


# ------------------------------------------------------------------ recurrence
# rows (0: more than a CU each), tokens of bfloat16, the name's end
WALKS = [(3, 100, "recurrence_short_"), (5, 128, "recurrence_short_"), (5, 129, "recurrence_"),
         (3, 4097, "recurrence_"), (3, 8192, "recurrence_"), (3, 8193, "recurrence_one"), (2, 41000, "recurrence_one"),
         (0, 9001, "recurrence_")]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,v,name", WALKS)
def test_recurrence_kernels(rows, v, name, dt):
    v = v if dt == "bf16" else -(-v // 2)
    c = rows or int(1.6 * _cus())
    for reverse, mask in ((False, None), (True, "holes")):
        tags = _tags(lambda: TR.test_recurrence((1, c, v, reverse, mask, 1.0, 8.0), dt))
        want = {"recurrence_lambda"}
        if name == "recurrence_one":
            want |= {"recurrence_begin", "recurrence_fwd_one", "recurrence_bwd_one"}
        else:
            want |= {name + "fwd", name + "bwd"}
        assert set(tags) == want


@pytest.mark.parametrize("dt,v", [("bf16", 33000), ("f32", 16500)])
def test_one_row_a_cu(dt, v):
    """Sixteen waves a workgroup."""
    c = _cus() + 2
    TR.test_recurrence((1, c, v, False, None, 1.0, 8.0), dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("reverse", [False, True])
def test_more_segments_than_find_one_another(reverse, dt):
    """A launch of its own joins them: against the same row in pieces, one state handed to
    the next."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    block = 8 * (512 if dt == "bf16" else 256)
    v = 2048 * block + 5
    g = torch.Generator(device="cuda:0").manual_seed(9)
    r, i, x, dy = (torch.randn((1, 1, v), generator=g, device="cuda:0").to(U.tdtype(dt))
                   for _ in range(4))
    lam = torch.full((1,), -9.0, device="cuda:0")  # decays of 0.9995: a long memory
    h0, dh = torch.full((1, 1), 3.0, device="cuda:0"), torch.full((1, 1), -2.0, device="cuda:0")

    def run(first, last, h0, dh, need_carry=True):
        cut = lambda t: t[..., first:last].contiguous()  # noqa: E731
        ins = [cut(t) for t in (r, i, x, dy)]
        d = R.recurrence_desc(1, 1, last - first, U.code(dt), reverse=reverse)
        need = [R.rat3d_recurrence_workspace_size(d, p) for p in (0, 1)]
        carry = _ws(R.rat3d_recurrence_carry_size(d))
        o = dict(y=torch.empty_like(ins[0]), h_last=torch.empty_like(h0), dlam=torch.empty_like(lam),
                 dh0=torch.empty_like(h0), **{k: torch.empty_like(ins[0]) for k in ("dr", "di", "dx")})
        fwd = lambda h0: R.rat3d_recurrence_fwd(d, *ins[:3], lam, None, h0, o["y"], o["h_last"],  # noqa: E731
                                                carry, _ws(need[0]), need[0])
        bwd = lambda dh: R.rat3d_recurrence_bwd(d, ins[3], dh, *ins[:3], lam, None, carry, o["dr"],  # noqa: E731
                                                o["di"], o["dx"], o["dlam"], o["dh0"], 0,
                                                _ws(need[1]), need[1])
        fwd(h0)
        return o, bwd

    out = {}
    tags = _tags(lambda: out.update(zip(("o", "bwd"), run(0, v, h0, dh))) or out["bwd"](dh))
    assert set(tags) == {"recurrence_fwd_join", "recurrence_fwd_cut", "recurrence_bwd_join",
                         "recurrence_bwd_cut", "recurrence_lambda"}
    U.sync()
    whole = out["o"]
    size = -(-v // 5)
    cuts = [(k, min(k + size, v)) for k in range(0, v, size)]
    cuts = cuts[::-1] if reverse else cuts
    state, parts = h0, []
    for a, b in cuts:
        parts.append(run(a, b, state, None))
        state = parts[-1][0]["h_last"]
    grad = dh
    for o, bwd in reversed(parts):
        bwd(grad)
        grad = o["dh0"]
    U.sync()
    # Both ways stay within the bound of the recurrence; here, with magnitudes near the
    # values' (a sum of some 2000 terms of random signs): 2000 steps' decays off by 4 f each,
    # and the type's rounding twice.
    tol = 2000 * 16 * 2.0 ** -24
    for k in ("y", "dr", "di", "dx"):
        joined = torch.cat([o[k] for o, _ in (parts[::-1] if reverse else parts)], dim=-1).float()
        d = (whole[k].float() - joined).abs()
        assert bool((d <= 2 * RU.U[dt] * joined.abs() + tol * float(joined.abs().max())).all()), k
    assert float((whole["h_last"] - state).abs()) <= tol * 10
    assert float((whole["dh0"] - grad).abs()) <= tol * 10
    total = sum(float(o["dlam"]) for o, _ in parts)
    assert float(whole["dlam"]) == pytest.approx(total, rel=1e-3)


def test_recurrence_results_past_the_cache():
    """Results of more than 256 MB: the bits of the same volumes in smaller calls."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, c, v = 4, 512, 70001
    g = torch.Generator(device="cuda:0").manual_seed(6)
    r, i, x, dy = (torch.randn((n, c, v), generator=g, device="cuda:0").to(torch.bfloat16)
                   for _ in range(4))
    lam = torch.full((c,), -3.0, device="cuda:0")

    def run(sl):
        ins = [t[sl] for t in (r, i, x, dy)]
        m = ins[0].shape[0]
        d = R.recurrence_desc(m, c, v, R.BF16)
        need = [R.rat3d_recurrence_workspace_size(d, p) for p in (0, 1)]
        carry = _ws(R.rat3d_recurrence_carry_size(d))
        o = [torch.empty_like(ins[0]) for _ in range(4)]
        dl = torch.empty(c, device="cuda:0")
        R.rat3d_recurrence_fwd(d, *ins[:3], lam, None, None, o[0], None, carry, _ws(need[0]), need[0])
        R.rat3d_recurrence_bwd(d, ins[3], None, *ins[:3], lam, None, carry, *o[1:], dl, None, 0,
                               _ws(need[1]), need[1])
        U.sync()
        return o

    assert r.numel() * 2 > 256e6
    whole = run(slice(None))
    for k in range(0, n, 2):
        for a, b in zip(whole, run(slice(k, k + 2))):
            assert torch.equal(a[k:k + 2], b)


def test_recurrence_of_2_31_tokens():
    """A row of more than 2^31 tokens: its end against float64, as far as the decay
    remembers."""
    from oracle import recurrent as Q
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    v, tail = (1 << 31) + 1000, 6000
    rng = _rng("long")
    ref = {k: None for k in "rix"}
    dev = {}
    for k in ref:
        end, ref[k] = U.dev_input(rng.standard_normal((1, 1, tail)), "bf16")
        dev[k] = torch.zeros((1, 1, v), dtype=torch.bfloat16, device="cuda:0")
        dev[k][..., v - tail:] = end
    lam = torch.full((1,), -2.0, device="cuda:0")
    d = R.recurrence_desc(1, 1, v, R.BF16)
    need = R.rat3d_recurrence_workspace_size(d, 0)
    y, last = torch.empty_like(dev["r"]), torch.empty((1, 1), device="cuda:0")
    R.rat3d_recurrence_fwd(d, dev["r"], dev["i"], dev["x"], lam, None, None, y, last, None, _ws(need),
                           need)
    U.sync()
    # the state is 0 up to the tail
    want = RU.recurrence_refs(ref["r"], ref["i"], ref["x"], np.full(1, -2.0), None, None, 8.0, False,
                              "bf16")
    RU.within(U.f64(y[..., v - tail:]), want["y"], "y")
    RU.within(U.f64(last), want["h_last"], "h_last")
    assert bool((y[..., :v - tail:4099] == 0).all())
    del Q
