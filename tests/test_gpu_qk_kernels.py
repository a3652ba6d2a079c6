"""Every instance of the head norms' kernel against float64: whole and partial tiles,
with and without a norm, four and eight tokens a thread; results over their inputs,
captured calls."""
import numpy as np
import pytest

from oracle import attention as A
from tests import attn_util as AU
from tests import gpu_util as U
from tests import test_gpu_qk_dropout as TQ
from tests.test_gpu_any import _tags

pytestmark = pytest.mark.gpu


def _volumes(tiles):
    """Volumes whose tiles are 10 % more than the four a CU from which bfloat16 takes
    eight tokens a thread."""
    cus = U.torch_mod().cuda.get_device_properties(0).multi_processor_count
    return -(-int(4.4 * cus) // tiles)


# n (0: enough for eight tokens a thread), heads, kv, hd, grid, rot, norm,
# eight tokens forward, backward (in bfloat16)
WIDE = [(0, 1, 1, hd, (3, 5, 19), rot, norm, hd <= 32 or 64 < hd <= 96, hd <= 64)
        for hd, rot in ((16, (4, 6, 4)), (24, (8, 8, 8)), (32, (10, 10, 10)), (40, (12, 12, 12)),
                        (64, (20, 20, 20)), (80, (0, 26, 26)))
        for norm in (True, False)]
ODD = [(0, 2, 1, 9, (1, 3, 171), (2, 2, 2), True, True, True),  # two whole tiles and a token
       (0, 1, 0, 31, (2, 16, 16), (10, 0, 20), True, True, True),  # no partial tile
       (0, 0, 1, 17, (19, 9, 3), (4, 4, 8), True, True, True)]  # rows shorter than a thread's tokens
# four tokens a thread: the tiles that the others leave out
FOUR = [(3, 2, 1, hd, (3, 5, 19), (2, 4, 2), norm, False, False)
        for hd in (8, 20, 48, 60, 90, 120) for norm in (True, False)]


def _id(c):
    return c if isinstance(c, str) else "n%d_h%d_%d_d%d_%s_%s" % (
        c[0], c[1], c[2], c[3], "x".join(map(str, c[4])), "norm" if c[6] else "turn")


@pytest.mark.parametrize("case,dt", [(c, "bf16") for c in WIDE + ODD + FOUR] +
                         [(c, "f32") for c in FOUR], ids=_id)
def test_kernels(case, dt):
    n, heads, kv, hd, grid, rot, norm, wf, wb = case
    if n == 0:
        n = _volumes(-(-int(np.prod(grid)) // 256))
    tags = _tags(lambda: TQ.test_qk_norm_rope((n, heads, kv, hd, grid, rot, (0, 2, 0), norm), dt))
    eight = dt == "bf16"
    assert {t for t in tags if t.startswith("qk_rope")} == {
        "qk_rope_fwd_8" if wf and eight else "qk_rope_fwd",
        "qk_rope_bwd_8" if wb and eight else "qk_rope_bwd"}


def _setup(dt, n, heads, kv, hd, grid, rot, norm=True):
    from paper_2104_05035_amd import rat3d as R
    v = int(np.prod(grid))
    rng = TQ._rng((dt, n, heads, kv, hd, grid, "kernels"))
    d = dict(v=v)
    for s, many in (("q", heads), ("k", kv)):
        for name, amp in ((s, 2.0), ("d" + s, 1.0)):
            d[name], d[name + "r"] = U.dev_input(rng.standard_normal((n, many * hd, v)) * amp, dt)
        d["g" + s], d["g" + s + "r"] = U.dev_input(1 + 0.3 * rng.standard_normal(hd), "f32")
        d["dg" + s] = U.zeros_f32(hd)
    d["desc"] = R.qk_desc(n, heads, kv, hd, *grid, U.code(dt), rot=rot, eps=1e-5, norm=norm)
    d["table"] = TQ._ws(R.rat3d_rope_table_size(d["desc"]))
    R.rat3d_rope_table(d["desc"], d["table"])
    d["need"] = R.rat3d_qk_norm_rope_workspace_size(d["desc"])
    d["ws"] = TQ._ws(d["need"])
    d["turn"] = A.rotation(hd, grid, rot, (0, 0, 0), 100.0)
    return R, d


def _backward(R, d, dq, dk):
    R.rat3d_qk_norm_rope_bwd(d["desc"], d["dq"], d["dk"], d["q"], d["k"], d["gq"], d["gk"],
                             d["table"], dq, dk, d["dgq"], d["dgk"], 0, d["ws"], d["need"])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("hd", [20, 33, 64, 96, 128])
def test_gradients_over_their_inputs(dt, hd, norm):
    """dq over doq and dk over dok: the same bits as into tensors of their own, and the
    gradients themselves."""
    n, heads, kv, grid, rot = 2, 3, 2, (3, 5, 19), (6, 4, 6)
    R, d = _setup(dt, n, heads, kv, hd, grid, rot, norm)
    torch = U.torch_mod()
    own = [torch.empty_like(d["dq"]), torch.empty_like(d["dk"])]
    _backward(R, d, *own)
    gains = [d["dgq"].clone(), d["dgk"].clone()]
    U.sync()
    _backward(R, d, d["dq"], d["dk"])
    U.sync()
    for s, many, dx, dg in (("q", heads, own[0], gains[0]), ("k", kv, own[1], gains[1])):
        assert torch.equal(d["d" + s], dx)
        want, wdg = TQ._qk_bounds(dt, d[s + "r"], many, d["g" + s + "r"] if norm else None,
                                  d["turn"], 1e-5, d["d" + s + "r"])
        AU.within(U.f64(dx), want, "d" + s)
        if norm:
            assert torch.equal(d["dg" + s], dg)
            AU.within(U.f64(dg), wdg, "dg" + s)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_captured_and_replayed(dt):
    """Forward and backward in a HIP graph, replayed on new inputs, with eager work
    between the replays."""
    n, heads, kv, hd, grid, rot = 2, 3, 2, 40, (3, 5, 19), (12, 12, 12)
    R, d = _setup(dt, n, heads, kv, hd, grid, rot)
    torch = U.torch_mod()
    out = [torch.empty_like(d[s]) for s in ("q", "k", "dq", "dk")]

    def both():
        R.rat3d_qk_norm_rope_fwd(d["desc"], d["q"], d["k"], d["gq"], d["gk"], d["table"], out[0],
                                 out[1])
        _backward(R, d, out[2], out[3])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    U.sync()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for i in range(3):
        g = torch.Generator(device="cuda:0").manual_seed(40 + i)
        for s in ("q", "k", "dq", "dk"):
            d[s].copy_(torch.randn(d[s].shape, generator=g, device="cuda:0"))
        d["ws"].fill_(0xFF)
        U.sync()
        graph.replay()
        U.sync()
        all_ = out + [d["dgq"], d["dgk"]]
        got = [t.clone() for t in all_]
        for t in all_:
            t.fill_(55.0)
        both()
        U.sync()
        assert all(torch.equal(a, b) for a, b in zip(got, all_))
