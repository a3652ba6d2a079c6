"""What the recurrent block's calls promise at their limits: long sums of gains, values near
the largest float, gains, states and gradients that are not finite beside masked voxels, the
longest rows."""
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
