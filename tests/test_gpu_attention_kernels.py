"""Every instance of the attention's kernels against float64: sizes follow the number of
CUs, and the measurement tags say which kernels ran, so that a changed rule of choice
shows here and does not quietly leave a kernel untested."""
import pytest

from tests import test_gpu_attention as TA
from tests import gpu_util as U
from tests.test_gpu_any import _tags

pytestmark = pytest.mark.gpu


def _volumes(per_cu, each):
    """Volumes of `each` workgroups that are `per_cu` a CU."""
    cus = U.torch_mod().cuda.get_device_properties(0).multi_processor_count
    return -(-int(per_cu * cus) // each)


# per_cu (None: one volume), workgroups a volume that counts for it, then
# heads, kv, hd, tq, tk, mask and the backward's kernels.  "sum": a walk is split.
# Two column blocks (256 kept tokens a workgroup) are taken from 1.5 workgroups a CU on.
TWO = [
    # dK/dV, dQ; the walks long and short, whole and partial records and tiles
    (1.7, 1, 1, 1, 64, 330, 100, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 2, 2, 2, 64, 70, 70, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 1, 2, 1, 64, 300, 130, None, {"attn_dkv2", "attn_dq2"}),  # grouped: 20 turns
    (1.7, 1, 2, 1, 50, 97, 256, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 4, 4, 2, 40, 200, 300, "half", {"attn_dkv2", "attn_dq2", "attn_sum"}),
    (1.7, 3, 6, 3, 48, 260, 200, "run", {"attn_dkv2", "attn_dq2", "attn_sum"}),
    (1.7, 2, 4, 2, 33, 65, 64, "first_none", {"attn_dkv2", "attn_dq2", "attn_sum"}),
    (1.7, 2, 2, 2, 64, 130, 700, None, {"attn_dkv2", "attn_dq2"}),  # 21 whole records of keys
    (1.7, 1, 1, 1, 64, 65, 673, "half", {"attn_dkv2", "attn_dq2"}),
    (1.7, 1, 1, 1, 32, 290, 290, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 1, 1, 1, 20, 40, 1, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 1, 2, 1, 17, 300, 97, None, {"attn_dkv2", "attn_dq2"}),
    (1.7, 1, 1, 1, 24, 33, 600, "one", {"attn_dkv2", "attn_dq2"}),
    # one of the two walks alone has workgroups enough
    (1.7, 4, 4, 1, 64, 40, 50, None, {"attn_dq2", "attn_bwd", "attn_sum"}),
    (1.7, 3, 1, 1, 30, 12, 600, None, {"attn_dkv2", "attn_bwd", "attn_sum"}),
    (1.7, 3, 1, 1, 60, 12, 600, "half", {"attn_dkv2", "attn_bwd", "attn_sum"}),
]
# One column block: head_dim above 64, float32, few workgroups.
ONE = [
    (1.6, 1, 1, 1, 96, 40, 40, None, {"attn_bwd"}), (1.6, 1, 1, 1, 128, 70, 65, None, {"attn_bwd"}),
    (1.6, 1, 2, 1, 72, 40, 200, "half", None), (1.6, 2, 2, 2, 112, 130, 33, "half", None),
    # one walk split, the other not; both; neither
    (1.6, 1, 8, 1, 80, 33, 70, None, None), (1.6, 1, 8, 1, 100, 33, 130, "half", None),
    (None, 1, 1, 1, 96, 40, 600, None, {"attn_bwd", "attn_sum"}),
    (None, 1, 1, 1, 90, 600, 40, None, {"attn_bwd", "attn_sum"}),
    (None, 1, 2, 1, 100, 600, 40, None, {"attn_bwd", "attn_sum"}),
    (None, 1, 2, 1, 128, 40, 600, None, {"attn_bwd", "attn_sum"}),
    (None, 1, 1, 1, 70, 300, 300, None, {"attn_bwd", "attn_sum"}),
    (None, 1, 2, 2, 128, 300, 300, "half", {"attn_bwd", "attn_sum"}),
    # few kept tokens against so many that those fill the GPU
    (None, 1, 1, 1, 80, 17, 44900, None, None), (None, 1, 1, 1, 100, 17, 44900, None, None),
    (None, 1, 1, 1, 80, 44900, 5, None, None), (None, 1, 1, 1, 100, 44900, 5, None, None),
]
# One query row over keys enough for the wide pieces.
READ = [(2.2, 14, 2, 2, 40, 1, 13400, None, None), (2.2, 14, 2, 2, 16, 1, 13400, "half", None)]


def _case(c, dt):
    per_cu, each, heads, kv, hd, tq, tk, mk, _ = c
    n = 1 if per_cu is None else _volumes(per_cu, each)
    return (n, heads, kv, hd, tq, tk, mk, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("c", TWO + ONE + READ, ids=lambda c: "x%s_%d_h%d_%d_d%d_q%d_k%d_%s" % c[:8])
def test_kernels(c, dt):
    case = _case(c, dt)
    tags = _tags(lambda: TA._check(case))
    ran = {t for t in tags if t in ("attn_dkv2", "attn_dq2", "attn_bwd", "attn_sum")}
    print(case, ran, flush=True)
    if dt == "f32":
        assert "attn_bwd" in ran and not ran & {"attn_dkv2", "attn_dq2"}
    elif c[8] is not None:
        assert ran == c[8]
    if c in READ:
        assert "attn_few" in tags
