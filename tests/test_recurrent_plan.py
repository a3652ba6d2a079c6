"""Plans of the recurrent block's norms (host side, no GPU needed): every size has a kernel
that is built for it, and stays within what that kernel assumes."""
import ctypes

import pytest

from paper_2104_05035_amd import rat3d as R

CHANNELS = [1, 3, 4, 15, 16, 17, 33, 48, 64, 65, 100, 127, 128, 129, 130, 144, 160, 200, 240, 255,
            256, 257, 272, 300, 384, 511, 512, 513, 600, 1024, 1 << 20]
VOXELS = [1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 32, 63, 64, 65, 127, 128, 130, 252, 1000, 1024, 2016, 16128,
          1 << 20, 1 << 24, (1 << 24) + 1, (1 << 25) + 64, (1 << 26) + 3, (1 << 27) + 64, 1 << 28]


def norm_plan(desc, pass_, masked, nxt):
    """None, or (tokens a thread, channels a thread, groups, tiles, workgroups)."""
    out = (ctypes.c_int64 * 5)()
    fn = R.lib().rat3d_norm_plan
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(R.NormDesc)] + [ctypes.c_int] * 3 + \
        [ctypes.POINTER(ctypes.c_int64)]
    return tuple(out) if fn(ctypes.byref(desc), pass_, masked, nxt, out) else None


@pytest.mark.parametrize("dt", [R.F32, R.BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gate", [R.GATE_NONE, R.GATE_SILU], ids=["plain", "gated"])
def test_norm_plans(gate, dt):
    es = 4 if dt == R.F32 else 2
    calls = [(0, m, 0) for m in (0, 1)] + [(1, m, 0) for m in (0, 1)] + \
        [(p, m, k) for p in (2, 3) for m in (0, 1) for k in (0, 1)]
    for c in CHANNELS:
        for v in VOXELS:
            for n in (1, 9, 300):
                d = R.norm_desc(n, c, v, dt, gate=gate)
                size = R.rat3d_norm_workspace_size(d)
                if (v / 16 + 1) * n >= 2e9:  # refused: too many tiles of single tokens
                    assert size == ctypes.c_size_t(-1).value
                    continue
                for call in calls:
                    plan = norm_plan(d, *call)
                    case = (n, c, v, call, plan)
                    assert plan is not None, case
                    tok, pc, groups, tiles, grid = plan
                    assert 1 <= tok * es <= 16 and tok <= v, case
                    assert groups % 4 == 0 and 4 <= groups <= 64, case  # whole waves
                    assert pc == 0 or pc * groups >= c, case
                    assert groups * v * es <= 1 << 32, case  # a group's rows in 32 bits
                    assert tiles == -(-v // (16 * tok)) * n < 1 << 31, case
                    if call[0] in (1, 3):
                        assert grid * 2 * c * (4 if pc else 8) <= size, case
                    else:
                        assert grid == tiles, case


def test_norm_plans_of_refused_descriptors():
    assert norm_plan(R.norm_desc(1, 0, 5, R.F32), 0, 0, 0) is None
    assert norm_plan(R.norm_desc(1, 4, 5, R.F32), 4, 0, 0) is None
