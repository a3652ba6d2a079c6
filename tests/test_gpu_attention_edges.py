"""Voxel self-attention on inputs at the edge of what it takes: infinite keys, sums over
very many voxels."""
import zlib

import numpy as np
import pytest

from tests import attn_util as AU
from tests import gpu_util as U

pytestmark = pytest.mark.gpu


def _rng(case):
    return np.random.default_rng(zlib.crc32(repr(case).encode()))


def _ws(nbytes):
    torch = U.torch_mod()
    return torch.full((max(int(nbytes), 16),), 0xFF, dtype=torch.uint8, device="cuda:0")


def _cus():
    return U.torch_mod().cuda.get_device_properties(0).multi_processor_count


# n (0: as many volumes as fill 1.5 workgroups a CU), heads, kv, hd, tq, tk, masked
INF = [(1, 1, 1, 20, 33, 65, False), (2, 4, 2, 32, 63, 130, True), (1, 2, 1, 128, 1, 300, False),
       (1, 2, 2, 96, 64, 64, False), (0, 2, 1, 24, 70, 60, False), (0, 1, 1, 40, 33, 70, True)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", INF, ids=lambda c: "n%d_h%d_%d_d%d_q%d_k%d_%d" % c)
def test_minus_infinity_in_a_key(case, dt):
    """A live key of -infinity in a channel where every query is positive has the score
    -infinity, so the probability 0: it takes no part in any result, and its gradients
    are 0.  dQ is NaN in that channel, 0 * -infinity, and nowhere else.  (tq leaves the
    last 32 queries' block unfilled in all cases but one.)"""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    n, heads, kv, hd, tq, tk, masked = case
    n = n or (3 * _cus() + 1) // 2
    rng = _rng((case, dt))
    mask = np.ones((n, tk), np.uint8)
    if masked:
        mask[:] = rng.random((n, tk)) < 0.5
    at = rng.integers(0, tk, (n, 3))
    at[:, 0] = tk - 1
    for i in range(n):
        mask[i, at[i]] = 1
        mask[i, (at[i].max() + 7) % tk] = 1
    a = rng.standard_normal((n, heads, hd, tq))
    a[:, :, 0] = np.abs(a[:, :, 0]) + 0.125
    q, qr = U.dev_input(a.reshape(n, heads * hd, tq), dt)
    k, kr = U.dev_input(rng.standard_normal((n, kv * hd, tk)), dt)
    v, vr = U.dev_input(rng.standard_normal((n, kv * hd, tk)), dt)
    do, dor = U.dev_input(rng.standard_normal((n, heads * hd, tq)), dt)
    without = mask.copy()
    for i in range(n):
        without[i, at[i]] = 0
        for j in at[i]:
            k[i, ::hd, int(j)] = float("-inf")
    m = torch.from_numpy(mask).to("cuda:0") if masked else None
    desc = R.attention_desc(n, heads, kv, hd, tq, tk, U.code(dt))
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    o, dq, dk, dv = (torch.empty_like(t) for t in (q, q, k, v))
    lse = U.zeros_f32((n, heads, tq))
    print("-inf", case, dt, flush=True)
    R.rat3d_attention_fwd(desc, q, k, v, m, o, lse, _ws(need[0]), need[0])
    U.sync()
    R.rat3d_attention_bwd(desc, do, q, k, v, m, o, lse, dq, dk, dv, _ws(need[1]), need[1])
    U.sync()
    want = AU.attention_refs(qr, kr, vr, heads, kv, without, hd ** -0.5, dt, dor)
    for name, t in (("o", o), ("lse", lse), ("dk", dk), ("dv", dv)):
        AU.within(U.f64(t), want[name], name)
    first = np.arange(heads * hd) % hd == 0
    g = U.f64(dq)
    assert np.all(np.isnan(g[:, first]))
    AU.within(g[:, ~first], tuple(t[:, ~first] for t in want["dq"]), "dq")

@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_gain_gradient_of_a_very_large_map(dt):
    """2^27 voxels with equal terms: the parts' float32 sums would drift by 4e-5
    (float32) and 4.7e-6 (bfloat16).  Terms: the norm and the product, head_dim + 16
    roundings as in the other tests; a thread adds up to 8 tokens and joins 32 threads
    in 5 steps; the parts are added in float64 and rounded once."""
    from paper_2104_05035_amd import rat3d as R
    torch = U.torch_mod()
    hd, grid = 2, (512, 512, 512)
    v = 512 ** 3
    desc = R.qk_desc(1, 1, 0, hd, *grid, U.code(dt), eps=1e-5)
    x = torch.ones((1, hd, v), dtype=U.tdtype(dt), device="cuda:0")
    dy = torch.full_like(x, 0.55)
    c = float(dy[0, 0, 0])
    g, dg = torch.ones(hd, device="cuda:0"), torch.zeros(hd, device="cuda:0")
    need = R.rat3d_qk_norm_rope_workspace_size(desc)
    dx = torch.empty_like(x)
    R.rat3d_qk_norm_rope_bwd(desc, dy, None, x, None, g, None, None, dx, None, dg, None, 0,
                             _ws(need), need)
    U.sync()
    want = np.full(hd, c / np.sqrt(1 + np.float64(np.float32(1e-5))) * v)
    AU.within(U.f64(dg), (want, (hd + 16 + 8 + 5 + 1) * AU.F * want), "dgamma")
