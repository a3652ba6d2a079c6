"""Voxel self-attention on channel ranges of wider tensors: every operand with a stride
and a first element of its own, in every path; what lies between the ranges stays."""
import numpy as np
import pytest

from oracle import attention as A
from tests import attn_util as AU
from tests import gpu_util as U
from tests import test_gpu_attention as TA
from tests import test_gpu_qk_dropout as TQ

pytestmark = pytest.mark.gpu

REST = 77.0


class Range:
    """`shape` [n][c][t] inside a buffer filled with REST: volume i begins at element
    first + i * stride."""

    def __init__(self, shape, dt, first, gap):
        torch = U.torch_mod()
        n, c, t = shape
        self.shape, self.first, self.stride = shape, first, c * t + gap
        self.buf = torch.full((first + n * self.stride + 16,), REST, dtype=U.tdtype(dt),
                              device="cuda:0")
        self.ptr = self.buf.data_ptr() + first * self.buf.element_size()

    def _view(self, buf):
        n, c, t = self.shape
        return [buf[self.first + i * self.stride:][:c * t] for i in range(n)]

    def put(self, x):
        for row, v in zip(self._view(self.buf), x):
            row.copy_(v.reshape(-1))
        return self

    def get(self):
        """The values, float64, after a look at what lies between them."""
        a = U.f64(self.buf)
        out = np.stack([r.copy() for r in self._view(a)]).reshape(self.shape)
        for r in self._view(a):
            r[:] = REST
        assert np.all(a == REST), "written between the ranges"
        return out


#        n heads kv hd tq tk mask: one tile, split, many volumes, few rows of either width
CASES = [(2, 4, 2, 24, 75, 61, "half"), (3, 2, 1, 40, 130, 700, None), (2, 2, 2, 64, 300, 300, "run"),
         (2, 2, 1, 100, 50, 600, "half"), (230, 2, 2, 40, 33, 70, "half"), (230, 2, 2, 64, 65, 40, None),
         (3, 4, 2, 33, 1, 900, "half"), (2, 4, 2, 20, 1, 2049, None), (2, 6, 2, 16, 2, 1030, "half"),
         (20, 3, 3, 8, 1, 20500, "half"), (2, 3, 1, 24, 40, 2100, "first_none")]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "n%d_h%d_%d_d%d_q%d_k%d_%s" % c)
def test_attention(case, dt):
    from paper_2104_05035_amd import rat3d as R
    n, heads, kv, hd, tq, tk, mk = case
    (q, k, v, do, m), (qr, kr, vr, dor, mask) = TA._tensors(case + (dt,))
    x = dict(q=(q, 1, 7), k=(k, 3, 129), v=(v, 5, 0), do=(do, 2, 31))
    x = {s: Range(t.shape, dt, at, gap).put(t) for s, (t, at, gap) in x.items()}
    # a descriptor has one stride for o and dout, one for q and dq, and so on
    y = {s: Range(like.shape, dt, at, gap) for s, like, at, gap in (
        ("o", q, 9, 31), ("dq", q, 11, 7), ("dk", k, 1, 129), ("dv", v, 7, 0))}
    lse, buf = U.guarded((n, heads, tq), "f32")
    desc = R.attention_desc(n, heads, kv, hd, tq, tk, U.code(dt), q_stride=x["q"].stride,
                            k_stride=x["k"].stride, v_stride=x["v"].stride,
                            o_stride=y["o"].stride)
    assert y["o"].stride == x["do"].stride
    need = [R.rat3d_attention_workspace_size(desc, i) for i in (0, 1)]
    print("strides", case, dt, flush=True)
    R.rat3d_attention_fwd(desc, x["q"].ptr, x["k"].ptr, x["v"].ptr, m, y["o"].ptr, lse,
                          TA._ws(need[0]), need[0])
    U.sync()
    R.rat3d_attention_bwd(desc, x["do"].ptr, x["q"].ptr, x["k"].ptr, x["v"].ptr, m, y["o"].ptr, lse,
                          y["dq"].ptr, y["dk"].ptr, y["dv"].ptr, TA._ws(need[1]), need[1])
    U.sync()
    U.guard_intact(buf, "lse")
    want = AU.attention_refs(qr, kr, vr, heads, kv, mask, hd ** -0.5, dt, dor)
    AU.within(U.f64(lse), want["lse"], "lse")
    for s, r in y.items():
        AU.within(r.get(), want[s], s)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("n,hd,norm", [(2, 24, True), (2, 33, False), (2, 90, True), (600, 20, True)])
def test_qk_norm_rope(n, hd, norm, dt):
    from paper_2104_05035_amd import rat3d as R
    heads, kv, grid, rot = 2, 1, (3, 5, 19), (6, 4, 6)
    v = 285
    rng = TQ._rng((n, hd, norm, dt, "strides"))
    turn = A.rotation(hd, grid, rot, (0, 0, 0), 100.0)
    d = {}
    for s, many, gap in (("q", heads, 3), ("k", kv, 64)):
        x, d[s + "r"] = U.dev_input(rng.standard_normal((n, many * hd, v)) * 2, dt)
        dy, d["d" + s + "r"] = U.dev_input(rng.standard_normal((n, many * hd, v)), dt)
        d["g" + s], d["g" + s + "r"] = U.dev_input(1 + 0.3 * rng.standard_normal(hd), "f32")
        d[s] = Range(x.shape, dt, 1, gap).put(x)
        d["do" + s] = Range(x.shape, dt, 3, gap + 6).put(dy)
        d["o" + s] = Range(x.shape, dt, 5, gap + 6)
        d["d" + s] = Range(x.shape, dt, 7, gap)
        d["dg" + s] = U.guarded((hd,), "f32")
    desc = R.qk_desc(n, heads, kv, hd, *grid, U.code(dt), rot=rot, eps=1e-5, norm=norm,
                     q_stride=d["q"].stride, k_stride=d["k"].stride, oq_stride=d["oq"].stride,
                     ok_stride=d["ok"].stride)
    table = TQ._ws(R.rat3d_rope_table_size(desc))
    R.rat3d_rope_table(desc, table)
    need = R.rat3d_qk_norm_rope_workspace_size(desc)
    print("strides", n, hd, norm, dt, flush=True)
    R.rat3d_qk_norm_rope_fwd(desc, d["q"].ptr, d["k"].ptr, d["gq"], d["gk"], table, d["oq"].ptr,
                             d["ok"].ptr)
    R.rat3d_qk_norm_rope_bwd(desc, d["doq"].ptr, d["dok"].ptr, d["q"].ptr, d["k"].ptr, d["gq"],
                             d["gk"], table, d["dq"].ptr, d["dk"].ptr, d["dgq"][0], d["dgk"][0], 0,
                             TQ._ws(need), need)
    U.sync()
    for s, many in (("q", heads), ("k", kv)):
        gr = d["g" + s + "r"] if norm else None
        AU.within(d["o" + s].get(), TQ._qk_bounds(dt, d[s + "r"], many, gr, turn, 1e-5), "o" + s)
        dx, dg = TQ._qk_bounds(dt, d[s + "r"], many, gr, turn, 1e-5, d["d" + s + "r"])
        AU.within(d["d" + s].get(), dx, "d" + s)
        U.guard_intact(d["dg" + s][1], "dg")
        if norm:
            AU.within(U.f64(d["dg" + s][0]), dg, "dg" + s)
