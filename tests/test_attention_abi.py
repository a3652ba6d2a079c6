"""The voxel self-attention calls refuse what they do not take, on the host, before
anything is enqueued; workspace sizes follow the descriptor."""
import ctypes

import pytest

from paper_2104_05035_amd import rat3d as R

FAKE = 0x10000  # aligned, never read: every call here is refused first
BAD = ctypes.c_size_t(-1).value


def _refused(status, f, *a):
    with pytest.raises(R.Rat3dError) as e:
        f(*a, stream=0)
    assert e.value.status == status
    assert str(e.value).split(": ", 1)[1]


def _att(**kw):
    d = dict(n=2, heads=4, kv_heads=2, head_dim=32, tq=50, tk=60, dtype=R.BF16)
    d.update(kw)
    return R.attention_desc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), R.EINVAL), (dict(heads=0), R.EINVAL), (dict(kv_heads=0), R.EINVAL),
    (dict(heads=3), R.EINVAL), (dict(head_dim=0), R.EINVAL), (dict(tq=0), R.EINVAL),
    (dict(tk=0), R.EINVAL), (dict(tk=-5), R.EINVAL), (dict(head_dim=129), R.EUNSUPPORTED),
    (dict(dtype=R.U8), R.EUNSUPPORTED), (dict(scale=-1.0), R.EINVAL),
    (dict(scale=1e-30), R.EINVAL), (dict(scale=1e30), R.EINVAL), (dict(scale=float("nan")), R.EINVAL), (dict(scale=float("inf")), R.EINVAL),
    (dict(q_stride=4 * 32 * 50 - 1), R.EINVAL), (dict(k_stride=1), R.EINVAL),
    (dict(v_stride=-1), R.EINVAL), (dict(o_stride=5), R.EINVAL),
    (dict(tk=(1 << 28) + 1), R.EUNSUPPORTED), (dict(n=1 << 30), R.EUNSUPPORTED),
    (dict(n=4096, tq=1 << 20), R.EUNSUPPORTED), (dict(n=1 << 21, tq=2, tk=1), R.EUNSUPPORTED), (dict(heads=1 << 30), R.EUNSUPPORTED),
])
def test_attention_descriptor(kw, status):
    d = _att(**kw)
    for i in (0, 1):
        assert R.rat3d_attention_workspace_size(d, i) == BAD
    _refused(status, R.rat3d_attention_fwd, d, FAKE, FAKE, FAKE, None, FAKE, None, FAKE, 1 << 40)
    _refused(status, R.rat3d_attention_bwd, d, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE,
             FAKE, FAKE, FAKE, 1 << 40)


def test_attention_pointers():
    d = _att()
    need = [R.rat3d_attention_workspace_size(d, i) for i in (0, 1)]
    assert 0 < need[0] < need[1] and R.rat3d_attention_workspace_size(d, 2) == BAD
    fwd = [FAKE, FAKE, FAKE, None, FAKE, None, FAKE, need[0]]
    for i in (0, 1, 2, 4):
        _refused(R.EINVAL, R.rat3d_attention_fwd, d, *(fwd[:i] + [None] + fwd[i + 1:]))
        _refused(R.EALIGN, R.rat3d_attention_fwd, d, *(fwd[:i] + [FAKE + 1] + fwd[i + 1:]))
    _refused(R.EWORKSPACE, R.rat3d_attention_fwd, d, *(fwd[:7] + [need[0] - 1]))
    _refused(R.EINVAL, R.rat3d_attention_fwd, d, *(fwd[:6] + [None, need[0]]))
    _refused(R.EALIGN, R.rat3d_attention_fwd, d, *(fwd[:6] + [FAKE + 8, need[0]]))
    bwd = [FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, need[1]]
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9):
        _refused(R.EINVAL, R.rat3d_attention_bwd, d, *(bwd[:i] + [None] + bwd[i + 1:]))
    _refused(R.EWORKSPACE, R.rat3d_attention_bwd, d, *(bwd[:11] + [need[1] - 1]))


def _qk(**kw):
    d = dict(n=2, heads=4, kv_heads=2, head_dim=32, d=3, h=4, w=5, dtype=R.BF16, rot=(8, 8, 8))
    d.update(kw)
    return R.qk_desc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(n=0), R.EINVAL), (dict(heads=-1), R.EINVAL), (dict(heads=0, kv_heads=0), R.EINVAL),
    (dict(head_dim=0), R.EINVAL), (dict(d=0), R.EINVAL), (dict(w=-3), R.EINVAL),
    (dict(rot=(3, 2, 2)), R.EINVAL), (dict(rot=(-2, 2, 2)), R.EINVAL),
    (dict(rot=(16, 16, 2)), R.EINVAL), (dict(rot=(2 ** 30, 2 ** 30, 2 ** 30)), R.EINVAL),
    (dict(origin=(1 << 25, 0, 0)), R.EINVAL), (dict(base=0.0), R.EINVAL),
    (dict(base=float("nan")), R.EINVAL), (dict(eps=0.0), R.EINVAL), (dict(eps=1e-40), R.EINVAL),
    (dict(eps=float("inf")), R.EINVAL), (dict(head_dim=130), R.EUNSUPPORTED),
    (dict(dtype=R.U8), R.EUNSUPPORTED), (dict(q_stride=1), R.EINVAL),
    (dict(ok_stride=2 * 32 * 60 - 1), R.EINVAL), (dict(d=1 << 20, h=1 << 20), R.EUNSUPPORTED),
    (dict(n=1 << 30), R.EUNSUPPORTED), (dict(d=1 << 30), R.EUNSUPPORTED),
    (dict(n=1 << 21), R.EUNSUPPORTED),
])
def test_qk_descriptor(kw, status):
    d = _qk(**kw)
    assert R.rat3d_rope_table_size(d) == BAD
    assert R.rat3d_qk_norm_rope_workspace_size(d) == BAD
    _refused(status, R.rat3d_rope_table, d, FAKE)
    _refused(status, R.rat3d_qk_norm_rope_fwd, d, *[FAKE] * 7)
    _refused(status, R.rat3d_qk_norm_rope_bwd, d, *[FAKE] * 11, 0, FAKE, 1 << 40)


def test_qk_pointers():
    d = _qk()
    assert R.rat3d_rope_table_size(d) == 8 * 4 * (3 + 4 + 5)
    need = R.rat3d_qk_norm_rope_workspace_size(d)
    assert need > 0
    fwd = [FAKE] * 7
    for i in range(7):
        _refused(R.EINVAL, R.rat3d_qk_norm_rope_fwd, d, *(fwd[:i] + [None] + fwd[i + 1:]))
    for i in (0, 1, 4, 5, 6):
        _refused(R.EALIGN, R.rat3d_qk_norm_rope_fwd, d, *(fwd[:i] + [FAKE + 1] + fwd[i + 1:]))
    bwd = [FAKE] * 11
    for i in range(11):
        _refused(R.EINVAL, R.rat3d_qk_norm_rope_bwd, d, *(bwd[:i] + [None] + bwd[i + 1:]), 0, FAKE,
                 need)
    _refused(R.EWORKSPACE, R.rat3d_qk_norm_rope_bwd, d, *bwd, 0, FAKE, need - 1)
    _refused(R.EINVAL, R.rat3d_rope_table, d, None)
    # without a norm no workspace, without rotation no table
    assert R.rat3d_qk_norm_rope_workspace_size(_qk(norm=False, eps=0.0)) == 0
    assert R.rat3d_rope_table_size(_qk(rot=(0, 0, 0), base=0.0)) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(count=0), R.EINVAL), (dict(unit=0), R.EINVAL), (dict(p=-0.1), R.EINVAL),
    (dict(p=1.1), R.EINVAL), (dict(p=float("nan")), R.EINVAL), (dict(dtype=R.U8), R.EUNSUPPORTED),
    (dict(count=(1 << 50) + 1), R.EUNSUPPORTED), (dict(unit=1 << 60), R.EUNSUPPORTED),
])
def test_dropout_descriptor(kw, status):
    d = dict(count=100, p=0.5, dtype=R.F32, unit=1)
    d.update(kw)
    d = R.dropout_desc(**d)
    _refused(status, R.rat3d_dropout_fwd, d, 0, None, FAKE, None, FAKE)
    _refused(status, R.rat3d_dropout_bwd, d, 0, None, FAKE, FAKE, 0)


def test_dropout_pointers():
    d = R.dropout_desc(100, 0.5, R.F32)
    _refused(R.EINVAL, R.rat3d_dropout_fwd, d, 0, None, None, None, FAKE)
    _refused(R.EINVAL, R.rat3d_dropout_fwd, d, 0, None, FAKE, None, None)
    _refused(R.EALIGN, R.rat3d_dropout_fwd, d, 0, None, FAKE + 4, None, FAKE)
    _refused(R.EALIGN, R.rat3d_dropout_fwd, d, 0, None, FAKE, FAKE + 4, FAKE)
    _refused(R.EALIGN, R.rat3d_dropout_fwd, d, 0, FAKE + 4, FAKE, None, FAKE)
    _refused(R.EINVAL, R.rat3d_dropout_bwd, d, 0, None, FAKE, None, 0)
    _refused(R.EALIGN, R.rat3d_dropout_bwd, d, 0, None, FAKE + 8, FAKE, 0)
