"""Calls of the voxel self-attention that the library refuses on the host because
their result would be wrong: float32 operands between two elements, one gradient for
two gains, results that lie over another volume's input."""
import pytest

from paper_2104_05035_amd import rat3d as R

FAKE = 0x10000  # aligned, never read: every call here is refused first


def _refused(status, f, *a):
    with pytest.raises(R.Rat3dError) as e:
        f(*a, stream=0)
    assert e.value.status == status
    assert str(e.value).split(": ", 1)[1]


def _with(args, at, value):
    return args[:at] + [value] + args[at + 1:]


def _qk(**kw):
    d = dict(n=2, heads=4, kv_heads=2, head_dim=32, d=3, h=4, w=5, dtype=R.BF16, rot=(8, 8, 8))
    d.update(kw)
    return R.qk_desc(**d)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_float32_operands_are_aligned(off):
    # gains: operands 2 and 3 of the forward, 4, 5 and (gradients) 9, 10 of the backward
    d = _qk()
    need = R.rat3d_qk_norm_rope_workspace_size(d)
    for i in (2, 3):
        _refused(R.EALIGN, R.rat3d_qk_norm_rope_fwd, d, *_with([FAKE] * 7, i, FAKE + off))
    for i in (4, 5, 9, 10):
        _refused(R.EALIGN, R.rat3d_qk_norm_rope_bwd, d, *_with([FAKE] * 11, i, FAKE + off), 0,
                 FAKE, need)
    a = R.attention_desc(2, 4, 2, 32, 50, 60, R.BF16)
    need = [R.rat3d_attention_workspace_size(a, i) for i in (0, 1)]
    _refused(R.EALIGN, R.rat3d_attention_fwd, a, FAKE, FAKE, FAKE, None, FAKE, FAKE + off, FAKE,
             need[0])
    _refused(R.EALIGN, R.rat3d_attention_bwd, a, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE + off,
             FAKE, FAKE, FAKE, FAKE, need[1])


@pytest.mark.parametrize("apart", [0, 1, 31, -31])
def test_gain_gradients_have_a_place_each(apart):
    """One gain for queries and keys is fine, one gradient for both is not: each side
    writes its own (or adds to it), and the sum would be lost."""
    d = _qk()
    need = R.rat3d_qk_norm_rope_workspace_size(d)
    _refused(R.EINVAL, R.rat3d_qk_norm_rope_bwd, d, *[FAKE] * 9, FAKE, FAKE + 4 * apart, 0, FAKE,
             need)
    _refused(R.EINVAL, R.rat3d_qk_norm_rope_bwd, d, *[FAKE] * 9, FAKE, FAKE + 4 * apart, 1, FAKE,
             need)


def test_in_place_needs_equal_strides():
    """Over its input a result has to lie where the input lies, in every volume."""
    packed = 4 * 32 * 60
    for kw in (dict(q_stride=packed + 8), dict(oq_stride=packed + 8), dict(k_stride=packed),
               dict(ok_stride=packed)):
        d = _qk(**kw)
        need = R.rat3d_qk_norm_rope_workspace_size(d)
        q = kw.keys() & {"q_stride", "oq_stride"}
        fwd = [FAKE, FAKE * 2, FAKE, FAKE, FAKE] + ([FAKE, FAKE * 3] if q else [FAKE * 3, FAKE * 2])
        _refused(R.EINVAL, R.rat3d_qk_norm_rope_fwd, d, *fwd)
        bwd = [FAKE, FAKE * 2] + [FAKE * 5] * 5 + fwd[5:] + [FAKE * 6, FAKE * 7]
        _refused(R.EINVAL, R.rat3d_qk_norm_rope_bwd, d, *bwd, 0, FAKE, need)
