"""What the attention's plan promises, without a GPU: kernels that are built are kernels
that calls reach."""
import re

from paper_2104_05035_amd import rat3d as R


def test_no_two_block_dq_over_split_keys():
    """dQ on two column blocks a wave is taken from 1.5 workgroups a CU on, where a split
    of the keys would give floor(2 CUs / groups + 1/2) = 1 part: an instance over several
    parts could not run, and one that would not skip an empty part would add the last
    keys again for it."""
    R.lib()
    with open(R.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"attn_dq2_kI([A-Za-z0-9]+?)EEv", f.read()))
    assert names and all(re.fullmatch(rb"Li[12]E|Li[12]ELb0E?", n) for n in names), names
    for cus in (1, 8, 64, 256, 304):
        for groups in range((3 * cus + 1) // 2, 6 * cus):
            assert (2 * cus + groups // 2) // groups <= 1


def test_read_out_workspace_holds_its_sums_alone():
    """A forward of few query rows reads the mask itself: its workspace is the pieces'
    maxima, sums and values, with no list of live keys (4 bytes a key)."""
    for n, heads, kv, hd, tq, tk, dt, rows in ((1, 1, 1, 128, 1, 20_000_003, R.BF16, 1),
                                               (3, 4, 2, 40, 1, 5_000_001, R.F32, 2),
                                               (2, 6, 2, 32, 2, 3_000_000, R.F32, 8)):
        d = R.attention_desc(n, heads, kv, hd, tq, tk, dt)
        piece = 2048 if dt == R.BF16 else 1024  # keys
        sums = n * kv * -(-tk // piece) * rows * (hd + 2) * 4
        assert R.rat3d_attention_workspace_size(d, 0) == -(-sums // 256) * 256
