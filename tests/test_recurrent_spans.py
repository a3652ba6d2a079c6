"""Which results lie over other tensors: exact for any number of volumes and any strides."""
import ctypes
import random
import time

from paper_2104_05035_amd import rat3d as R
from tests.test_recurrent_abi import BIG, FAKE, _refused


def _meet(a, b):
    """Parts as (first address, number, stride, bytes held)."""
    fn = R.lib().rat3d_spans_meet
    fn.restype, fn.argtypes = ctypes.c_int, [ctypes.POINTER(ctypes.c_int64)] * 2
    return bool(fn(*((ctypes.c_int64 * 4)(*t) for t in (a, b))))


def _plain(a, b):
    return any(a[0] + i * a[2] < b[0] + j * b[2] + b[3] and b[0] + j * b[2] < a[0] + i * a[2] + a[3]
               for i in range(a[1]) for j in range(b[1]))


def test_small_parts_as_counted_one_by_one():
    rng = random.Random(5)
    seen = [0, 0]
    for _ in range(30000):
        t = []
        for _ in range(2):
            held = rng.randint(1, 12)
            t.append((1000 + rng.randint(0, 60), rng.randint(1, 7), held + rng.randint(0, 25), held))
        want = _plain(*t)
        seen[want] += 1
        assert _meet(*t) == want and _meet(*t[::-1]) == want, t
    assert min(seen) > 3000


def test_many_parts_of_different_strides():
    """Parts that first meet far behind the first, and ones that never do."""
    start = time.time()
    for n in (70000, 1 << 20, 1 << 30):
        a = (1 << 20, n, 128, 32)  # bytes 0 to 31 of every 128
        assert not _meet(a, (a[0] + 64, n, 256, 32))
        assert not _meet(a, (a[0] + 32, n, 384, 96))
        assert _meet(a, (a[0] + 32, n, 384, 97))
        assert _meet(a, (a[0] + 32, n, 97, 1))  # 97 is prime to 128
        # two parts, the first apart: the second over a's last part, or a byte before or behind
        last = 128 * (n - 1)
        assert _meet(a, (a[0] + 40, 2, last - 40, 1)) and _meet(a, (a[0] + 40, 2, last - 9, 1))
        assert not _meet(a, (a[0] + 40, 2, last - 41, 1))
        assert not _meet(a, (a[0] + 40, 2, last - 8, 1))
    assert time.time() - start < 5


def test_overlaps_behind_the_first_volumes():
    """A result whose volume 69999 alone lies in an input of another stride."""
    n, c, v = 70000, 3, 5
    held = 2 * c * v
    p = [FAKE + (i << 30) for i in range(9)]
    x = p[8]
    u = x - (n - 1) * (held + 4) - held + 2  # its last volume ends over x's first element
    assert u > p[7]
    d = R.norm_desc(n, c, v, R.BF16, u_stride=c * v + 2)
    _refused(R.EINVAL, R.rat3d_pre_norm_fwd, d, x, p[0], None, u)
    d = R.recurrence_desc(n, c, v, R.BF16, y_stride=c * v + 2)
    _refused(R.EINVAL, R.rat3d_recurrence_fwd, d, p[0], p[1], x, p[2], None, None, u, None, None,
             p[3], BIG)
