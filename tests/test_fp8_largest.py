"""The largest sizes that the 8-bit quantiser takes (no GPU: the calls here end in its checks, and have no memory)."""
import ctypes

import pytest

from paper_2412_20796_amd import binding as bd
from paper_2412_20796_amd import ops

P = 1 << 20  # an address that is aligned and never read


def _matrix(rows, cols, br):
    return ops._Fp8(rows, cols, P, -(-cols // 16) * 16, P, -(-cols // 512) * 4, br)


@pytest.mark.parametrize("forms,br", [("q", 128), ("t", 128), ("t", 1), ("qt", 1), ("qt", 128)])
@pytest.mark.parametrize("rows,cols", [(1 << 23, 1 << 23), (1 << 23, (1 << 17) - 127), ((1 << 17) - 511, 1 << 23)])
def test_more_tiles_than_a_launch_has(rows, cols, forms, br):
    """2^24 blocks of 256 threads, one for 512 x 128 values, would be 2^32 threads."""
    q, t = (_matrix(rows, cols, br) if "q" in forms else None), (_matrix(cols, rows, br) if "t" in forms else None)
    ref = lambda m: None if m is None else ctypes.addressof(m)
    assert ops.lib().chgnet_fp8_quantize(rows, cols, 1, P, cols, ref(q), ref(t), None) == bd.CHGNET_EINVAL
    assert b"2^40" in bd.lib().chgnet_last_error_string()
