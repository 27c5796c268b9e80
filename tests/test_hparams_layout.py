"""chgnet_hparams as callers built before act_bits pass it."""
import ctypes
import struct

import pytest

from paper_2412_20796_amd import binding as bd


def test_hparams_keep_their_size():
    """Ten 32-bit fields, as before act_bits: a caller built with the older header passes these, and what lies behind them
    in its memory is not read."""
    bits = lambda x: struct.unpack("<i", struct.pack("<f", x))[0]
    assert ctypes.sizeof(bd.HParams) == 40
    n, want = ctypes.c_int64(), bd.param_count(bd.hparams())
    for behind in (0, 8, 0x7F7F7F7F, -1):
        old = (ctypes.c_int32 * 11)(64, 4, 31, 31, 8, bits(6.0), bits(3.0), 0, 0, 0, behind)
        assert bd.lib().chgnet_param_count(ctypes.cast(old, ctypes.POINTER(bd.HParams)), ctypes.byref(n)) == bd.CHGNET_OK
        assert n.value == want
    for conservative in (2, -1, 1 << 16, -(1 << 16)):  # refused as before
        old = (ctypes.c_int32 * 10)(64, 4, 31, 31, 8, bits(6.0), bits(3.0), 0, 0, conservative)
        assert bd.lib().chgnet_param_count(ctypes.cast(old, ctypes.POINTER(bd.HParams)), ctypes.byref(n)) == bd.CHGNET_EINVAL
    for kw in (dict(conservative=1 << 16), dict(act_bits=1 << 16), dict(act_bits=(1 << 16) + 8), dict(act_bits=-(1 << 15) - 8)):
        with pytest.raises(bd.ChgnetError) as e:  # and not by their low bits
            bd.param_count(bd.hparams(**kw))
        assert e.value.code == bd.CHGNET_EINVAL
