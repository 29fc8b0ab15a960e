"""CPU tests of the 8-bit integer operators at and past the ends of their
ranges."""
import ctypes

import pytest

from paper_2506_01374_amd import rc

R, B, F, G = rc.RC_FLAG_RESIDUAL, rc.RC_FLAG_BIAS, rc.RC_FLAG_OUT_F32, rc.RC_FLAG_GATED


@pytest.mark.parametrize("kind,flags", [(rc.RC_OP_QUANT_I8, 0), (rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)])
@pytest.mark.parametrize("rows", [2 ** 26, 2 ** 57, 2 ** 58, 2 ** 58 + 1, 2 ** 62 + 3, 2 ** 63 - 1])
def test_rows_past_every_limit_are_refused(kind, flags, rows):
    # (64 threads for each row leave 64 bits from 2^58 rows on)
    with pytest.raises(rc.RCError) as e:
        rc.Op(kind, (rows, 8), flags)
    assert e.value.status == rc.RC_ERR_UNSUPPORTED
    op = rc.Op(kind, (8, 8), flags)
    sched = op.suggest()
    op.desc.dim[0] = rows
    s = rc.rc_schedule()
    assert rc.lib().rc_default_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    assert rc.lib().rc_suggest_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    assert "2^32 - 1 threads" in sched.validate()
