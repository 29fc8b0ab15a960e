"""CPU tests of attention in serving with tables wider than the sequences need."""
import pytest

from paper_2506_01374_amd import rc

from cases_seqs import C, I8


@pytest.mark.parametrize("flags", [0, C, I8, I8 | C])
@pytest.mark.parametrize("t,b", [(1, 1), (64, 64), (80, 16), (600, 1), (512, 8), (2048, 4), (640, 32), (16384, 2), (100, 2000)])
def test_a_suggestion_holds_at_any_width(t, b, flags):
    for d in (64, 128, 256):
        for need in (1, 10, 40, 500):
            op = rc.Op(rc.RC_OP_ATTENTION_PAGED, (t, b, 32, 8, d, 16, 3000, need), flags)
            text = str(op.suggest())
            for width in (1, need, 8 * need, 2 ** 26):
                wide = rc.Op(rc.RC_OP_ATTENTION_PAGED, (t, b, 32, 8, d, 16, 3000, width), flags)
                sched = wide.from_string(text)
                assert sched.validate() == ""
                assert rc.kernel_defines(wide, sched) == rc.kernel_defines(op, op.suggest())
