"""GPU tests of attention in serving at the ends of what fp32 holds."""
import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_seqs as S
from cases_seqs import C, I8
from test_gpu_seqs import _gpu, f64, ints, packed_inputs, paged_inputs, run_packed, run_paged, starts  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

VALUES = (float("nan"), float("inf"), -float("inf"), 1.0)


@pytest.mark.parametrize("flags", [0, C, I8, I8 | C])
def test_a_row_whose_scores_all_are_minus_infinity_is_zero(flags):
    # over values that are not finite too, in tiles that every row sees whole
    case = ([1, 40], [300, 290], 1, 2, 64, 16)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 97)
    rows[:] = 0
    rows[..., 0] = 1
    if flags & I8:
        cache[0][..., 0] = -1
        cache[2][:] = float("inf")
    else:
        cache[0][..., 0] = -float("inf")
    for bad in VALUES:
        cache[3 if flags & I8 else 1][:] = bad
        for text in S.legal(op, S.ATTENTION_TEXTS):
            got = f64(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]))
            assert not np.any(got != 0), bad


def test_a_packed_row_whose_scores_all_are_minus_infinity_is_zero():
    case = ([70, 3], [200, 300], 2, 4, 128)
    op = S.packed_op(case, C)
    q, k, v = packed_inputs(case, 98)
    q[:] = 0
    q[..., 0] = 1
    k[..., 0] = -float("inf")
    for bad in VALUES:
        v[:] = bad
        for text in S.legal(op, S.ATTENTION_TEXTS):
            got = f64(run_packed(op, text, [q, k, v], [0, 70, 73], [0, 200, 500]))
            assert not np.any(got != 0), bad
