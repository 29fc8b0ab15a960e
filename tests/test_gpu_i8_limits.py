"""GPU tests of the 8-bit integer operators at and past the ends of their
ranges, against 64-bit references (test_gpu_i8's, with its tolerances)."""
import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_i8_limits as cases
from test_gpu_i8 import R, U, _gpu, bf16, f64, gemm_inputs, rows_reference, run_rows  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def test_overlapping_buffers_are_refused():
    x, y = torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda"), torch.zeros(64, 256, dtype=torch.bfloat16, device="cuda")
    w, q, s = y[0], torch.empty(64, 256, dtype=torch.int8, device="cuda"), torch.empty(64, device="cuda")
    over = x.view(torch.int8).flatten()[:64 * 256].view(64, 256)
    for kind, flags, ins, outs in ((rc.RC_OP_QUANT_I8, 0, [x], (over, s)), (rc.RC_OP_RMSNORM_I8, R, [x, w, y], (over, s, y)),
                                   (rc.RC_OP_RMSNORM_I8, R, [x, x[0], y], (q, s, x))):
        op = rc.Op(kind, (64, 256), flags)
        plan = rc.Plan(op, op.suggest())
        for launch in (plan.launch, plan.launch_static, plan.time):
            with pytest.raises(rc.RCError, match="overlaps") as e:
                launch(ins, outs)
            assert e.value.status == rc.RC_ERR_INVALID_ARGUMENT
    # the workspace, where a schedule needs one
    dims = (33, 70, 1001)
    op = rc.Op(rc.RC_OP_GEMM_I8, dims)
    plan = rc.Plan(op, op.from_string("tile_m=32,tile_n=32,tile_k=128,mfma=16,stages=2,splits=4,pad=1"))
    ws = plan.workspace()
    ins = [t.cuda() for t in gemm_inputs(dims, 0, 1)]
    out = ws[:33 * 70 * 2].view(torch.bfloat16).view(33, 70)
    with pytest.raises(rc.RCError, match="workspace overlaps"):
        plan.launch(ins, out, ws)


# ---------------------------------------------------------------------------
# Long rows
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("flags", [0, R])
@pytest.mark.parametrize("cols,text", cases.LONG_ROWS)
def test_the_sum_of_squares_of_a_long_row(cols, text, flags):
    # Equal squares, whose additions all round the same way.  The tolerance
    # knows nothing of the row's length: 8 terms of a vector, 3 u of the
    # compensated sum, 6 + 15 across lanes and waves, halved by the root, and 5 u.
    x = np.full((2, cols), f64(bf16(np.array([1.1171875])))[0])
    x[1] = 3.0 + 2.0 ** -6
    x[:, ::2] *= -1
    w, r = np.ones(cols), 0.0 * x if flags else None
    q, scale, h = rows_reference(x, w, r)
    got = run_rows(rc.RC_OP_RMSNORM_I8, flags, x, w, r, text)
    assert np.array_equal(got[0].cpu().numpy(), q)
    assert np.all(np.abs(f64(got[1]) - scale) <= ((8 + 3 + 21) / 2 + 5) * U * scale)
    if flags:
        assert np.array_equal(f64(got[2]), h)
