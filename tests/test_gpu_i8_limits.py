"""GPU tests of the 8-bit integer operators at and past the ends of their
ranges, against 64-bit references (test_gpu_i8's, with its tolerances)."""
import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_i8_limits as cases
from test_gpu_i8 import (B, BF16, F, G, R, U, _gpu, bf16, check_rows, f64, gemm_inputs, gemm_reference,  # noqa: F401
                         rows_inputs, rows_reference, run_gemm, run_rows)

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
# Products of a norm past fp32's range
# ---------------------------------------------------------------------------

def wide_reference(x, w, r, eps):
    """rows_reference, with a scale past fp32 as NaN."""
    q, scale, h = rows_reference(x, w, r, eps)
    past = ~(scale < 2.0 ** 128 - 2.0 ** 103)           # (rounds to an infinity)
    scale[past] = np.nan
    q[past] = 0
    return q, scale, h


def check_wide(x, w, r, text, eps, alias=None):
    x, w, r = (None if v is None else f64(bf16(v)) for v in (x, w, r))
    q, scale, h = wide_reference(x, w, r, eps)
    got = run_rows(rc.RC_OP_RMSNORM_I8, 0 if r is None else R, x, w, r, text, eps, alias)
    assert np.array_equal(got[0].cpu().numpy(), q)
    s, ok = f64(got[1]), ~np.isnan(scale)
    assert np.array_equal(np.isnan(s), ~ok)
    # as test_gpu_i8's; a scale below fp32's normal range has its absolute step
    tol = ((-(-x.shape[1] // 64) + 21) / 2 + 5) * U
    assert np.all(np.abs(s - scale)[ok] <= tol * scale[ok] + 2.0 ** -149)
    if r is not None:
        assert np.array_equal(f64(got[2]), h, equal_nan=True)
    return q, scale


@pytest.mark.parametrize("text", cases.WIDE_TEXTS)
@pytest.mark.parametrize("hx,wx,eps", [(58, 70, 1e-5), (-75, -70, 1e-5), (-80, -75, 2.0 ** -100), (-120, 100, 1e-5), (50, 120, 1e-5),
                                       (30, 125, 2.0 ** -100), (-130, -130, 2.0 ** -100), (0, -63, 1e-5), (-4, 66, 1e-5),
                                       (-60, -66, 1e-5)])
def test_products_past_fp32(text, hx, wx, eps):
    # rows around the exponents hx of h and wx of w, next to ordinary ones, with
    # zeros, NaN and an infinity among them
    g = np.random.default_rng(1000 * (hx + 200) + wx + 200)
    t, c = 12, cases.WIDE_COLS
    x = g.standard_normal((t, c)) * 2.0 ** hx
    x[3] = g.standard_normal(c)
    x[5] = 0
    x[6, 10], x[7, 699] = np.nan, np.inf
    x[8, ::2] *= 2.0 ** -20
    x[9] = np.where(np.arange(c) % 3 == 0, x[9], 0)
    w = g.standard_normal(c) * 2.0 ** wx
    w[5], w[11] = 0, 2.0 ** wx
    q, scale = check_wide(x, w, None, text, eps)
    assert np.abs(q[0]).max() == 127 and np.isnan(scale[6]) and scale[5] == 0
    r = g.standard_normal((t, c)) * 2.0 ** hx
    check_wide(x, w, r, text, eps)
    check_wide(x, w, r, text, eps, alias=0)
    check_wide(x, w, r, text, eps, alias=2)


def test_products_of_all_exponents_in_one_row():
    # each row's products span fp32's range and more: h and w from 2^-130 to
    # 2^60 and 2^120, the largest product anywhere
    g = np.random.default_rng(5)
    t, c = 40, cases.WIDE_COLS
    x = g.standard_normal((t, c)) * 2.0 ** g.integers(-130, 60, (t, c))
    w = g.standard_normal(c) * 2.0 ** g.integers(-130, 120, c)
    check_wide(x, w, None, None, 1e-5)
    # and a few next to the largest, at and next to halves of its 127th
    x = 2.0 ** -70 * f64(bf16(np.concatenate([np.full((t, 1), 127.0), (g.integers(-127, 127, (t, c - 1)) + 0.5)], axis=1)))
    w = np.full(c, 2.0 ** -70)
    check_wide(x, w, None, None, 1e-5)
    w = 2.0 ** -70 * f64(bf16(1 + g.random(c)))
    check_wide(x, w, None, None, 1e-5)


def test_a_scale_past_fp32():
    # one value in 2^17 columns: y is 2^8.5 times its weight
    c = 1 << 17
    x, w = np.zeros((3, c)), np.ones(c)
    x[0, 7], x[1, 8], x[2, 9] = 1.0, -3.0, 5.0
    w[7], w[8], w[9] = 2.0 ** 127, 1.0, 2.0 ** 125
    q, scale = check_wide(x, w, None, None, 2.0 ** -100)
    assert np.isnan(scale[0]) and q[0, 7] == 0 and q[1, 8] == -127 and q[2, 9] == 127


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


# ---------------------------------------------------------------------------
# Every suggested schedule
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("kind,flags", [(rc.RC_OP_QUANT_I8, 0), (rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)])
def test_every_suggested_schedule_of_rows(kind, flags):
    for i, ((t, c), text) in enumerate(cases.suggested_rows(kind, flags)):
        x, w, r = rows_inputs(t, c, 500 + i)
        norm = kind == rc.RC_OP_RMSNORM_I8
        check_rows(kind, flags, x, w if norm else None, r if flags else None, text=text)


@pytest.mark.parametrize("stages", [1, 2, 3])
@pytest.mark.parametrize("flags", [0, B, F, B | F, G])
def test_every_suggested_product(flags, stages):
    jobs = [(d, t) for d, t in cases.suggested_products(flags) if f"stages={stages}" in t]
    assert jobs
    for i, (dims, text) in enumerate(jobs):
        ins = gemm_inputs(dims, flags, 1000 * flags + i)
        dev = [t.cuda().double() for t in ins]

        # the exact sums, as in gemm_reference (64 bits hold them), and its bounds
        def product(b, s):
            return torch.mm(dev[0], b.t().contiguous()).mul_(dev[1][:, None]).mul_(s[None, :])

        want = product(dev[2], dev[3])
        got = run_gemm(dims, flags, ins, text).double()
        if flags & G:
            y, u = want, product(dev[4], dev[5])
            want = y / (1 + torch.exp(-y)) * u
            tol = want.abs() * (BF16 + 2 * (4 * y.abs() + 9 + 3 * (1 + y.abs()) + 3 + 1) * U) + 2.0 ** -133
        else:
            tol = 3 * U * want.abs()
            if flags & B:
                want = want + dev[4][None, :]
                tol = tol + U * want.abs()
            tol = tol * 1.01 + (0 if flags & F else BF16) * want.abs() + 2.0 ** -133
        assert bool(((got - want).abs() <= tol).all()), (dims, text)


# ---------------------------------------------------------------------------
# Scales whose product leaves fp32's range
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("text", ["tile_m=16,tile_n=16,tile_k=64,stages=1", "tile_m=32,tile_n=32,tile_k=128,stages=2",
                                  "tile_m=16,tile_n=16,tile_k=64,stages=3,waves_k=2", "tile_m=32,tile_n=32,tile_k=64,stages=1,splits=2"])
@pytest.mark.parametrize("flags", [F, G])
def test_scales_whose_product_leaves_fp32(flags, text):
    dims = (40, 70, 512)
    ins = gemm_inputs(dims, flags, 17)
    ins[0][5], ins[0][6] = 0, 0                                     # sums of 0
    low = ins[1] * 2.0 ** -70
    high = ins[1] * 2.0 ** 90
    for sa, sb, whole in ((low, 2.0 ** -55, 0), (high, 2.0 ** 60, 1), (high, 2.0 ** -100, 0)):
        if flags & G:
            sets = [ins[0], sa, ins[2], ins[3] * sb, ins[4], ins[5] * sb]
        else:
            sets = [ins[0], sa, ins[2], ins[3] * sb]
        got = f64(run_gemm(dims, flags, sets, text))
        want, tol = gemm_reference(sets, flags)
        if whole:
            # past fp32 but for the rows of zeros (gated: 0 times anything finite)
            assert np.all(got[5:7] == 0) and not np.isfinite(got[0]).all()
            continue
        # (below the types' normal range a step is absolute)
        least = 2.0 ** -149 if flags & F else 2.0 ** -133
        assert np.all(np.abs(got - want) <= tol + least), np.max(np.abs(got - want) - tol)
        assert np.abs(want).max() > 2.0 ** -126 or flags & G       # (a normal number)
