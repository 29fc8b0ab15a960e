"""CPU tests of the 8-bit integer operators: descriptors, refusals, schedules
and their legality, the work model, and the tensor checks of the binding."""
import ctypes

import pytest

from paper_2506_01374_amd import rc

import cases_i8

torch = pytest.importorskip("torch")

R, B, F, G = rc.RC_FLAG_RESIDUAL, rc.RC_FLAG_BIAS, rc.RC_FLAG_OUT_F32, rc.RC_FLAG_GATED
KINDS = [(rc.RC_OP_RMSNORM_I8, (3, 100), 0), (rc.RC_OP_RMSNORM_I8, (3, 100), R), (rc.RC_OP_QUANT_I8, (3, 100), 0)] + [
    (rc.RC_OP_GEMM_I8, (3, 100, 70), f) for f in (0, B, F, B | F, G)]


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_descriptor_and_default(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    assert op.default().validate() == "" and op.suggest().validate() == ""
    for i, name in enumerate(op.knob_names()):
        assert op.default().raw.knob[i] == min(op.knob_values(i)), name
        assert op.knob_class(i) in ("TileSize", "Parallel", "Vectorize", "Unroll", "ComputeLocation", "Layout")
    # every move from the default is legal and can be undone
    for t in op.default().moves():
        assert op.default().apply(t).validate() == ""


@pytest.mark.parametrize("kind,dims,flags,status", [
    (rc.RC_OP_RMSNORM_I8, (0, 8), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_RMSNORM_I8, (8, 0), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_RMSNORM_I8, (8,), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_RMSNORM_I8, (8, 8), B, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_QUANT_I8, (8, 8), R, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_QUANT_I8, (1 << 26, 8), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_QUANT_I8, (1, (1 << 30) + 1), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_I8, (8, 8), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_GEMM_I8, (8, 8, -1), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_GEMM_I8, (8, 8, 8), R, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_GEMM_I8, (8, 8, 8), G | B, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_GEMM_I8, (8, 8, 8), G | F, rc.RC_ERR_INVALID_ARGUMENT),
    (rc.RC_OP_GEMM_I8, (8, 8, 131072), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_I8, (1 << 31, 8, 8), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_I8, (8, (1 << 30) + 1, 8), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_I8, (1 << 20, 16400, 8), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_F32, (8, 8, 8), B, rc.RC_ERR_INVALID_ARGUMENT)])
def test_refused_descriptors(kind, dims, flags, status):
    with pytest.raises(rc.RCError) as e:
        rc.Op(kind, dims, flags)
    assert e.value.status == status


def test_a_descriptor_made_by_hand_is_checked_too():
    op = rc.Op(rc.RC_OP_GEMM_I8, (8, 8, 64))
    op.desc.dim[2] = 131072
    s = rc.rc_schedule()
    assert rc.lib().rc_default_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    assert rc.lib().rc_suggest_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    op = rc.Op(rc.RC_OP_RMSNORM_I8, (8, 64))
    sched = op.suggest()
    op.desc.eps = -1.0
    assert "eps" in sched.validate()


def test_eps():
    assert rc.Op(rc.RC_OP_RMSNORM_I8, (1, 8)).eps == pytest.approx(1e-6)
    assert rc.Op(rc.RC_OP_RMSNORM_I8, (1, 8), eps=2.0 ** -100).eps == 2.0 ** -100
    for eps in (-1e-9, 0.0, 1e-31, float("nan"), float("inf"), 1e39):
        with pytest.raises(ValueError):
            rc.Op(rc.RC_OP_RMSNORM_I8, (1, 8), eps=eps)
    with pytest.raises(ValueError):
        rc.Op(rc.RC_OP_QUANT_I8, (1, 8), eps=1e-6)


def test_the_other_kinds_have_no_suggestion():
    with pytest.raises(rc.RCError) as e:
        rc.Op(rc.RC_OP_GEMM_F32, (8, 8, 8)).suggest()
    assert e.value.status == rc.RC_ERR_UNSUPPORTED


def test_work_model():
    q = rc.Op(rc.RC_OP_QUANT_I8, (10, 100))
    assert q.flops() == 0 and q.bytes() == 3 * 1000 + 40 and q.bound() == "hbm"
    assert rc.Op(rc.RC_OP_RMSNORM_I8, (10, 100)).bytes() == 3 * 1000 + 200 + 40
    assert rc.Op(rc.RC_OP_RMSNORM_I8, (10, 100), R).bytes() == 7 * 1000 + 200 + 40
    g = rc.Op(rc.RC_OP_GEMM_I8, (10, 20, 30))
    assert g.flops() == 2 * 6000 and g.peak_flops() == 5033.2e12
    assert g.bytes() == 300 + 40 + 600 + 80 + 400
    assert rc.Op(rc.RC_OP_GEMM_I8, (10, 20, 30), B | F).bytes() == 300 + 40 + 600 + 160 + 800
    gated = rc.Op(rc.RC_OP_GEMM_I8, (10, 20, 30), G)
    assert gated.flops() == 4 * 6000 and gated.bytes() == 300 + 40 + 2 * 680 + 400


def test_rows_legality():
    op = rc.Op(rc.RC_OP_QUANT_I8, (100, 1000))
    assert "16 waves" in op.schedule(waves=8, rows=4).validate()
    assert "do not hold" in op.schedule(vec=8, held=1).validate()
    assert op.schedule(vec=8, held=2).validate() == ""
    assert "already hold" in op.schedule(vec=8, held=4).validate()
    assert "already cover" in op.schedule(vec=8, waves=4).validate()
    assert "already cover T" in rc.Op(rc.RC_OP_QUANT_I8, (1, 1000)).schedule(rows=2).validate()
    # a grid is counted in threads: 2^26 - 1 rows are a wave each
    huge = rc.Op(rc.RC_OP_QUANT_I8, (2 ** 26 - 1, 4096))
    assert huge.default().validate() == "" and "2^32 - 1 threads" in huge.schedule(waves=2).validate()
    assert huge.suggest()["waves"] == 1
    assert "vec 4 already" in rc.Op(rc.RC_OP_QUANT_I8, (1, 4)).schedule(vec=8).validate()


def test_gemm_legality():
    op = rc.Op(rc.RC_OP_GEMM_I8, (1000, 1000, 1000))
    assert "multiple of the 32x32" in op.schedule(mfma=32).validate()
    assert "exceed 256" in op.schedule(tile_m=256, tile_n=256).validate()
    assert "LDS" in op.schedule(tile_m=256, tile_n=256, waves_m=4, waves_n=4, tile_k=256).validate()
    huge = rc.Op(rc.RC_OP_GEMM_I8, (1 << 20, 16000, 1024))
    assert huge.default().validate() == "" and "2^32 - 1 threads" in huge.schedule(splits=2).validate()
    # the ring: aligned rows, whole wave-loads, a depth of three, enough K
    # tiles where the MFMA steps of one are odd
    ring = dict(tile_m=64, tile_n=64, tile_k=128, waves_m=2, waves_n=2, stages=2)
    assert rc.Op(rc.RC_OP_GEMM_I8, (1000, 1000, 1008)).schedule(**ring).validate() == ""
    assert "multiple of 16" in op.schedule(**ring).validate()
    # or rows copied to whole chunks, which nothing else needs
    assert op.schedule(**ring, pad=1).validate() == ""
    assert "only the ring" in op.schedule(pad=1).validate()
    assert "multiple of 16 already" in rc.Op(rc.RC_OP_GEMM_I8, (1000, 1000, 1008)).schedule(**ring, pad=1).validate()
    tall = rc.Op(rc.RC_OP_GEMM_I8, ((1 << 30) - 64, 1, 65))
    assert "copying launch" in tall.schedule(**{**ring, "tile_n": 16, "waves_n": 1}, pad=1).validate()
    op = rc.Op(rc.RC_OP_GEMM_I8, (1000, 1000, 1024))
    assert "wave-loads" in op.schedule(**{**ring, "tile_m": 64, "waves_m": 4, "tile_n": 32, "tile_k": 64}).validate()
    assert "K tiles" in rc.Op(rc.RC_OP_GEMM_I8, (1000, 1000, 256)).schedule(**{**ring, "tile_k": 64}).validate()
    assert "ring stages" in op.schedule(tile_m=256, tile_n=256, tile_k=128, waves_m=4, waves_n=4, stages=2).validate()
    # streaming: one wave column, few rows, no splits over workgroups
    assert op.schedule(stages=3, waves_k=8).validate() == ""
    assert "one wave column" in op.schedule(stages=3, waves_n=2, tile_n=32).validate()
    assert "at most 64 rows" in op.schedule(stages=3, tile_m=128).validate()
    assert "over waves" in op.schedule(stages=3, splits=2).validate()
    assert "half of them" in op.schedule(stages=3, waves_k=16, tile_k=256).validate()
    assert "streaming stage (3) only" in op.schedule(waves_k=2).validate()
    # K splits of which none is empty; half-height tiles where they help
    assert op.schedule(splits=16).validate() == "" and "empty" in op.schedule(splits=16, tile_k=128).validate()
    wide = dict(tile_m=256, tile_n=128, tile_k=64, waves_m=2, waves_n=4, stages=2, tail=1)
    assert rc.Op(rc.RC_OP_GEMM_I8, (256, 128 * 300, 1024)).schedule(**wide).validate() == ""
    assert "no partial round" in rc.Op(rc.RC_OP_GEMM_I8, (256, 128 * 256, 1024)).schedule(**wide).validate()
    assert "need the ring" in op.schedule(tail=1).validate()
    small = rc.Op(rc.RC_OP_GEMM_I8, (1, 16, 64))
    assert "tile_m" in small.schedule(tile_m=32).validate()
    assert "tile_n" in small.schedule(tile_n=32).validate()
    assert "tile_k" in small.schedule(tile_k=128).validate()


def test_suggestions_share_few_code_objects():
    # sizes are kernel arguments: the suggestions over the whole range of
    # sizes are a handful of schedules, built ahead of time
    jobs = cases_i8.compile_jobs()
    # (the copying of rows is a code object of its own, pad 1 no other product)
    objects = {(o.kind, o.flags, str(s[0]).replace("pad=1", "pad=0")) for o, s in jobs}
    assert len(objects) < 900
    for m, n, k in ((1, 1, 1), (3, 5000, 77), (999, 12345, 11008), (100000, 64, 64), (1, 128256, 8192)):
        for flags in (0, B, F, B | F, G):
            op = rc.Op(rc.RC_OP_GEMM_I8, (m, n, k), flags)
            assert op.suggest().validate() == ""
            assert any(o.kind == op.kind and o.flags == flags and str(s[0]) == str(op.suggest()) for o, s in jobs), (m, n, k)
    for t, c in ((1, 1), (3, 5000), (5000, 3), (1, 128256), (2, 1 << 30), (1 << 22, 4096), (2 ** 26 - 1, 100)):
        op = rc.Op(rc.RC_OP_QUANT_I8, (t, c))
        assert any(o.kind == op.kind and str(s[0]) == str(op.suggest()) for o, s in jobs), (t, c)


def test_search_over_an_8_bit_operator():
    # the generic search runs over these kinds' knobs: with the tile area as
    # the reward it ends at the largest legal tile
    op = rc.Op(rc.RC_OP_GEMM_I8, (512, 512, 1024), G)
    s = rc.Search(op, lambda x: float(x["tile_m"] * x["tile_n"]), budget=150, seed=3).run()
    best, reward, _ = s.best()
    assert best.validate() == "" and reward >= 128 * 128
    assert all(h["schedule"].validate() == "" for h in s.history())


def test_kernels_do_not_depend_on_the_sizes():
    a, b = (rc.Op(rc.RC_OP_GEMM_I8, d) for d in ((500, 700, 300), (900, 1300, 4000)))
    text = cases_i8.GEMM_TEXTS[2]
    assert rc.kernel_defines(a, a.from_string(text)) == rc.kernel_defines(b, b.from_string(text))


def _tensors(op):
    want = rc._i8_tensors(op)
    return [[torch.zeros(shape, dtype=dtype) for _, dtype, shape in side] for side in want]


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_tensor_checks(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    want = rc._i8_tensors(op)
    ins, outs = _tensors(op)

    def check(i, o, device=-1, workspace=None):
        return rc._check_tensors(want, device, i, o, workspace, None)

    assert check(ins, tuple(outs)) == (ins, outs)
    if len(outs) == 1:
        assert check(iter(ins), outs[0]) == (ins, outs)
    with pytest.raises(ValueError, match="plan on cuda:0"):
        check(ins, outs, device=0)
    with pytest.raises(ValueError, match="inputs: the operator has"):
        check(ins[:-1], outs)
    with pytest.raises(ValueError, match="outputs: the operator has"):
        check(ins, outs + [outs[0]])
    for side, side_list in ((0, ins), (1, outs)):
        for j, (name, dtype, shape) in enumerate(want[side]):
            for bad in (None, torch.zeros(shape, dtype=torch.float64), torch.zeros((2,) + shape, dtype=dtype),
                        torch.zeros(shape[:-1] + (shape[-1] + 1,), dtype=dtype),
                        torch.zeros(shape + (2,), dtype=dtype)[..., 0]):
                sides = [list(ins), list(outs)]
                sides[side][j] = bad
                with pytest.raises(ValueError, match=f"{name} must be"):
                    check(*sides)


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_packed_block_is_the_structure(kind, dims, flags, monkeypatch):
    op = rc.Op(kind, dims, flags)
    want = rc._i8_tensors(op)
    ins, outs = _tensors(op)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    pack = rc._i8_packer(want, -1)
    assert pack(ins, tuple(outs), None, None) == (bytes(rc.Plan._args(ins, outs)), 0)
    if len(outs) == 1:
        assert pack(iter(ins), outs[0], None, None) == (bytes(rc.Plan._args(ins, outs)), 0)
    for bad in ((ins[:-1], outs), (ins, outs[:-1]), (ins + outs, ()), (ins, outs + [outs[0]]), ([None] + ins[1:], outs),
                ([ins[0].double()] + ins[1:], outs), (ins, [outs[0][:-1]] + outs[1:])):
        with pytest.raises(ValueError):
            pack(bad[0], bad[1], None, None)
    with pytest.raises(ValueError):
        rc._i8_packer(want, 0)(ins, outs, None, None)


def test_argument_block_of_several_outputs():
    class Tensor:
        def __init__(self, p):
            self.p = p

        def data_ptr(self):
            return self.p

    outs = tuple(Tensor(4096 * (i + 1)) for i in range(4))
    ins = [Tensor(16 * i) for i in range(3)]
    for n in range(1, 5):
        assert rc._pack_args(ins, outs[:n]) == bytes(rc.Plan._args(ins, outs[:n]))
    with pytest.raises(IndexError):
        rc._pack_args(ins, outs + outs[:1])
