"""CPU tests of attention in serving: descriptors, refusals, schedules and their
legality, the work model, and the checks of a launch's buffers."""
import ctypes
import math

import pytest

from paper_2506_01374_amd import rc

import cases_seqs as S
from cases_seqs import C, I8

W, RD, PG, PK = rc.RC_OP_KV_WRITE, rc.RC_OP_KV_READ, rc.RC_OP_ATTENTION_PAGED, rc.RC_OP_ATTENTION_PACKED
KINDS = [(W, (7, 3, 2, 64, 16, 9, 5), 0), (W, (7, 3, 2, 64, 16, 9, 5), I8), (RD, (7, 3, 2, 128, 32, 9, 5), 0),
         (RD, (7, 3, 2, 128, 32, 9, 5), I8), (PG, (7, 3, 6, 2, 64, 16, 9, 5), 0), (PG, (7, 3, 6, 2, 128, 16, 9, 5), C),
         (PG, (7, 3, 6, 2, 256, 64, 9, 5), I8), (PG, (7, 3, 6, 2, 64, 256, 9, 5), I8 | C), (PK, (7, 30, 3, 6, 2, 64), 0),
         (PK, (70, 30, 3, 6, 2, 128), C)]


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_descriptor_and_schedules(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    assert op.default().validate() == "" and op.suggest().validate() == ""
    for i, name in enumerate(op.knob_names()):
        assert op.default().raw.knob[i] == min(op.knob_values(i)), name
        assert op.knob_class(i) in ("TileSize", "Parallel", "Vectorize", "Unroll", "ComputeLocation", "Layout")
    for t in op.default().moves():
        assert op.default().apply(t).validate() == ""
    with pytest.raises(ValueError):
        rc.Op(kind, dims, flags, eps=1e-6)


@pytest.mark.parametrize("kind,dims,flags,status", [
    (W, (0, 3, 2, 64, 16, 9, 5), 0, rc.RC_ERR_INVALID_ARGUMENT), (W, (7, 3, 2, 64, 16, 9), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (W, (7, 3, 2, 64, 16, 9, 5), C, rc.RC_ERR_INVALID_ARGUMENT), (W, (7, 3, 2, 96, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (W, (7, 3, 2, 64, 24, 9, 5), 0, rc.RC_ERR_UNSUPPORTED), (W, (7, 3, 2, 64, 512, 9, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (RD, (7, 3, 2, 64, 16, 9, 2 ** 27), 0, rc.RC_ERR_UNSUPPORTED), (RD, (2 ** 30, 3, 2, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (RD, (7, 3, 2 ** 15, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED), (RD, (7, 2 ** 25, 2, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (RD, (7, 3, 2, 64, 16, 2 ** 31, 5), 0, rc.RC_ERR_UNSUPPORTED), (RD, (7, 3, 2, 64, 16, 2 ** 62, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (RD, (2 ** 62, 3, 2, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED), (RD, (7, 3, 2, 64, 16, 9, 2 ** 62), 0, rc.RC_ERR_UNSUPPORTED),
    (PG, (7, 3, 5, 2, 64, 16, 9, 5), 0, rc.RC_ERR_INVALID_ARGUMENT), (PG, (7, 3, 1, 2, 64, 16, 9, 5), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (PG, (7, 3, 6, 2, 32, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED), (PG, (2 ** 28, 3, 8, 2, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED),
    (PG, (7, 3, 6, 2, 64, 16, 9, 5), 2, rc.RC_ERR_INVALID_ARGUMENT), (PG, (7, 3, 6, 2, 64, 16, 0, 5), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (PG, (7, 2 ** 24, 8, 4, 64, 16, 9, 5), 0, rc.RC_ERR_UNSUPPORTED), (PK, (7, 7, 2 ** 24, 8, 4, 64), 0, rc.RC_ERR_UNSUPPORTED),
    (PK, (7, 30, 3, 6, 2, 64), I8, rc.RC_ERR_INVALID_ARGUMENT), (PK, (7, 30, 3, 6, 4, 64), 0, rc.RC_ERR_INVALID_ARGUMENT),
    (PK, (7, 0, 3, 6, 2, 64), 0, rc.RC_ERR_INVALID_ARGUMENT), (PK, (7, 2 ** 30, 3, 6, 2, 64), 0, rc.RC_ERR_UNSUPPORTED),
    (rc.RC_OP_GEMM_I8, (8, 8, 8), I8, rc.RC_ERR_INVALID_ARGUMENT), (rc.RC_OP_ATTENTION, (1, 1, 64, 64), I8, rc.RC_ERR_INVALID_ARGUMENT)])
def test_refused_descriptors(kind, dims, flags, status):
    with pytest.raises(rc.RCError) as e:
        rc.Op(kind, dims, flags)
    assert e.value.status == status


def test_a_descriptor_made_by_hand_is_checked_too():
    op = rc.Op(PG, (7, 3, 6, 2, 64, 16, 9, 5))
    sched = op.suggest()
    op.desc.dim[5] = 24
    s = rc.rc_schedule()
    assert rc.lib().rc_default_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    assert rc.lib().rc_suggest_schedule(op.ref, ctypes.byref(s)) == rc.RC_ERR_UNSUPPORTED
    assert "pages hold" in sched.validate()


def test_work_model():
    w = rc.Op(W, (10, 2, 3, 64, 16, 9, 5))
    where = 4 * 3 + 4 * 2 * 6
    assert w.flops() == 0 and w.bytes() == 10 * 3 * 64 * 8 + where
    assert rc.Op(RD, (10, 2, 3, 64, 16, 9, 5), I8).bytes() == 10 * 3 * (64 * 4 + 64 * 2 + 8) + where
    p = rc.Op(PG, (10, 2, 6, 3, 64, 16, 9, 5))
    assert p.flops() == 4 * 64 * 6 * 10 * 80 and p.bytes() == 10 * 6 * 64 * 4 + 2 * 80 * 3 * 256 + where
    assert rc.Op(PG, (10, 2, 6, 3, 64, 16, 9, 5), C).flops() == 4 * 64 * 6 * 2 * sum(range(76, 81))
    k = rc.Op(PK, (10, 10, 1, 6, 3, 64), C)
    assert k.flops() == 4 * 64 * 6 * 55 and k.bytes() == 10 * 9 * 64 * 4 + 16
    assert p.peak_flops() == 2516.6e12 and p.bound() == "hbm"


def test_legality():
    op = rc.Op(PG, (1, 1, 16, 1, 128, 16, 9, 5))
    assert "already covers" in op.schedule(block_m=32).validate()
    op = rc.Op(PG, (100, 1, 16, 1, 128, 16, 9, 5))
    assert op.schedule(block_m=32).validate() == ""
    assert "LDS" in rc.Op(PG, (100, 1, 16, 1, 64, 16, 9, 5)).schedule(block_m=128, waves=8).validate()
    assert "registers" in rc.Op(PG, (100, 1, 16, 1, 256, 16, 9, 5)).schedule(block_m=32).validate()
    huge = rc.Op(PG, (2 ** 26 - 64, 1, 16, 16, 64, 16, 9, 5))
    assert huge.default().validate() == "" and "2^32 - 1 threads" in huge.schedule(waves=2).validate()
    assert "already cover" in rc.Op(W, (1, 1, 1, 64, 16, 9, 5)).schedule(waves=2).validate()
    many = rc.Op(PG, (4000, 2049, 16, 16, 64, 16, 9, 500))
    assert many.suggest().as_dict()["splits"] == 0 and "2049, more than 2048" in many.schedule(splits=1).validate()
    # a sequence without rows has an index where there are many
    empty = rc.Op(PG, (1, 2 ** 22, 8, 8, 64, 16, 9, 5))
    assert empty.suggest().validate() == "" and "2^32 - 1 threads" in empty.schedule(waves=4).validate()


@pytest.mark.parametrize("kind,flags", [(W, 0), (W, I8), (RD, 0), (RD, I8), (PG, 0), (PG, C), (PG, I8), (PG, I8 | C), (PK, 0), (PK, C)])
def test_every_suggestion_is_listed(kind, flags):
    listed = rc.suggestions(kind, flags)
    at = {PG: 4, PK: 5}.get(kind, 3)
    texts = {(op.dims[at], str(s)) for op, s in listed}
    assert len(texts) == len(listed) <= 60
    for op, s in listed:
        assert op.kind == kind and op.flags == flags and s.validate() == ""
    for d in (64, 128, 256):
        for t in (1, 2, 3, 4, 5, 16, 17, 64, 100, 512, 777, 4000, 16384, 2 ** 20):
            for b in (1, 2, 15, 16, 64, 128, 1000):
                for hkv, g in ((1, 1), (1, 16), (2, 3), (8, 4), (8, 1), (4, 7)):
                    for page, width in ((16, 1), (16, 20), (64, 600), (256, 4096)):
                        dims = {PG: (t, b, hkv * g, hkv, d, page, 100, width), PK: (t, t + width, b, hkv * g, hkv, d)}.get(
                            kind, (t, b, hkv, d, page, 100, width))
                        assert (d, str(rc.Op(kind, dims, flags).suggest())) in texts, dims


def test_suggestions_of_bad_kinds_are_refused():
    for kind, flags, status in ((PG, 2, rc.RC_ERR_INVALID_ARGUMENT), (13, 0, rc.RC_ERR_UNSUPPORTED)):
        with pytest.raises(rc.RCError) as e:
            rc.suggestions(kind, flags)
        assert e.value.status == status


def test_kernels_do_not_depend_on_the_sizes():
    a, b = rc.Op(PG, (7, 3, 6, 2, 64, 16, 9, 5), C), rc.Op(PG, (700, 30, 20, 4, 64, 256, 90, 50))
    text = "block_m=32,waves=2,splits=1"
    assert rc.kernel_defines(a, a.from_string(text)) == rc.kernel_defines(b, b.from_string(text))


def test_search():
    op = rc.Op(PG, (64, 64, 32, 8, 128, 16, 5000, 100), C)
    s = rc.Search(op, lambda x: float(x["block_m"] * x["waves"]), budget=30, seed=3).run()
    best, reward, _ = s.best()
    assert best.validate() == "" and all(h["schedule"].validate() == "" for h in s.history())


# ---------------------------------------------------------------------------
# The checks of a launch
# ---------------------------------------------------------------------------

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_tensor_checks(kind, dims, flags, monkeypatch):
    op = rc.Op(kind, dims, flags)
    want = rc._i8_tensors(op)
    ins, outs = ([torch.zeros(shape, dtype=dtype) for _, dtype, shape in side] for side in want)

    def check(i, o, device=-1):
        return rc._check_tensors(want, device, i, o, None, None)

    assert check(ins, tuple(outs)) == (ins, outs)
    with pytest.raises(ValueError, match="plan on cuda:0"):
        check(ins, outs, device=0)
    with pytest.raises(ValueError, match="inputs: the operator has"):
        check(ins[:-1], outs)
    for side, side_list in ((0, ins), (1, outs)):
        for j, (name, dtype, shape) in enumerate(want[side]):
            for bad in (None, torch.zeros(shape, dtype=torch.float64), torch.zeros((2,) + shape, dtype=dtype),
                        torch.zeros(shape[:-1] + (shape[-1] + 1,), dtype=dtype),
                        torch.zeros(shape + (2,), dtype=dtype)[..., 0]):
                sides = [list(ins), list(outs)]
                sides[side][j] = bad
                with pytest.raises(ValueError, match=f"{name} must be"):
                    check(*sides)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    assert rc._i8_packer(want, -1)(ins, tuple(outs), None, None) == (bytes(rc.Plan._args(ins, outs)), 0)


def checked(op, ins, outs, ws=None, ws_bytes=0):
    a = rc.rc_args()
    a.struct_size = ctypes.sizeof(rc.rc_args)
    for i, p in enumerate(ins):
        a.in_[i] = p
    for i, p in enumerate(outs):
        a.out[i] = p
    st = rc.lib().rc_check_args(op.ref, ctypes.byref(a), ws, ws_bytes)
    return st, rc.lib().rc_last_error().decode() if st else ""


@pytest.mark.parametrize("kind,dims,flags", KINDS)
def test_what_a_launch_writes_overlaps_nothing(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    size = {"torch.int8": 1, "torch.bfloat16": 2, "torch.float32": 4, "torch.int32": 4}
    sizes = [[size[str(dtype)] * math.prod(shape) for _, dtype, shape in side] for side in rc._i8_tensors(op)]
    at, places = 1 << 20, []
    for n in sizes[0] + sizes[1] + [512]:
        places.append(at)
        at += -(-n // 256) * 256
    ni, no = len(sizes[0]), len(sizes[1])
    ins, outs, ws = places[:ni], places[ni:ni + no], places[-1]
    assert checked(op, ins, outs, ws, 512) == (rc.RC_OK, "")
    assert checked(op, [ins[0]] * ni, outs, ws, 512) == (rc.RC_OK, "")
    for o in range(no):
        for i in range(ni):
            moved = list(outs)
            for p in (ins[i], ins[i] + (sizes[0][i] - 1) // 16 * 16, ins[i] - (sizes[1][o] - 1) // 16 * 16):
                moved[o] = p
                st, why = checked(op, ins, moved, ws, 512)
                assert st == rc.RC_ERR_INVALID_ARGUMENT and "overlaps" in why
            far = list(ins)
            far[i] = 1 << 30
            moved[o] = far[i] + -(-sizes[0][i] // 16) * 16
            assert checked(op, far, moved, ws, 512)[0] == rc.RC_OK
        for i in range(no):
            if i != o:
                moved = list(outs)
                moved[o] = outs[i]
                assert checked(op, ins, moved, ws, 512)[0] == rc.RC_ERR_INVALID_ARGUMENT
        assert checked(op, ins, outs, outs[o], 512)[0] == rc.RC_ERR_INVALID_ARGUMENT
    for i in range(ni):
        assert checked(op, ins, outs, ins[i] + (sizes[0][i] - 1) // 256 * 256, 512)[0] == rc.RC_ERR_INVALID_ARGUMENT
        for bad, status in ((0, rc.RC_ERR_INVALID_ARGUMENT), (ins[i] + 8, rc.RC_ERR_MISALIGNED)):
            assert checked(op, ins[:i] + [bad] + ins[i + 1:], outs, ws, 512)[0] == status
