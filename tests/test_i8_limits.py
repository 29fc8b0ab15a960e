"""CPU tests of the 8-bit integer operators at and past the ends of their
ranges."""
import ctypes
import math
import random

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


# ---------------------------------------------------------------------------
# Buffers that overlap
# ---------------------------------------------------------------------------

def operand_bytes(op):
    """Bytes of each input and each output."""
    size = {"torch.int8": 1, "torch.bfloat16": 2, "torch.float32": 4}
    return [[size[str(dtype)] * math.prod(shape) for _, dtype, shape in side] for side in rc._i8_tensors(op)]


def checked(op, ins, outs, ws=None, ws_bytes=0):
    a = rc.rc_args()
    a.struct_size = ctypes.sizeof(rc.rc_args)
    for i, p in enumerate(ins):
        a.in_[i] = p
    for i, p in enumerate(outs):
        a.out[i] = p
    st = rc.lib().rc_check_args(op.ref, ctypes.byref(a), ws, ws_bytes)
    return st, rc.lib().rc_last_error().decode() if st else ""


OVERLAP_KINDS = [(rc.RC_OP_RMSNORM_I8, (5, 64), 0), (rc.RC_OP_RMSNORM_I8, (5, 64), R), (rc.RC_OP_QUANT_I8, (5, 64), 0)] + [
    (rc.RC_OP_GEMM_I8, (4, 16, 32), f) for f in (0, B, F, B | F, G)]


@pytest.mark.parametrize("kind,dims,flags", OVERLAP_KINDS)
def test_what_a_launch_writes_overlaps_nothing(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    sizes = operand_bytes(op)
    # all operands side by side, each at a multiple of 256 bytes, then a workspace
    at, places = 1 << 20, []
    for n in sizes[0] + sizes[1] + [512]:
        places.append(at)
        at += -(-n // 256) * 256
    ni, no = len(sizes[0]), len(sizes[1])
    ins, outs, ws = places[:ni], places[ni:ni + no], places[-1]
    assert checked(op, ins, outs, ws, 512) == (rc.RC_OK, "")
    assert checked(op, ins, outs) == (rc.RC_OK, "")
    # inputs may share memory
    assert checked(op, [ins[0]] * ni, outs, ws, 512) == (rc.RC_OK, "")
    for o in range(no):
        for i in range(ni):
            moved = list(outs)
            # the output's first chunk, and its last, on the input's last and first
            for p in (ins[i], ins[i] + (sizes[0][i] - 1) // 16 * 16, ins[i] - (sizes[1][o] - 1) // 16 * 16):
                moved[o] = p
                st, why = checked(op, ins, moved, ws, 512)
                allowed = kind == rc.RC_OP_RMSNORM_I8 and o == 2 and i != 1 and p == ins[i]
                if allowed:
                    assert st == rc.RC_OK
                else:
                    assert st == rc.RC_ERR_INVALID_ARGUMENT and "overlaps" in why
            # next to it is no overlap: a lone pair of buffers far from the rest
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
        assert checked(op, ins, outs, ins[i], 512)[0] == rc.RC_ERR_INVALID_ARGUMENT
        assert checked(op, ins, outs, ins[i] + (sizes[0][i] - 1) // 256 * 256, 512)[0] == rc.RC_ERR_INVALID_ARGUMENT


def test_pointer_checks_need_no_device():
    op = rc.Op(rc.RC_OP_QUANT_I8, (5, 64))
    assert checked(op, [4096], [8192, 0])[0] == rc.RC_ERR_INVALID_ARGUMENT
    assert checked(op, [4096 + 8], [8192, 12288])[0] == rc.RC_ERR_MISALIGNED
    assert checked(op, [4096], [8192, 12288], 16384 + 16, 64)[0] == rc.RC_ERR_MISALIGNED
    # the kinds whose sizes are not held against each other keep their checks
    op = rc.Op(rc.RC_OP_GEMM_F32, (8, 8, 8))
    assert checked(op, [4096, 4096], [4096])[0] == rc.RC_OK
    assert checked(op, [4096, 0], [4096])[0] == rc.RC_ERR_INVALID_ARGUMENT


def test_a_workspace_of_fewer_bytes_than_elements_is_refused():
    torch = pytest.importorskip("torch")
    op = rc.Op(rc.RC_OP_GEMM_I8, (4, 16, 32))
    want = rc._i8_tensors(op)
    ins, outs = ([torch.zeros(shape, dtype=dtype) for _, dtype, shape in side] for side in want)
    whole = torch.empty(4096, dtype=torch.uint8)
    assert rc._check_tensors(want, -1, ins, outs, whole, None) == (ins, outs)
    for ws in (torch.empty(1, dtype=torch.uint8).expand(4096), whole[::2]):
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            rc._check_tensors(want, -1, ins, outs, ws, None)
        with pytest.raises(ValueError, match="workspace must be contiguous"):
            rc._i8_packer(want, -1)(ins, outs, ws, None)


# ---------------------------------------------------------------------------
# The list of suggested schedules
# ---------------------------------------------------------------------------

SUGGESTING = [(rc.RC_OP_QUANT_I8, 0), (rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)] + [
    (rc.RC_OP_GEMM_I8, f) for f in (0, B, F, B | F, G)]


def some_sizes(kind, seed):
    """Sizes over the whole range, and next to powers of two."""
    g = random.Random(seed)
    most = (2 ** 26 - 1, 1 << 30) if kind != rc.RC_OP_GEMM_I8 else (1 << 20, 1 << 18, 131071)
    for _ in range(4000):
        yield tuple(max(1, int(2 ** g.uniform(0, math.log2(m)))) for m in most)
        yield tuple(min(m, max(1, 2 ** g.randint(0, m.bit_length()) + g.choice((-1, 0, 1)))) for m in most)
        if kind == rc.RC_OP_GEMM_I8:
            # what is served: few to some thousand rows, and weights
            yield tuple(max(1, int(2 ** g.uniform(0, math.log2(m)))) // s * s or s
                        for m, s in zip((5000, 32768, 32768), (1, g.choice((1, 16)), g.choice((1, 4, 16)))))


@pytest.mark.parametrize("kind,flags", SUGGESTING)
def test_every_suggestion_is_listed(kind, flags):
    listed = rc.suggestions(kind, flags)
    texts = {str(s) for _, s in listed}
    assert len(texts) == len(listed) <= 160
    for op, s in listed:
        assert op.kind == kind and op.flags == flags and s.validate() == ""
    if kind == rc.RC_OP_GEMM_I8:
        assert sum(s["pad"] for _, s in listed) == 1
    sizes = list(some_sizes(kind, 11 * kind + flags))
    if kind == rc.RC_OP_GEMM_I8:
        sizes += [(23, 1915, 1656), (20, 4668, 1188), (70400, 64, 352)]
    for dims in sizes:
        if kind == rc.RC_OP_GEMM_I8 and -(-dims[0] // 16) * -(-dims[1] // 16) > 2 ** 26 - 1:
            continue
        text = str(rc.Op(kind, dims, flags).suggest())
        assert text.replace("pad=1", "pad=0") in texts, dims


def test_the_list_of_suggestions_is_of_the_8_bit_kinds():
    for kind, flags, status in ((rc.RC_OP_GEMM_F32, 0, rc.RC_ERR_UNSUPPORTED), (99, 0, rc.RC_ERR_UNSUPPORTED),
                                (rc.RC_OP_GEMM_I8, R, rc.RC_ERR_INVALID_ARGUMENT),
                                (rc.RC_OP_GEMM_I8, G | B, rc.RC_ERR_INVALID_ARGUMENT)):
        with pytest.raises(rc.RCError) as e:
            rc.suggestions(kind, flags)
        assert e.value.status == status
    n = ctypes.c_int32()
    assert rc.lib().rc_suggestions(rc.RC_OP_QUANT_I8, 0, None, None, 1, ctypes.byref(n)) == rc.RC_ERR_INVALID_ARGUMENT
    assert rc.lib().rc_suggestions(rc.RC_OP_QUANT_I8, 0, None, None, 0, None) == rc.RC_ERR_INVALID_ARGUMENT


def test_k_splits_share_their_code_objects():
    # the sums of the splits are those of every epilogue, and their join that
    # of every tile
    texts = ["tile_m=64,tile_n=64,tile_k=128,waves_m=2,waves_n=2,stages=2,splits=2", "tile_m=32,tile_n=32,tile_k=64,stages=1,splits=2"]
    split, join = {}, {}
    for flags in (0, B, F, B | F, G):
        for i, text in enumerate(texts):
            op = rc.Op(rc.RC_OP_GEMM_I8, (200, 300, 1024), flags)
            for found, at, key in ((split, 0, (i, flags & G)), (join, 1, flags)):
                got = rc.kernel_defines(op, op.from_string(text), at)
                assert found.setdefault(key, got) == got
    assert {(int(d["BIAS"]), int(d["F32"]), int(d["GATED"])) for d in join.values()} == {
        (int(bool(f & B)), int(bool(f & F)), int(bool(f & G))) for f in (0, B, F, B | F, G)}
