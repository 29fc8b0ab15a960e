"""GPU tests of how attention in serving cuts keys into pieces: how long the pieces
are, many sequences of which few are cut, and pieces in the library's own workspace.

References and bounds are those of test_gpu_seqs, with a term more for the ring over
bf16 (stages=3), where the sum of p is that of the rounded p too: with roundings d_j of
p_j, sum p_j (1 + d_j) v_j / sum p_j (1 + d_j) differs from the result by sum p_j d_j (v_j
- out) / sum p_j, at most 2^-8 (A + |out|) and not 2^-8 A, to first order; what is of
second order is below 2^-7 of that."""
import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_seqs as S
from cases_seqs import C, I8
from test_gpu_seqs import BF16, _gpu, check, f64, ints, keys_of, paged_inputs, reference, starts  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

UNUSED = 0x7FC12345            # a NaN that no state holds


def run_cut(op, text, rows, cache, where):
    """(result, how many pieces' states a launch leaves in its workspace); what is
    behind the workspace stays as it was."""
    print(f"[gpu] paged dims={op.dims} flags={op.flags} sched={text}", flush=True)
    sched = op.from_string(text)
    assert sched.validate() == ""
    plan = rc.Plan(op, sched)
    n = plan.workspace_bytes
    ws = torch.full((n // 4 + 1024,), UNUSED, dtype=torch.int32, device="cuda")
    out = torch.full(tuple(rows.shape), float("nan"), dtype=torch.bfloat16, device="cuda")
    plan.launch([x.cuda() for x in [rows] + cache + where], out, ws[:n // 4])
    torch.cuda.synchronize()
    assert bool((ws[n // 4:] == UNUSED).all())
    at, n = plan.buffer("partials")
    size = sched["block_m"] * (op.dims[4] + 2)
    return out, int((ws[at // 4:(at + n) // 4:size] != UNUSED).sum())


def check_cut(got, op, text, want, tol):
    ring = op.from_string(text)["stages"] == 3 and not op.flags & I8
    check(got, want, tol + (1.01 * BF16 * np.abs(want) if ring else 0))


def longest_piece(tiles, hkv, groups, least):
    """Twice what all tiles, and five for the start and end of a workgroup, are over
    the workgroups."""
    return 2 * max(least, -(-(sum(tiles) + 5 * len(tiles)) * hkv // groups))


@pytest.mark.parametrize("at", [0, 50, 99])
@pytest.mark.parametrize("longest", [16384, 5000])
def test_a_long_sequence_among_many_short_ones_is_cut(longest, at):
    # 99 sequences of two tiles, whose blocks and heads are more than a round of
    # workgroups
    lens = [128] * 100
    lens[at] = longest
    case = ([5] * 100, lens, 4, 4, 128, 64)
    op = S.paged_op(case, C)
    text = str(op.suggest())
    k = op.suggest().as_dict()
    assert (k["stages"], k["splits"], k["block_m"], k["waves"]) == (3, 1, 64, 8)
    rows, cache, table = paged_inputs(case, 0, 80)
    keys, _ = keys_of(cache, table, lens, 64, 0)
    want, tol = reference(case[0], lens, f64(rows), keys, True, 128 ** -0.5)
    out, made = run_cut(op, text, rows, cache, [ints(starts(case[0])), ints(lens), ints(table)])
    check_cut(out, op, text, want, tol)
    tiles = [-(-n // 64) for n in lens]
    assert made % 4 == 0 and made // 4 >= -(-max(tiles) // longest_piece(tiles, 4, 256, 16))


def test_some_long_sequences_among_many_short_ones_are_cut():
    lens = [256] * 63
    lens[3::8] = [8192] * 8
    case = ([5] * 63, lens, 8, 4, 128, 64)
    op = S.paged_op(case, C)
    text = str(op.suggest())
    rows, cache, table = paged_inputs(case, 0, 81)
    keys, _ = keys_of(cache, table, lens, 64, 0)
    want, tol = reference(case[0], lens, f64(rows), keys, True, 128 ** -0.5)
    out, made = run_cut(op, text, rows, cache, [ints(starts(case[0])), ints(lens), ints(table)])
    check_cut(out, op, text, want, tol)
    assert made >= 8 * 8 * -(-128 // longest_piece([-(-n // 64) for n in lens], 8, 256, 16))


@pytest.mark.parametrize("few", [True, False])
@pytest.mark.parametrize("b", [65, 257, 1000, 2048])
def test_few_of_many_sequences_are_cut(b, few):
    # long ones first, last, in the middle and on either side of 64; the states of
    # all lie behind each other.  With rows of every 40th sequence alone, the direct
    # kernel's pieces are joined by rows, else by blocks
    r = np.random.default_rng(b)
    long = sorted({0, 63, 64, b // 2, b - 1})
    q = [3 if not few else 0 if i % 40 else 1 for i in range(b)]
    lens = [int(n) for n in r.integers(1, 80, b)]
    for i, at in enumerate(long):
        q[at], lens[at] = 1 + i, 3000 + 517 * i
    q[long[2]] = 40
    case = (q, lens, 2, 4, 64, 64)
    for flags in (C, I8 | C):
        op = S.paged_op(case, flags)
        rows, cache, table = paged_inputs(case, flags & I8, 90)
        keys, _ = keys_of(cache, table, lens, 64, flags & I8)
        want, tol = reference(q, lens, f64(rows), keys, True, 64 ** -0.5)
        assert (sum(q) * 8 <= 1536) == few
        for text in ("waves=4,splits=2", "block_m=32,waves=2,splits=1", "block_m=64,waves=8,stages=3,occ=2,splits=4",
                     "block_m=128,waves=4,stages=3,occ=2,splits=2"):
            got, made = run_cut(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)])
            check_cut(got, op, text, want, tol)
            blocks = sum(-(-q[i] * 4 // op.from_string(text)["block_m"]) for i in long)
            assert made >= 2 * 2 * blocks


def test_pieces_in_the_library_s_own_workspace():
    case = ([1, 1, 30, 1, 1, 1], [3000, 1, 500, 64, 2000, 77], 2, 4, 128, 16)
    q, lens = case[:2]
    for flags in (C, I8 | C):
        op = S.paged_op(case, flags)
        rows, cache, table = paged_inputs(case, flags & I8, 95)
        where = [ints(starts(q)), ints(lens), ints(table)]
        ins = [x.cuda() for x in [rows] + cache + where]
        for text in ("waves=4,splits=2", "block_m=64,waves=8,stages=3,occ=2,splits=1"):
            want, made = run_cut(op, text, rows, cache, where)
            plan = rc.Plan(op, op.from_string(text))
            assert made > 0 and 0 < plan.workspace_bytes <= rc.lib().rc_static_scratch_bytes()
            for _ in range(2):
                got = torch.full_like(want, float("nan"))
                plan.launch_static(ins, got)
                torch.cuda.synchronize()
                assert torch.equal(got, want)
        # more than the library keeps
        plan = rc.Plan(op, op.from_string("block_m=128,waves=4,stages=3,occ=2,splits=4"))
        assert plan.workspace_bytes > rc.lib().rc_static_scratch_bytes()
        with pytest.raises(rc.RCError) as e:
            plan.launch_static(ins, got)
        assert e.value.status == rc.RC_ERR_OUT_OF_MEMORY and "use rc_launch" in str(e.value)
