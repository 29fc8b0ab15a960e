"""GPU tests of how attention in serving cuts keys into pieces: how long the pieces
are, many sequences of which few are cut, and the pieces' states in every kind of
workspace.  References and bounds are those of test_gpu_seqs."""
import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_seqs as S
from cases_seqs import C
from test_gpu_seqs import _gpu, check, f64, ints, keys_of, paged_inputs, reference, starts  # noqa: F401

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

UNUSED = 0x7FC12345            # a NaN that no state holds


def states_left(op, text, rows, cache, where, out):
    """How many pieces' states a launch leaves in its workspace."""
    print(f"[gpu] paged dims={op.dims} flags={op.flags} sched={text}", flush=True)
    plan = rc.Plan(op, op.from_string(text))
    ws = plan.workspace()
    ws.view(torch.int32).fill_(UNUSED)
    plan.launch([x.cuda() for x in [rows] + cache + where], out, ws)
    torch.cuda.synchronize()
    at, n = plan.buffer("partials")
    size = op.from_string(text)["block_m"] * (op.dims[4] + 2) * 4
    return int((ws[at:at + n].view(torch.int32)[::size // 4] != UNUSED).sum())


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
    out = torch.empty_like(rows, device="cuda")
    made = states_left(op, text, rows, cache, [ints(starts(case[0])), ints(lens), ints(table)], out)
    check(out, want, tol)
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
    out = torch.empty_like(rows, device="cuda")
    made = states_left(op, text, rows, cache, [ints(starts(case[0])), ints(lens), ints(table)], out)
    check(out, want, tol)
    assert made >= 8 * 8 * -(-128 // longest_piece([-(-n // 64) for n in lens], 8, 256, 16))
