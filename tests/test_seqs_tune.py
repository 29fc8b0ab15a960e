"""Tuning of attention in serving: workloads, inputs, features and a search, on the
CPU with a made-up timing and on the GPU with the real one."""
import os

import numpy as np
import pytest

from paper_2506_01374_amd import rc, tune, workloads as W

from cases_seqs import C, I8

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OPS = [(rc.RC_OP_KV_WRITE, (37, 3, 2, 64, 16, 20, 5), 0), (rc.RC_OP_KV_WRITE, (37, 3, 2, 64, 16, 20, 5), I8),
       (rc.RC_OP_KV_READ, (37, 3, 2, 64, 16, 12, 5), 0), (rc.RC_OP_KV_READ, (37, 3, 2, 64, 16, 12, 5), I8),
       (rc.RC_OP_ATTENTION_PAGED, (37, 3, 6, 2, 64, 16, 12, 5), 0), (rc.RC_OP_ATTENTION_PAGED, (37, 3, 6, 2, 64, 16, 20, 5), C | I8),
       (rc.RC_OP_ATTENTION_PACKED, (37, 90, 3, 6, 2, 64), 0), (rc.RC_OP_ATTENTION_PACKED, (37, 37, 3, 6, 2, 64), C)]


def cpu_inputs(op, seed):
    return W.to_device(W.stored_inputs(op, op.default(), W.host_inputs(op, seed=seed)), device="cpu")


@pytest.mark.parametrize("kind,dims,flags", OPS)
def test_inputs_and_outputs_are_those_of_a_launch(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    ins, outs = cpu_inputs(op, 3), W.empty_output(op, device="cpu")
    rc._check_tensors(rc._i8_tensors(op), -1, ins, outs, None, None)
    assert all(torch.equal(x, y) for x, y in zip(ins, cpu_inputs(op, 3)))
    for x, y in zip(ins, cpu_inputs(op, 4)):
        assert torch.equal(x, y) == (x.dtype == torch.int32)
    arrays = W.output_to_f64(op, outs)
    assert len(arrays) == len(outs) if isinstance(outs, tuple) else arrays.shape == tuple(ins[0].shape)
    # what a launch needs: offsets over all rows, no slot of two sequences
    assert ins[-3 if kind != rc.RC_OP_ATTENTION_PACKED else -2].tolist()[::3] == [0, 37]
    if kind != rc.RC_OP_ATTENTION_PACKED:
        held = ins[-1][ins[-1] >= 0].tolist()
        assert len(set(held)) == len(held) and max(held) < dims[-2]
        assert ins[-1].min() == (-1 if dims[-2] < 15 else 0)


@pytest.mark.parametrize("name", list(W.SEQS_WORKLOADS))
def test_workloads_have_a_reference_schedule(name):
    op = W.workload_op(name)
    assert op.from_string(tune.reference_schedule(name)).validate() == ""
    assert name not in W.WORKLOADS and name not in W.I8_WORKLOADS


def test_features_of_schedules():
    for kind, dims, flags in OPS:
        op = rc.Op(kind, dims, flags)
        found = [tune.schedule_features(op, s) for s in tune.random_walk_space(op, 12, seed=1)]
        assert len({len(f) for f in found}) == 1 and len(found[0]) > len(op.knob_names())
        assert np.all(np.isfinite(found))


@pytest.mark.parametrize("proposer,surrogate", [(None, False), ("model_repair", True)])
def test_a_search_with_a_made_up_timing(proposer, surrogate):
    op = rc.Op(rc.RC_OP_ATTENTION_PAGED, (512, 8, 32, 8, 128, 64, 300, 32), C)

    def timed(s):
        return {"schedule": str(s), "valid": True, "ms": 1.0 / s["block_m"], "reward": s["block_m"] / 128}

    ev = tune.ParallelGpuEvaluator(op, time_fn=timed, compile_fn=lambda job: 0)
    res = tune.run_search(op, ev, "uct", budget=40, seed=1, proposer=proposer, surrogate=surrogate)
    ev.close()
    assert res["valid"] > 1 and op.from_string(res["best"]).validate() == "" and res["best_reward"] >= 0.25


def test_the_command_lists_walks(tmp_path):
    name = "attention_paged_b64_h32_kv8_d128_l2048"
    tune.main(["--workload", name, "--walks", "5", "--out", str(tmp_path)])
    lines = open(tmp_path / f"{name}.space.txt").read().split()
    op = W.workload_op(name)
    assert len(lines) == 5 and all(op.from_string(t).validate() == "" for t in lines)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dims,flags", OPS)
def test_a_search_on_the_gpu_measures_launches_that_are_right(kind, dims, flags):
    from test_gpu_seqs import check, f64, keys_of, reference
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rc.set_cache_dir(os.path.join(ROOT, "paper_2506_01374_amd", "jit_cache"))
    torch.cuda.set_device(0)
    op = rc.Op(kind, dims, flags)
    print(f"[gpu] search kind={kind} dims={dims} flags={flags}", flush=True)
    ev = tune.GpuEvaluator(op, repeat=2, warmup=1)
    res = tune.run_search(op, ev, "uct", budget=4, seed=2)
    assert res["valid"] >= 1 and res["best_reward"] > 0
    torch.cuda.synchronize()
    ins = [t.cpu() for t in ev._inputs(op.default())]
    offsets = ins[-3 if kind != rc.RC_OP_ATTENTION_PACKED else -2].tolist()
    q = [y - x for x, y in zip(offsets, offsets[1:])]
    if kind == rc.RC_OP_ATTENTION_PACKED:
        at = ins[4].tolist()
        keys, kept, lens = [[f64(x)[at[b]:at[b + 1]] for x in ins[1:3]] for b in range(3)], None, np.diff(at).tolist()
        check(ev.out, *reference(q, lens, f64(ins[0]), keys, flags & C, 64 ** -0.5, kept))
        return
    lens, table = ins[-2].tolist(), ins[-1].numpy()
    cache = [x.cpu() for x in ev.out] if kind == rc.RC_OP_KV_WRITE else ins[1 if kind == rc.RC_OP_ATTENTION_PAGED else 0:-3]
    keys, kept = keys_of(cache, table, lens, dims[-3], flags & I8)
    if kind == rc.RC_OP_ATTENTION_PAGED:
        check(ev.out, *reference(q, lens, f64(ins[0]), keys, flags & C, 64 ** -0.5, kept))
        return
    rows = [f64(x) for x in (ins[:2] if kind == rc.RC_OP_KV_WRITE else ev.out)]
    for b, n in enumerate(q):
        for row, key, there in zip(rows, keys[b], [kept[b]] * 2):
            x = np.where(there[:, None, None], key, 0)[lens[b] - n:] if n else key[:0]
            got = row[offsets[b]:offsets[b + 1]]
            if kind == rc.RC_OP_KV_READ:                     # int8 values with their scale: one rounding to bf16
                assert np.all(np.abs(got - x) <= (2.0 ** -8 + 2.0 ** -24) * np.abs(x) if flags else got == x)
            else:                                            # half a step, of max / 127, and the scale's two roundings
                step = np.abs(got).max(-1, keepdims=True) / 127
                assert np.all(np.abs(got - x) <= (0.5 + 127 * 3 * 2.0 ** -24) * step if flags else got == x)
