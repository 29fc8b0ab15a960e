"""Tuning of the 8-bit integer operators: workloads, inputs, features and a
search, on the CPU with a made-up timing and on the GPU with the real one."""
import os

import numpy as np
import pytest

from paper_2506_01374_amd import rc, tune, workloads as W

torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
R, B, F, G = rc.RC_FLAG_RESIDUAL, rc.RC_FLAG_BIAS, rc.RC_FLAG_OUT_F32, rc.RC_FLAG_GATED
OPS = [(rc.RC_OP_RMSNORM_I8, (37, 300), 0), (rc.RC_OP_RMSNORM_I8, (37, 300), R), (rc.RC_OP_QUANT_I8, (37, 300), 0)] + [
    (rc.RC_OP_GEMM_I8, (70, 100, 272), f) for f in (0, B, F, B | F, G)]


@pytest.mark.parametrize("kind,dims,flags", OPS)
def test_inputs_and_outputs_are_those_of_a_launch(kind, dims, flags):
    op = rc.Op(kind, dims, flags)
    ins = W.to_device(W.stored_inputs(op, op.default(), W.host_inputs(op, seed=3)), device="cpu")
    outs = W.empty_output(op, device="cpu")
    want = rc._i8_tensors(op)
    rc._check_tensors(want, -1, ins, outs, None, None)
    again = W.to_device(W.stored_inputs(op, op.default(), W.host_inputs(op, seed=3)), device="cpu")
    other = W.to_device(W.stored_inputs(op, op.default(), W.host_inputs(op, seed=4)), device="cpu")
    assert all(torch.equal(x, y) for x, y in zip(ins, again))
    assert not any(torch.equal(x, y) for x, y in zip(ins, other))
    for t in ins:
        if t.dtype == torch.int8:
            assert t.min() >= -127 and t.float().std() > 16
    arrays = W.output_to_f64(op, outs)
    assert len(arrays) == len(outs) if isinstance(outs, tuple) else arrays.shape == tuple(dims[:2])
    if kind == rc.RC_OP_GEMM_I8:
        assert [W.output_shape(op)] == W.output_shapes(op)
    else:
        with pytest.raises(ValueError):
            W.output_shape(op)


@pytest.mark.parametrize("name", list(W.I8_WORKLOADS))
def test_workloads_have_a_reference_schedule(name):
    op = W.workload_op(name)
    assert op.from_string(tune.reference_schedule(name)).validate() == ""
    assert name not in W.WORKLOADS


def test_features_of_schedules():
    for kind, dims, flags in OPS:
        op = rc.Op(kind, dims, flags)
        found = [tune.schedule_features(op, s) for s in tune.random_walk_space(op, 12, seed=1)]
        assert len({len(f) for f in found}) == 1 and len(found[0]) > len(op.knob_names())
        assert np.all(np.isfinite(found))


@pytest.mark.parametrize("proposer,surrogate", [(None, False), ("feedback", False), ("model_repair", True)])
def test_a_search_with_a_made_up_timing(proposer, surrogate):
    op = rc.Op(rc.RC_OP_GEMM_I8, (512, 512, 1024))

    def timed(s):
        ms = 1.0 / (s["tile_m"] * s["tile_n"])
        return {"schedule": str(s), "valid": True, "ms": ms, "reward": s["tile_m"] * s["tile_n"] / 65536}

    ev = tune.ParallelGpuEvaluator(op, time_fn=timed, compile_fn=lambda job: 0)
    res = tune.run_search(op, ev, "uct", budget=40, seed=1, proposer=proposer, surrogate=surrogate)
    ev.close()
    assert res["valid"] > 1 and op.from_string(res["best"]).validate() == "" and res["best_reward"] >= 4 * 16 * 16 / 65536


def test_the_command_lists_walks_of_an_8_bit_workload(tmp_path):
    tune.main(["--workload", "gemm_i8_m16_n4096_k4096", "--walks", "5", "--out", str(tmp_path)])
    lines = open(tmp_path / "gemm_i8_m16_n4096_k4096.space.txt").read().split()
    op = W.workload_op("gemm_i8_m16_n4096_k4096")
    assert len(lines) == 5 and all(op.from_string(t).validate() == "" for t in lines)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,dims,flags", OPS)
def test_a_search_on_the_gpu_measures_launches_that_are_right(kind, dims, flags):
    from test_gpu_i8 import bf16, f64, gemm_reference, rows_reference
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
    got = W.output_to_f64(op, ev.out)
    if kind == rc.RC_OP_GEMM_I8:
        want, tol = gemm_reference(ins, flags)
        assert np.all(np.abs(got - want) <= tol)
    else:
        w = f64(ins[1]) if kind == rc.RC_OP_RMSNORM_I8 else None
        q, scale, h = rows_reference(f64(ins[0]), w, f64(ins[2]) if flags else None, op.eps or 1.0)
        assert np.array_equal(got[0], q)
        # 300 columns: test_gpu_i8's bound
        assert np.all(np.abs(got[1] - scale) <= ((5 + 21) / 2 + 5) * 2.0 ** -24 * scale)
        if flags:
            assert np.array_equal(f64(bf16(h)), got[2])
