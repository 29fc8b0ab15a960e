"""CPU tests of what build() compiles."""
import os
import shutil
import subprocess
import sys

from paper_2506_01374_amd import rc, workloads as W

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
sys.path.insert(0, {root!r})
import __graft_entry__ as g
jobs, walks = g.jobs_of_tests({folder!r})
assert "cases_i8" not in sys.modules, "the tests' list is not part of the package"
print(len(jobs), len(walks), len(g.product_jobs()))
"""


def counts(folder):
    out = subprocess.run([sys.executable, "-c", PROGRAM.format(root=ROOT, folder=str(folder))], capture_output=True, text=True,
                         timeout=300)
    assert out.returncode == 0, out.stderr
    return [int(x) for x in out.stdout.split()]


def test_build_needs_no_test_module_of_the_8_bit_operators(tmp_path):
    # tests that do not know these operators, or none at all
    folder, package = tmp_path / "tests", tmp_path / "paper_2506_01374_amd"
    folder.mkdir()
    package.mkdir()
    jobs, walks, product = counts(folder)
    assert jobs == walks == 0 and product > 700
    shutil.copy(os.path.join(ROOT, "tests", "cases.py"), folder)
    shutil.copy(os.path.join(ROOT, "paper_2506_01374_amd", "tuned.json"), package)      # (which it reads)
    jobs, walks, again = counts(folder)
    assert jobs > 0 and walks > 0 and again == product


def test_build_compiles_what_the_package_launches():
    import __graft_entry__ as g
    jobs = {(op.kind, op.dims, op.flags, str(s)) for op, scheds in g.product_jobs() for s in scheds}
    for name in W.WORKLOADS:
        op = W.workload_op(name)
        assert (op.kind, op.dims, op.flags, str(op.default())) in jobs
    kinds = {(kind, flags) for kind, _, flags, _ in jobs}
    for kind in (rc.RC_OP_QUANT_I8, rc.RC_OP_RMSNORM_I8):
        assert (kind, 0) in kinds
    for flags in (0, rc.RC_FLAG_BIAS, rc.RC_FLAG_OUT_F32, rc.RC_FLAG_BIAS | rc.RC_FLAG_OUT_F32, rc.RC_FLAG_GATED):
        assert (rc.RC_OP_GEMM_I8, flags) in kinds
    op = rc.Op(rc.RC_OP_GEMM_I8, (20, 4668, 1188), rc.RC_FLAG_BIAS | rc.RC_FLAG_OUT_F32)
    assert str(op.suggest()).replace("pad=1", "pad=0") in {text for kind, _, flags, text in jobs
                                                          if (kind, flags) == (op.kind, op.flags)}


def test_compilation_says_how_far_it_is_and_what_failed(tmp_path, capfd):
    import __graft_entry__ as g
    import pytest
    op = rc.Op(rc.RC_OP_QUANT_I8, (3, 100))
    good, bad = [op.schedule(vec=2), op.default()], op.schedule(waves=16, rows=8)
    g.compile_kernels([(op, good + good)], [(op, [bad])], str(tmp_path))
    assert "build: kernels of 3 of 3 schedules" in capfd.readouterr().out
    assert sum(f.endswith(".hsaco") for f in os.listdir(tmp_path)) == 2
    with pytest.raises(RuntimeError, match="failed for 1 schedules"):
        g.compile_kernels([(op, [bad])], [], str(tmp_path))
