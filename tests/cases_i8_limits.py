"""Sizes and schedules of the tests of the 8-bit integer operators at the ends
of their ranges."""
from __future__ import annotations

from paper_2506_01374_amd import rc

from cases_i8 import R

# one row much longer than its threads: (columns, schedule)
LONG_ROWS = [((1 << 24) + 5, ""), ((1 << 24) + 5, "vec=8,waves=16"), (1 << 20, "vec=2,waves=4"), ((1 << 22) + 1, "vec=8,waves=4")]


def compile_jobs():
    """(op, [schedules]) for ahead-of-time compilation (suggestions are the
    package's own)."""
    jobs = []
    for kind, flags in ((rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)):
        for cols, text in LONG_ROWS:
            op = rc.Op(kind, (2, cols), flags)
            jobs.append((op, [op.from_string(text)]))
    return jobs
