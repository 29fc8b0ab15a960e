"""Sizes and schedules of the tests of the 8-bit integer operators at the ends
of their ranges."""
from __future__ import annotations

from paper_2506_01374_amd import rc

from cases_i8 import R

# rows whose products leave fp32's range: one and several rows a workgroup and
# waves a row, held and read again, and the suggestion
WIDE_COLS = 700
WIDE_TEXTS = ["", "vec=8,waves=2,held=1", "vec=8,waves=2,rows=4,held=1", "vec=8,rows=4,held=2", "vec=4,waves=4,rows=2,held=1",
              "vec=8,waves=2,rows=2", "waves=2,rows=2", "rows=8"]

# one row much longer than its threads: (columns, schedule)
LONG_ROWS = [((1 << 24) + 5, ""), ((1 << 24) + 5, "vec=8,waves=16"), (1 << 20, "vec=2,waves=4"), ((1 << 22) + 1, "vec=8,waves=4")]


def rows_texts(op, texts):
    return list(dict.fromkeys([t for t in texts if op.from_string(t).validate() == ""] + [str(op.suggest())]))


def compile_jobs():
    """(op, [schedules]) for ahead-of-time compilation (suggestions are the
    package's own)."""
    jobs = []
    for kind, flags in ((rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)):
        op = rc.Op(kind, (12, WIDE_COLS), flags)
        jobs += [(op, [op.from_string(t)]) for t in rows_texts(op, WIDE_TEXTS)]
        for cols, text in LONG_ROWS:
            op = rc.Op(kind, (2, cols), flags)
            jobs.append((op, [op.from_string(text)]))
    return jobs
