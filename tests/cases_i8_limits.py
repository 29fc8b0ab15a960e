"""Sizes and schedules of the tests of the 8-bit integer operators at the ends
of their ranges, and of every suggested schedule."""
from __future__ import annotations

import functools

from paper_2506_01374_amd import rc

from cases_i8 import B, F, G, R

# rows whose products leave fp32's range: one and several rows a workgroup and
# waves a row, held and read again, and the suggestion
WIDE_COLS = 700
WIDE_TEXTS = ["", "vec=8,waves=2,held=1", "vec=8,waves=2,rows=4,held=1", "vec=8,rows=4,held=2", "vec=4,waves=4,rows=2,held=1",
              "vec=8,waves=2,rows=2", "waves=2,rows=2", "rows=8"]

# one row much longer than its threads: (columns, schedule)
LONG_ROWS = [((1 << 24) + 5, ""), ((1 << 24) + 5, "vec=8,waves=16"), (1 << 20, "vec=2,waves=4"), ((1 << 22) + 1, "vec=8,waves=4")]


def rows_texts(op, texts):
    return list(dict.fromkeys([t for t in texts if op.from_string(t).validate() == ""] + [str(op.suggest())]))


@functools.lru_cache(maxsize=None)
def suggested_products(flags):
    """(dims, schedule text) of every code object of the product's suggestions:
    ragged sizes of two row and two column tiles, K of more tiles than the ring
    is deep with the last one partial; a last, partial round where half-height
    tiles need one.  (The K splits of a bias or of fp32 output are those of the
    plain product.)"""
    jobs = []
    for op, sched in rc.suggestions(rc.RC_OP_GEMM_I8, flags):
        s = sched.as_dict()
        if s["splits"] > 1 and flags & (B | F):
            continue
        tm, tn, tk, sp, st = s["tile_m"], s["tile_n"], s["tile_k"], s["splits"], s["stages"]
        odd = 16 if st == 2 and not s["pad"] else 21

        def legal(dims):
            return rc.Op(rc.RC_OP_GEMM_I8, dims, flags).from_string(str(sched)).validate() == ""

        if st == 3:
            ks = [2 * s["waves_k"] * tk + 64 + odd]
        elif op.dims[2] == tk and tk < 256 and st == 2:
            ks = [tk - 16]                                          # tile_k halved to cover a short K
        else:
            ks = [sp * 13 * tk - tk + odd]                          # (a ring has at most 12 buffers)
        if s["tail"]:
            # a last row tile of less and of more than half
            found = [next(d for nt in (87, 90, 173, 260, 345) for k in ks if legal(d := (2 * tm + part, nt * tn - 5, k)))
                     for part in (tm // 4 + 1, 3 * tm // 4 + 1)]
        else:
            found = [(2 * tm - 3, 2 * tn - 5, k) for k in ks]
            assert legal(found[0]), (flags, str(sched))
        jobs += [(d, str(sched)) for d in found]
    return jobs


def suggested_rows(kind, flags):
    """(dims, schedule text) of every schedule suggested for rows: five rows of
    the fewest and of the most columns it is legal for, up to some 100,000."""
    jobs = []
    widths = sorted({w for p in range(18) for w in (2 ** p - 1, 2 ** p, 2 ** p + 1) if w > 0})
    for _, sched in rc.suggestions(kind, flags):
        legal = [w for w in widths if rc.Op(kind, (5, w), flags).from_string(str(sched)).validate() == ""]
        assert legal, str(sched)
        jobs += [((5, w), str(sched)) for w in dict.fromkeys((legal[0], legal[-1]))]
    return jobs


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
