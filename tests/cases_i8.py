"""Sizes and schedules of the 8-bit integer operators' tests."""
from __future__ import annotations

import math
import random

from paper_2506_01374_amd import rc

R, B, F, G = rc.RC_FLAG_RESIDUAL, rc.RC_FLAG_BIAS, rc.RC_FLAG_OUT_F32, rc.RC_FLAG_GATED

# (rows, columns): single elements, rows around a vector, a wave's and a
# workgroup's step, odd widths, more rows than a workgroup takes
ROWS_DIMS = [(1, 1), (3, 2), (5, 7), (1, 8), (4, 9), (2, 63), (7, 64), (3, 65), (2, 511), (9, 512), (2, 513), (5, 1001),
             (3, 2048), (2, 4097), (1, 14336), (2, 16385)]
ROWS_TEXTS = ["", "vec=8", "vec=4,rows=2", "waves=2,vec=2", "vec=8,held=1", "vec=8,held=2", "waves=4,vec=8,held=2,rows=2",
              "waves=4,vec=8,held=4", "waves=8,vec=8,held=4", "waves=16,vec=8,held=1", "waves=16,vec=8,held=4",
              "vec=2,held=1,rows=4", "waves=16,vec=1", "waves=2,vec=8,rows=8"]


def rows_jobs():
    """(dims, schedule text) of every size with its legal schedules."""
    jobs = []
    for dims in ROWS_DIMS:
        op = rc.Op(rc.RC_OP_QUANT_I8, dims)
        texts = [t for t in ROWS_TEXTS if op.from_string(t).validate() == ""]
        jobs += [(dims, t) for t in dict.fromkeys(texts + [str(op.suggest())])]
    return jobs


_TILE = "tile_m={},tile_n={},tile_k={},waves_m={},waves_n={},waves_k={},mfma={},stages={},order={},occ={},splits={}"
GEMM_TEXTS = [_TILE.format(*t) for t in (
    # double buffer
    (16, 16, 64, 1, 1, 1, 16, 1, 0, 1, 1), (32, 64, 64, 2, 2, 1, 16, 1, 1, 1, 1), (64, 64, 128, 2, 2, 1, 32, 1, 1, 2, 1),
    (128, 128, 128, 2, 4, 1, 16, 1, 1, 1, 1), (128, 64, 64, 4, 1, 1, 32, 1, 0, 1, 2), (256, 128, 64, 2, 4, 1, 16, 1, 1, 1, 1),
    (64, 32, 256, 4, 2, 1, 16, 1, 1, 1, 1), (16, 16, 64, 1, 1, 1, 16, 1, 1, 1, 4),
    # ring
    (64, 64, 128, 2, 2, 1, 16, 2, 1, 1, 1), (128, 128, 128, 2, 2, 1, 16, 2, 1, 1, 2), (256, 128, 64, 4, 2, 1, 32, 2, 1, 1, 1),
    (256, 256, 64, 2, 4, 1, 32, 2, 1, 1, 1), (32, 32, 128, 1, 1, 1, 16, 2, 0, 2, 4), (64, 128, 256, 2, 2, 1, 32, 2, 1, 1, 1),
    (128, 128, 64, 2, 2, 1, 32, 2, 1, 2, 16), (256, 256, 64, 2, 4, 1, 16, 2, 1, 1, 1), (64, 64, 64, 2, 2, 1, 16, 2, 1, 1, 1),
    (64, 64, 64, 2, 2, 1, 16, 2, 1, 1, 2),
    # streaming
    (16, 16, 64, 1, 1, 1, 16, 3, 0, 1, 1), (16, 16, 256, 1, 1, 8, 16, 3, 0, 1, 1), (16, 64, 128, 1, 1, 4, 16, 3, 1, 1, 1),
    (32, 32, 128, 1, 1, 16, 16, 3, 0, 1, 1), (64, 32, 128, 1, 1, 2, 16, 3, 1, 1, 1), (64, 64, 64, 1, 1, 8, 16, 3, 0, 1, 1))]
# the ring on rows copied to whole 16-byte chunks
GEMM_TEXTS += [_TILE.format(*t) + ",pad=1" for t in (
    (64, 64, 128, 2, 2, 1, 16, 2, 1, 1, 1), (32, 32, 128, 1, 1, 1, 16, 2, 0, 2, 4), (64, 128, 256, 2, 2, 1, 32, 2, 1, 1, 1),
    (16, 16, 256, 1, 1, 1, 16, 2, 1, 1, 1), (256, 256, 64, 2, 4, 1, 16, 2, 1, 1, 1), (128, 128, 128, 2, 4, 1, 16, 2, 1, 1, 2))]

# (M, N, K): one of each, around 16 and the tiles, K around a chunk, an MFMA
# step and the K tiles, rows that start on no alignment, a last split of K
# that is shorter than a load (773 in four splits of tiles of 64)
GEMM_DIMS = [(1, 1, 1), (1, 17, 16), (2, 3, 15), (15, 16, 17), (16, 100, 64), (17, 33, 65), (1, 260, 1000), (33, 64, 63),
             (64, 129, 127), (65, 128, 128), (100, 61, 129), (130, 257, 256), (257, 130, 257), (300, 272, 400),
             (128, 256, 1040), (16, 64, 4096), (70, 96, 2064), (300, 260, 1001), (16, 40, 2050), (5, 48, 1100),
             (20, 40, 773)]


# a last, partial round of workgroups in half-height tiles: with a last row
# tile that is whole, less than half and more than half, and K of one tile
# and many
TAIL_TEXT = "tile_m=32,tile_n=16,tile_k=128,waves_m=1,waves_n=1,mfma=16,stages=2,order=1,occ=1,tail=1"
TAIL_WIDE = "tile_m=256,tile_n=128,tile_k=64,waves_m=2,waves_n=4,mfma=16,stages=2,order=1,occ=1,tail=1"
TAIL_DIMS = [(32 * 10, 16 * 110, 128), (32 * 9 + 5, 16 * 140, 400), (32 * 9 + 20, 16 * 120 - 3, 1600), (32 * 20, 16 * 60, 80)]
TAIL_WIDE_DIMS = [(256 * 5 + 140, 128 * 45, 512), (256 * 6 + 4, 128 * 40 + 10, 1040)]
TAIL_PAD_DIMS = (256 * 6 + 4, 128 * 40 + 10, 1029)


def tail_jobs(flags):
    jobs = [(dims, TAIL_TEXT) for dims in TAIL_DIMS] + [(dims, TAIL_WIDE) for dims in TAIL_WIDE_DIMS]
    jobs += [(TAIL_PAD_DIMS, TAIL_WIDE + ",pad=1")]
    return [(dims, text) for dims, text in jobs if rc.Op(rc.RC_OP_GEMM_I8, dims, flags).from_string(text).validate() == ""]


# an operand, the output and the partial sums past 2^32 bytes or elements
LARGE = [
    ((3, 270000, 16384), dict(stages=3, tile_k=256, waves_k=4)),
    ((3, 270000, 16384), dict(stages=2, tile_k=256, tile_n=32, waves_n=2, order=1)),
    ((3, 270000, 16384), dict(stages=1, tile_n=64, tile_k=128, waves_n=2)),
    ((3, 270000, 16383), dict(stages=2, tile_k=256, tile_n=32, waves_n=2, order=1, pad=1)),
    ((270000, 48, 16384), dict(stages=2, tile_m=256, tile_n=64, tile_k=128, waves_m=4, order=1)),
    ((270000, 48, 16384), dict(stages=1, tile_m=128, tile_n=32, tile_k=128, waves_m=2, waves_n=2)),
    ((70000, 65536, 128), dict(stages=2, tile_m=128, tile_n=128, tile_k=128, waves_m=2, waves_n=2, order=1)),
    ((17000, 65536, 256), dict(stages=2, tile_m=128, tile_n=128, tile_k=128, waves_m=2, waves_n=2, order=1, splits=2))]


def gemm_jobs(flags):
    jobs = []
    for dims in GEMM_DIMS:
        op = rc.Op(rc.RC_OP_GEMM_I8, dims, flags)
        texts = [t for t in GEMM_TEXTS if op.from_string(t).validate() == ""]
        jobs += [(dims, t) for t in dict.fromkeys(texts + [str(op.suggest())])]
    return jobs


def _sizes(ndims, count, most, seed):
    """Sizes spread over the logarithm, whole multiples of 16 and odd ones."""
    g = random.Random(seed)
    for _ in range(count):
        dims = [max(1, int(2 ** g.uniform(0, math.log2(m)))) for m in most[:ndims]]
        if g.random() < 0.8:
            dims[-1] = min(most[ndims - 1], -(-dims[-1] // 16) * 16)
        yield dims


def suggested_jobs(count=20000, seed=1):
    """(op, schedule text): the different code objects that suggested schedules
    ask for over the range of sizes (the kernels take sizes as arguments, so
    that these are few), each with a size that it is suggested for."""
    found = {}
    for kind, flags in ((rc.RC_OP_QUANT_I8, 0), (rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)):
        for dims in _sizes(2, count // 3, (1 << 20, 1 << 18), seed):
            op = rc.Op(kind, dims, flags)
            found.setdefault((kind, flags, str(op.suggest())), op)
    for flags in (0, B, F, B | F, G):
        for dims in _sizes(3, count, (16384, 262144, 131071), seed):
            op = rc.Op(rc.RC_OP_GEMM_I8, dims, flags)
            found.setdefault((op.kind, flags, str(op.suggest())), op)
    return [(op, text) for (_, _, text), op in found.items()]


def compile_jobs():
    """(op, [schedules]) for ahead-of-time compilation."""
    jobs = [(op, [op.from_string(t)]) for op, t in suggested_jobs()]
    for dims, text in rows_jobs():
        for kind, flags in ((rc.RC_OP_QUANT_I8, 0), (rc.RC_OP_RMSNORM_I8, 0), (rc.RC_OP_RMSNORM_I8, R)):
            op = rc.Op(kind, dims, flags)
            jobs.append((op, [op.from_string(text)]))
    for flags in (0, B, F, B | F, G):
        for dims, text in gemm_jobs(flags) + tail_jobs(flags):
            op = rc.Op(rc.RC_OP_GEMM_I8, dims, flags)
            jobs.append((op, [op.from_string(text)]))
    op = rc.Op(rc.RC_OP_GEMM_I8, (130, 200, 1001), B)
    jobs.append((op, [op.schedule(tile_m=64, tile_n=64, tile_k=128, waves_m=2, waves_n=2, stages=2, order=1, splits=2, pad=1)]))
    for dims, knobs in LARGE:
        op = rc.Op(rc.RC_OP_GEMM_I8, dims)
        jobs.append((op, [op.schedule(**knobs)]))
    # one job a code object: a schedule and the flags, whatever the sizes
    return list({(op.kind, op.flags, str(s[0])): (op, s) for op, s in jobs}.values())
