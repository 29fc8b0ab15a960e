"""Sizes and schedules of the tests of attention in serving."""
from __future__ import annotations

from paper_2506_01374_amd import rc

C, I8 = rc.RC_FLAG_CAUSAL, rc.RC_FLAG_I8_CACHE

# (new rows of each sequence, tokens of each, K/V heads, head dimension, page):
# one token, lengths around a page and a tile, sequences without rows, empty
# ones, more new rows than tokens, more tokens than the table holds (a page
# less than the longest needs)
CACHE_CASES = [
    ([1], [1], 1, 64, 16), ([1, 1, 1], [1, 17, 64], 2, 128, 16), ([5, 0, 3, 16], [5, 9, 40, 16], 3, 64, 32),
    ([33, 1, 70], [100, 1, 70], 5, 128, 64), ([3, 4], [2, 300], 1, 256, 16), ([1] * 70, list(range(1, 71)), 2, 64, 16),
    ([2] * 130 + [0] * 5 + [1] * 4000, [2] * 4135, 1, 64, 16), ([40, 200], [40, 500], 2, 256, 256), ([9], [2], 2, 128, 128)]

# the same with query heads for each K/V head
PAGED_CASES = [
    ([1], [1], 1, 1, 64, 16), ([1], [40], 1, 4, 128, 16), ([1, 1, 1, 1], [1, 31, 32, 33], 2, 4, 128, 16),
    ([1, 0, 1], [500, 77, 0], 2, 7, 64, 32), ([5, 3, 1], [5, 300, 64], 1, 5, 128, 64), ([17], [17], 2, 3, 64, 16),
    ([1, 16, 2], [700, 16, 129], 1, 8, 256, 32), ([70, 1], [70, 333], 2, 4, 128, 128), ([3, 4], [2, 300], 1, 16, 64, 256),
    ([130], [1000], 1, 4, 128, 16), ([40, 3], [1500, 900], 2, 4, 128, 16), ([33, 64], [64, 640], 2, 2, 64, 32), ([70], [400], 1, 3, 256, 64), ([1] * 70, [1 + 13 * i % 200 for i in range(70)], 1, 2, 64, 16), ([9], [4], 1, 1, 256, 16)]

# (rows of Q of each sequence, of K, K/V heads, query heads for each, head dimension)
PACKED_CASES = [
    ([1], [1], 1, 1, 64), ([1, 37, 200], [1, 37, 200], 2, 4, 128), ([33, 0, 5], [33, 0, 5], 1, 3, 256),
    ([16, 32, 64], [16, 32, 64], 2, 1, 64), ([10, 1, 7], [100, 64, 3], 1, 8, 128), ([300], [300], 1, 4, 128),
    ([0, 2, 129], [5, 2, 129], 1, 5, 64), ([65], [257], 2, 2, 256), ([700, 3, 129], [700, 3, 129], 2, 4, 128), ([257], [600], 3, 1, 64)]

CACHE_TEXTS = ["", "vec=8", "waves=4,vec=8"]
ATTENTION_TEXTS = ["", "block_m=32", "waves=4", "block_m=32,waves=2,splits=1", "waves=4,splits=2",
                   "block_m=64,waves=8,stages=3,occ=2", "block_m=128,waves=8,stages=3,occ=2,splits=1", "block_m=64,waves=8,stages=3,occ=2,splits=4",
                   "stages=2,waves=2,occ=1,splits=1", "stages=1,waves=4,occ=2,splits=2",
                   "block_m=64,waves=4,stages=3,occ=2", "block_m=128,waves=4,stages=3,occ=2,splits=2"]


def cache_op(kind, case, flags, pages=None):
    q, lens, hkv, d, page = case
    width = max(1, -(-max(lens) // page))
    return rc.Op(kind, (sum(q), len(q), hkv, d, page, pages or sum(-(-n // page) for n in lens) + 2, width), flags)


def paged_op(case, flags, width=None, pages=None):
    q, lens, hkv, g, d, page = case
    width = width or max(1, -(-max(lens) // page))
    pages = pages or sum(-(-n // page) for n in lens) + 2
    return rc.Op(rc.RC_OP_ATTENTION_PAGED, (sum(q), len(q), hkv * g, hkv, d, page, pages, width), flags)


def packed_op(case, flags):
    q, k, hkv, g, d = case
    return rc.Op(rc.RC_OP_ATTENTION_PACKED, (sum(q), sum(k), len(q), hkv * g, hkv, d), flags)


def legal(op, texts):
    """The suggested schedule and those of `texts` that are legal."""
    found = [str(op.from_string(t)) for t in texts if op.from_string(t).validate() == ""]
    return list(dict.fromkeys([str(op.suggest())] + found))


def compile_jobs():
    """(op, [schedules]) for ahead-of-time compilation."""
    jobs = []
    for flags in (0, I8):
        for kind in (rc.RC_OP_KV_WRITE, rc.RC_OP_KV_READ):
            jobs += [(cache_op(kind, c, flags), CACHE_TEXTS) for c in CACHE_CASES]
        for causal in (0, C):
            jobs += [(paged_op(c, flags | causal), ATTENTION_TEXTS) for c in PAGED_CASES]
    jobs += [(packed_op(c, C), ATTENTION_TEXTS) for c in PACKED_CASES]
    jobs = [(op, [op.from_string(t) for t in legal(op, texts)]) for op, texts in jobs]
    # one job a code object: the sizes are arguments, but for the head dimension
    found = {}
    for op, scheds in jobs:
        for s in scheds:
            d = op.dims[{rc.RC_OP_ATTENTION_PAGED: 4, rc.RC_OP_ATTENTION_PACKED: 5}.get(op.kind, 3)]
            found.setdefault((op.kind, op.flags & I8, d, str(s)), (op, [s]))
    return list(found.values())
