"""GPU tests of attention in serving against 64-bit references.

What the cache holds and what is read from it is compared for equality.
Attention, with u = 2^-24 (half a step of fp32, relative), A = sum p |V| / sum p
(the result with the values' magnitudes) and B the largest sum |q| |k| / sqrt(D)
of the row:
  p       a score's sum of D products and its scales: (D + 4) u B; the exponent's
          multiply-add and its maximum: 4 u of the largest score; the exponential
          itself 4 u.  Its rounding to bf16 for the second product, with int8 of
          p times V's scale (u more): 2^-8 A.  (The sum of p takes fp32.)
  sums    keys + 256 additions and rescalings, of p V and of p: twice that u A.
  output  rounding to bf16: 2^-8 of the result.
"""
import math
import os

import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_seqs as S
from cases_seqs import C, I8

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U, BF16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rc.set_cache_dir(os.path.join(ROOT, "paper_2506_01374_amd", "jit_cache"))
    torch.cuda.set_device(0)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32).to(torch.bfloat16)


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


def starts(counts):
    return np.concatenate([[0], np.cumsum(counts)]).tolist()


GUARD = 32


def guarded(shape, dtype, fill=None):
    """A tensor of `shape` inside a buffer whose ends are checked."""
    n = math.prod(shape)
    buf = torch.full((n + 2 * GUARD,), 77, dtype=dtype, device="cuda")
    t = buf[GUARD:GUARD + n].view(shape)
    if fill is not None:
        t.copy_(fill)
    return buf, t


def intact(buf):
    return bool((buf[:GUARD] == 77).all()) and bool((buf[-GUARD:] == 77).all())


def quantised(x):
    """(q, scale) of the last dimension, in 64 bits."""
    a = np.abs(x).max(-1)
    with np.errstate(all="ignore"):
        q = np.rint(127 * x / a[..., None])
        scale = (a / 127).astype(np.float32)
    bad = ~np.isfinite(a)
    q = np.where((bad | (a == 0))[..., None], 0, q).astype(np.int8)
    return q, np.where(bad, np.float32(np.nan), scale)


# ---------------------------------------------------------------------------
# The cache
# ---------------------------------------------------------------------------

def tables(lens, page, pages, width, g):
    """Pages in any order, -1 where a sequence has none."""
    table = np.full((len(lens), width), -1, np.int64)
    ids = g.permutation(pages).tolist()
    for b, n in enumerate(lens):
        for i in range(min(width, -(-n // page))):
            table[b, i] = ids.pop()
    return table


def places(q, lens, table, page, pages):
    """(row, page, slot) of the rows that have a page; the others."""
    at, none, row = [], [], 0
    for b, (n, m) in enumerate(zip(q, lens)):
        for p in range(m - n, m):
            i = table[b, p // page] if 0 <= p and p // page < table.shape[1] else -1
            if 0 <= i < pages:
                at.append((row, int(i), p % page))
            else:
                none.append(row)
            row += 1
    return [np.array(x, dtype=np.int64) for x in zip(*at)] or [np.zeros(0, np.int64)] * 3, none


def cache_of(op, g, i8):
    hkv, d, page, pages = op.dims[2:6]
    shape = (pages, hkv, page, d)
    if i8:
        return [torch.from_numpy(g.integers(-127, 128, shape, dtype=np.int8)) for _ in range(2)] + [
            torch.from_numpy((0.5 + g.random(shape[:3])).astype(np.float32)) for _ in range(2)]
    return [bf16(g.standard_normal(shape)) for _ in range(2)]


def same(got, want):
    return np.array_equal(f64(got), np.asarray(want, dtype=np.float64), equal_nan=True)


def run_write(op, text, rows, where, cache):
    print(f"[gpu] write dims={op.dims} flags={op.flags} sched={text}", flush=True)
    bufs = [guarded(tuple(c.shape), c.dtype, c) for c in cache]
    plan = rc.Plan(op, op.from_string(text))
    plan.launch([x.cuda() for x in rows + where], tuple(t for _, t in bufs), plan.workspace())
    torch.cuda.synchronize()
    assert all(intact(b) for b, _ in bufs)
    return [t for _, t in bufs]


def check_write(op, text, q, lens, table, g, i8, rows=None, extra=0):
    t, b, hkv, d, page, pages, width = op.dims
    rows = rows or [bf16(g.standard_normal((t, hkv, d)) * 3) for _ in range(2)]
    cache = cache_of(op, g, i8)
    want = [f64(c) for c in cache]
    (at, page_at, slot), _ = places(q, lens, table, page, pages)
    for i, x in enumerate(rows):
        x = f64(x)[at]
        if i8:
            x, want[2 + i][page_at, :, slot] = quantised(x)
        want[i][page_at, :, slot] = x
    got = run_write(op, text, rows, [ints(starts(q)), ints(lens), ints(table)], cache)
    for x, y in zip(got, want):
        assert same(x, y)


@pytest.mark.parametrize("i8", [0, I8])
@pytest.mark.parametrize("case", S.CACHE_CASES)
def test_write(case, i8):
    q, lens, hkv, d, page = case
    op = S.cache_op(rc.RC_OP_KV_WRITE, case, i8)
    for i, text in enumerate(S.legal(op, S.CACHE_TEXTS)):
        g = np.random.default_rng(i)
        check_write(op, text, q, lens, tables(lens, page, op.dims[5], op.dims[6], g), g, i8)


@pytest.mark.parametrize("i8", [0, I8])
def test_write_without_pages(i8):
    # rows of no sequence at either end, tokens past the table, pages that are
    # not in the cache, a sequence with fewer tokens than new rows
    q, lens = [20, 7, 40], [50, 7, 30]
    op = rc.Op(rc.RC_OP_KV_WRITE, (80, 3, 2, 64, 16, 9, 3), i8)
    g = np.random.default_rng(5)
    table = np.array([[0, 3, 9], [-1, 2, 2], [2 ** 31 - 1, 7, -2 ** 31]])
    rows = [bf16(g.standard_normal((80, 2, 64))) for _ in range(2)]
    cache = cache_of(op, g, i8)
    want = [f64(c) for c in cache]
    (at, page_at, slot), none = places(q, lens, table, 16, 9)
    assert len(at) and len(none)
    for i, x in enumerate(rows):
        x = f64(x)[at + 4]
        if i8:
            x, want[2 + i][page_at, :, slot] = quantised(x)
        want[i][page_at, :, slot] = x
    got = run_write(op, str(op.suggest()), rows, [ints([4, 24, 31, 71]), ints(lens), ints(table)], cache)
    for x, y in zip(got, want):
        assert same(x, y)


@pytest.mark.parametrize("text", S.CACHE_TEXTS)
def test_write_of_zeros_nan_infinities_and_halves(text):
    # a = 127 m: the quotients are x / m, halves among them, and one step of
    # bf16 to either side; far magnitudes
    d = 128
    rows = []
    for m in (1.0, 2.0, 0.5, 3.0, 2.0 ** -70, 2.0 ** 70, 2.0 ** -126, 2.0 ** 120):
        for scale in (1.0, 1 + 2.0 ** -7, 1 - 2.0 ** -7):
            for part in (0, 1):
                x = f64(bf16((np.arange(-127, 127)[part::2] + 0.5) * m)) * scale
                rows.append(np.concatenate([x[:127], [127 * m]]))
    x = np.stack(rows)
    x[np.abs(x) > np.abs(x[:, -1:])] = 0
    special = np.zeros((6, d))
    special[1, 5], special[2, 127], special[3, 0], special[4, 9] = np.nan, np.inf, -np.inf, 2.0 ** -133
    special[5] = -3e38
    x = f64(bf16(np.concatenate([x, special])))
    n = len(x)
    case = ([n], [n], 1, d, 16)
    op = S.cache_op(rc.RC_OP_KV_WRITE, case, I8)
    g = np.random.default_rng(6)
    k = bf16(x[:, None])
    check_write(op, str(op.from_string(text)), [n], [n], tables([n], 16, op.dims[5], op.dims[6], g), g, I8, rows=[k, k.flip(0)])


@pytest.mark.parametrize("i8", [0, I8])
@pytest.mark.parametrize("case", S.CACHE_CASES)
def test_read(case, i8):
    q, lens, hkv, d, page = case
    op = S.cache_op(rc.RC_OP_KV_READ, case, i8)
    t, pages, width = op.dims[0], op.dims[5], op.dims[6]
    for i, text in enumerate(S.legal(op, S.CACHE_TEXTS)):
        print(f"[gpu] read dims={op.dims} flags={op.flags} sched={text}", flush=True)
        g = np.random.default_rng(10 + i)
        table = tables(lens, page, pages, width, g)
        cache = cache_of(op, g, i8)
        (at, page_at, slot), _ = places(q, lens, table, page, pages)
        bufs = [guarded((t, hkv, d), torch.bfloat16) for _ in range(2)]
        plan = rc.Plan(op, op.from_string(text))
        where = [ints(starts(q)), ints(lens), ints(table)]
        plan.launch([x.cuda() for x in cache + where], tuple(b[1] for b in bufs))
        torch.cuda.synchronize()
        for j, (buf, got) in enumerate(bufs):
            want = np.zeros((t, hkv, d))
            x = f64(cache[j])[page_at, :, slot]
            want[at] = f64(bf16(x * f64(cache[2 + j])[page_at, :, slot][..., None])) if i8 else x
            assert intact(buf) and same(got, want)


def test_read_leaves_the_rows_of_no_sequence():
    op = rc.Op(rc.RC_OP_KV_READ, (20, 2, 1, 64, 16, 4, 2))
    g = np.random.default_rng(3)
    cache = [x.cuda() for x in cache_of(op, g, 0)]
    outs = [torch.full((20, 1, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rc.Plan(op, op.suggest()).launch(cache + [ints([2, 5, 9]).cuda(), ints([20, 4]).cuda(), ints([[1, -1], [3, 0]]).cuda()],
                                     tuple(outs))
    torch.cuda.synchronize()
    for c, out in zip(cache, outs):
        want = np.full((20, 1, 64), 7.0)
        want[2:5] = 0                                       # 17, 18, 19: no page
        want[5:9] = f64(c)[3, :, 0:4].transpose(1, 0, 2)    # 0 .. 3
        assert same(out, want)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------

def attend(q, k, v, seen, scale):
    """(result, bound of its error) of rows q over keys k, v (one head), where
    row i sees the keys seen[i]."""
    s = q @ k.T * scale
    s = np.where(seen, s, -np.inf)
    top = s.max(1, initial=-np.inf)
    some = top > -np.inf
    with np.errstate(invalid="ignore"):
        p = np.where(seen, np.exp(s - np.where(some, top, 0)[:, None]), 0)
    total = np.where(some, p.sum(1), 1)[:, None]
    out, size = p @ v / total, p @ np.abs(v) / total
    big = np.where(seen, np.abs(q) @ np.abs(k).T * scale, 0).max(1, initial=0)[:, None]
    far = np.where(seen, np.abs(s), 0).max(1, initial=0)[:, None]
    rel = ((q.shape[1] + 4) * big + 4 * far + 4) * U
    return out, size * (BF16 + U + 2 * rel + 2 * (k.shape[0] + 256) * U) * 1.01 + BF16 * np.abs(out)


def reference(qs, ms, q, keys, causal, scale, kept=None):
    """Rows packed by qs over each sequence's (k, v) of ms tokens [m][Hkv][D];
    kept[b]: keys that are held."""
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    at, g = starts(qs), q.shape[1] // keys[0][0].shape[1]
    for b, (n, m) in enumerate(zip(qs, ms)):
        k, v = keys[b]
        have = k.shape[0]
        seen = np.ones((n, have), bool) if not causal else np.arange(have)[None, :] <= (np.arange(n) + m - n)[:, None]
        if kept is not None:
            seen &= kept[b][None, :have]
        rows = slice(at[b], at[b + 1])
        for h in range(q.shape[1]):
            # (what no row sees may be a NaN: it is left out here)
            some = seen.any(0)
            out[rows, h], tol[rows, h] = attend(q[rows, h], k[some][:, h // g], v[some][:, h // g], seen[:, some], scale)
    return out, tol


def check(got, want, tol):
    err = np.abs(f64(got) - want)
    assert np.all(err <= tol + 1e-30), (float(np.max(err - tol)), np.argwhere(err > tol)[:5].tolist())


def paged_inputs(case, i8, seed, width=None, pages=None):
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, i8, width, pages)
    r = np.random.default_rng(seed)
    pages, width = op.dims[6], op.dims[7]
    table = tables(lens, page, pages, width, r)
    shape = (pages, hkv, page, d)
    far = np.where(r.random(d) < 0.05, 4.0, 1.0)
    if i8:
        pairs = [quantised(r.standard_normal(shape) * far), quantised(r.standard_normal(shape))]
        cache = [torch.from_numpy(p[0]) for p in pairs] + [torch.from_numpy(p[1]) for p in pairs]
    else:
        cache = [bf16(r.standard_normal(shape) * far), bf16(r.standard_normal(shape))]
    rows = bf16(r.standard_normal((sum(q), hkv * g, d)))
    return rows, cache, table


def keys_of(cache, table, lens, page, i8):
    """(k, v) of each sequence [keys][Hkv][D] in 64 bits, and which are held."""
    x = [f64(c) for c in cache]
    if i8:
        x = [x[0] * x[2][..., None], x[1] * x[3][..., None]]
    pages, hkv, _, d = x[0].shape
    keys, kept = [], []
    for b, m in enumerate(lens):
        m = max(0, min(m, table.shape[1] * page))
        ids = table[b, np.arange(m) // page]
        held = (ids >= 0) & (ids < pages)
        at = np.where(held, ids, 0)
        keys.append([y[at, :, np.arange(m) % page].reshape(m, hkv, d) for y in x])
        kept.append(held)
    return keys, kept


def run_paged(op, text, rows, cache, where, out=None):
    print(f"[gpu] paged dims={op.dims} flags={op.flags} sched={text}", flush=True)
    buf, got = guarded(tuple(rows.shape), torch.bfloat16, out)
    plan = rc.Plan(op, op.from_string(text))
    plan.launch([x.cuda() for x in [rows] + cache + where], got, plan.workspace())
    torch.cuda.synchronize()
    assert intact(buf)
    return got


@pytest.mark.parametrize("flags", [0, C, I8, I8 | C])
@pytest.mark.parametrize("case", S.PAGED_CASES)
def test_paged(case, flags):
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 1)
    keys, _ = keys_of(cache, table, lens, page, flags & I8)
    want, tol = reference(q, lens, f64(rows), keys, flags & C, d ** -0.5)
    for text in S.legal(op, S.ATTENTION_TEXTS):
        check(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]), want, tol)


def packed_inputs(case, seed):
    q, k, hkv, g, d = case
    r = np.random.default_rng(seed)
    far = np.where(r.random(d) < 0.05, 4.0, 1.0)
    return [bf16(r.standard_normal((sum(q), hkv * g, d))), bf16(r.standard_normal((sum(k), hkv, d)) * far),
            bf16(r.standard_normal((sum(k), hkv, d)))]


def run_packed(op, text, ins, q, k, out=None):
    print(f"[gpu] packed dims={op.dims} flags={op.flags} sched={text}", flush=True)
    buf, got = guarded(tuple(ins[0].shape), torch.bfloat16, out)
    plan = rc.Plan(op, op.from_string(text))
    plan.launch([x.cuda() for x in ins + [ints(q), ints(k)]], got, plan.workspace())
    torch.cuda.synchronize()
    assert intact(buf)
    return got


@pytest.mark.parametrize("flags", [0, C])
@pytest.mark.parametrize("case", S.PACKED_CASES)
def test_packed(case, flags):
    q, k, hkv, g, d = case
    op = S.packed_op(case, flags)
    ins = packed_inputs(case, 2)
    at = starts(k)
    keys = [[f64(x)[at[b]:at[b + 1]] for x in ins[1:]] for b in range(len(k))]
    want, tol = reference(q, k, f64(ins[0]), keys, flags & C, d ** -0.5)
    for text in S.legal(op, S.ATTENTION_TEXTS):
        check(run_packed(op, text, ins, starts(q), at), want, tol)


@pytest.mark.parametrize("flags", [0, C, I8 | C])
def test_what_is_not_seen_may_be_anything(flags):
    # NaN and infinities in the free slots of pages, in pages not in use, and in
    # later tokens; pages that are not held
    case = ([40, 1, 3], [150, 33, 70], 2, 4, 128, 32)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 3)
    table[0, 1], table[2, 0] = -1, op.dims[6]
    keys, kept = keys_of(cache, table, lens, page, flags & I8)
    want, tol = reference(q, lens, f64(rows), keys, flags & C, d ** -0.5, kept)
    held = np.zeros((op.dims[6], page), bool)
    for b, m in enumerate(lens):
        for p in range(m):
            if 0 <= table[b, p // page] < op.dims[6]:
                held[table[b, p // page], p % page] = True
    free = torch.from_numpy(np.argwhere(~held))
    for c in cache[2 if flags & I8 else 0:]:
        for i, (at, slot) in enumerate(free.tolist()):
            c[at, :, slot] = (float("nan"), float("inf"), -float("inf"))[i % 3]
    for text in S.legal(op, S.ATTENTION_TEXTS):
        check(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]), want, tol)
    if not flags & C:
        return
    # token 120 of the first sequence: the rows from its own on see it, and are
    # NaN in the channel (or all of it) that it spoils
    at, slot = int(table[0, 120 // page]), 120 % page
    for c in range(2):
        spoilt = [x.clone() for x in cache]
        if flags & I8:
            spoilt[2 + c][at, :, slot] = float("nan")
        else:
            spoilt[c][at, :, slot, 5] = float("nan")
        for text in S.legal(op, S.ATTENTION_TEXTS):
            got = f64(run_paged(op, text, rows, spoilt, [ints(starts(q)), ints(lens), ints(table)]))
            nan = np.zeros(got.shape, bool)
            nan[10:40, :, 5 if c == 1 and not flags & I8 else slice(None)] = True
            assert np.array_equal(np.isnan(got), nan)
            err = np.abs(got - want)
            assert np.all(err[~nan] <= tol[~nan] + 1e-30)


@pytest.mark.parametrize("flags", [0, C])
def test_packed_neighbours_do_not_count(flags):
    case = ([20, 35, 9], [50, 35, 40], 1, 4, 128)
    q, k, hkv, g, d = case
    op = S.packed_op(case, flags)
    ins = packed_inputs(case, 4)
    at = starts(k)
    keys = [[f64(x)[at[b]:at[b + 1]] for x in ins[1:]] for b in range(3)]
    want, tol = reference(q, k, f64(ins[0]), keys, flags & C, d ** -0.5)
    for bad in (float("nan"), float("inf")):
        for b in (0, 2):
            spoilt = [x.clone() for x in ins]
            for x in spoilt[1:]:
                x[at[b]:at[b + 1]] = bad
            for text in S.legal(op, S.ATTENTION_TEXTS):
                got = f64(run_packed(op, text, spoilt, starts(q), at))
                rows = slice(20, 55)
                assert np.all(np.abs(got - want)[rows] <= tol[rows])
    # later tokens of the same sequence, and the rows of no sequence
    if flags & C:
        spoilt = [x.clone() for x in ins]
        spoilt[2][at[1] + 20:at[1] + 35] = float("inf")
        out = torch.full(tuple(ins[0].shape), 7.0, dtype=torch.bfloat16)
        for text in S.legal(op, S.ATTENTION_TEXTS):
            got = f64(run_packed(op, text, spoilt, [0, 20, 55, 60], at, out))
            assert np.all(np.abs(got - want)[:40] <= tol[:40]) and not np.isfinite(got[40:55]).any()
            assert np.all(got[60:] == 7)


def test_extreme_scores():
    # all scores at fp32's low end, all -infinity, one +infinity
    d = 64
    op = rc.Op(rc.RC_OP_ATTENTION_PACKED, (4, 60, 4, 1, 1, d))
    q, k, v = (torch.zeros(n, 1, d, dtype=torch.bfloat16) for n in (4, 60, 60))
    v[:, 0, 0] = torch.arange(60).to(torch.bfloat16)
    q[:, 0, 0] = torch.tensor([1.0, 1.0, 1.0, 1.0])
    k[0:15, 0, 0] = -2.0 ** 127
    k[15:30, 0, 0] = -float("inf")
    k[30:45, 0, 0] = 2.0 ** 127
    k[44, 0, 0] = -2.0 ** 127
    k[50, 0, 0] = float("inf")
    for text in S.legal(op, S.ATTENTION_TEXTS):
        got = f64(run_packed(op, text, [q, k, v], [0, 1, 2, 3, 4], [0, 15, 30, 45, 60]))[:, 0, 0]
        assert abs(got[0] - 7) <= 8 * BF16 + 7 * BF16 and got[1] == 0
        # keys 30 .. 43 are alike, the last far below
        assert abs(got[2] - 36.5) <= 2 * 36.5 * BF16 + 0.2 and np.isnan(got[3])


@pytest.mark.parametrize("flags", [0, C, I8 | C])
def test_a_row_that_is_not_finite_spoils_no_other(flags):
    case = ([70, 1, 3], [150, 40, 3], 2, 4, 128, 16)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 9)
    keys, _ = keys_of(cache, table, lens, page, flags & I8)
    want, tol = reference(q, lens, f64(rows), keys, flags & C, d ** -0.5)
    bad = [(0, 1), (17, 7), (69, 0), (70, 3), (73, 5)]
    for i, (row, head) in enumerate(bad):
        rows[row, head, 3 * i] = (float("nan"), float("inf"), -float("inf"))[i % 3]
    keep = np.ones(want.shape[:2], bool)
    keep[tuple(zip(*bad))] = False
    for text in S.legal(op, S.ATTENTION_TEXTS):
        got = f64(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]))
        assert np.all(np.abs(got - want)[keep] <= tol[keep] + 1e-30)
        assert np.isnan(got[0, 1]).all()


def test_offsets_and_lengths_that_make_no_sense_stay_in_bounds():
    case = ([8, 8, 8], [20, 20, 20], 1, 2, 64, 16)
    op = S.paged_op(case, C)
    rows, cache, table = paged_inputs(case, 0, 5)
    for offsets in ([-5, 100, 3, 7], [24, 0, 24, 24], [0, 2 ** 31 - 1, -2 ** 31, 24]):
        for lens in ([-1, 2 ** 31 - 1, 0], [-2 ** 31, 5, 1000]):
            for text in S.legal(op, S.ATTENTION_TEXTS):
                run_paged(op, text, rows, cache, [ints(offsets), ints(lens), ints(table)])
            wr = rc.Op(rc.RC_OP_KV_WRITE, (24, 3, 1, 64, 16, op.dims[6], op.dims[7]))
            kv = rows[:, :1].contiguous()
            run_write(wr, str(wr.suggest()), [kv, kv], [ints(offsets), ints(lens), ints(table)], cache)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,flags", [(rc.RC_OP_ATTENTION_PAGED, C), (rc.RC_OP_ATTENTION_PAGED, I8 | C), (rc.RC_OP_ATTENTION_PACKED, C)])
def test_every_suggested_schedule(kind, flags, d):
    case = ([70, 1, 0, 3], [150, 40, 9, 3], 2, 4, d, 16)
    q, lens, hkv, g, _, page = case
    if kind == rc.RC_OP_ATTENTION_PAGED:
        op = S.paged_op(case, flags)
        rows, cache, table = paged_inputs(case, flags & I8, 70)
        keys, _ = keys_of(cache, table, lens, page, flags & I8)
    else:
        op = S.packed_op((q, lens, hkv, g, d), flags)
        ins, at = packed_inputs((q, lens, hkv, g, d), 70), starts(lens)
        rows, keys = ins[0], [[f64(x)[at[b]:at[b + 1]] for x in ins[1:]] for b in range(4)]
    want, tol = reference(q, lens, f64(rows), keys, True, d ** -0.5)
    texts = [str(s) for o, s in rc.suggestions(kind, flags) if o.dims[5 if kind == rc.RC_OP_ATTENTION_PACKED else 4] == d]
    assert len(texts) >= 6
    for text in texts:
        if kind == rc.RC_OP_ATTENTION_PAGED:
            got = run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)])
        else:
            got = run_packed(op, text, ins, starts(q), at)
        check(got, want, tol)


@pytest.mark.parametrize("flags", [C, I8 | C])
@pytest.mark.parametrize("case", [([1], [9000], 1, 4, 64, 16), ([1] * 40, [700 + 61 * i for i in range(40)], 2, 16, 64, 16),
                                  ([90, 1, 0, 1], [2500, 4000, 5, 31], 2, 8, 64, 64)])
def test_many_pieces(case, flags):
    # one row, joined by rows; 1280 and 2944 rows' pieces: by rows and by blocks
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 21)
    keys, _ = keys_of(cache, table, lens, page, flags & I8)
    want, tol = reference(q, lens, f64(rows), keys, True, d ** -0.5)
    for text in S.legal(op, ["waves=4,splits=2", "waves=1,splits=4", "block_m=64,waves=8,stages=3,occ=2,splits=4",
                             "block_m=128,waves=4,stages=3,occ=2,splits=2"]):
        check(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]), want, tol)


@pytest.mark.parametrize("flags", [C, I8 | C])
def test_long_pieces_of_uneven_sequences(flags):
    # 25,000 tiles of 32 keys and heads over 256 workgroups: pieces of 98, which are
    # more than a round, and halved
    r = np.random.default_rng(22)
    lens = r.integers(16, 2000, 90).tolist() + [6000, 5000]
    case = ([1] * 92, lens, 8, 1, 64, 64)
    assert 64 * 256 < sum(-(-n // 32) for n in lens) * 8 < 98 * 2 * 256
    op = S.paged_op(case, flags)
    rows, cache, table = paged_inputs(case, flags & I8, 23)
    keys, _ = keys_of(cache, table, lens, 64, flags & I8)
    want, tol = reference(case[0], lens, f64(rows), keys, True, 64 ** -0.5)
    for text in ("waves=4,splits=1", "waves=1,splits=1", "waves=4,occ=2,splits=2"):
        check(run_paged(op, text, rows, cache, [ints(range(93)), ints(lens), ints(table)]), want, tol)


def test_thousands_of_sequences():
    r = np.random.default_rng(30)
    q = r.integers(0, 3, 5000).tolist()
    lens = [n + int(m) for n, m in zip(q, r.integers(0, 20, 5000))]
    q[4321], lens[4321], q[70], lens[70] = 100, 400, 40, 40
    case = (q, lens, 1, 2, 64, 16)
    op = S.paged_op(case, C)
    rows, cache, table = paged_inputs(case, 0, 31)
    keys, _ = keys_of(cache, table, lens, 16, 0)
    want, tol = reference(q, lens, f64(rows), keys, True, 64 ** -0.5)
    for text in S.legal(op, ["", "waves=4,splits=2", "block_m=128,waves=4,stages=3,occ=2,splits=2"]):
        check(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]), want, tol)


@pytest.mark.parametrize("b", [64, 65, 256, 257, 4097])
def test_sequences_on_either_side_of_what_is_scanned(b):
    # up to 256 sequences are gone through, more are searched; rows of some, of
    # the first and of the last alone, and offsets that make no sense
    r = np.random.default_rng(b)
    op = rc.Op(rc.RC_OP_ATTENTION_PACKED, (200, 200, b, 3, 1, 64), C)
    ins = packed_inputs(([200], [200], 1, 3, 64), b)
    some = np.zeros(b, np.int64)
    np.add.at(some, r.integers(0, b, 150), 1)
    some[b // 2] += 50
    first, last = np.zeros(b, np.int64), np.zeros(b, np.int64)
    first[0], last[-1] = 190, 200
    for q in (some, first, last):
        q = q.tolist()
        at = starts(q)
        keys = [[f64(x)[at[i]:at[i + 1]] for x in ins[1:]] for i in range(b)]
        n = at[-1]
        want, tol = reference(q, q, f64(ins[0])[:n], keys, True, 64 ** -0.5)
        for text in S.legal(op, ["", "waves=4,splits=2", "block_m=64,waves=8,stages=3,occ=2", "block_m=128,waves=4,stages=3,occ=2"]):
            check(run_packed(op, text, ins, at, at)[:n], want, tol)
    for offsets in (r.integers(-2 ** 31, 2 ** 31, b + 1), r.integers(0, 200, b + 1), np.arange(b + 1)[::-1]):
        for text in S.legal(op, ["", "waves=4,splits=2", "block_m=64,waves=8,stages=3,occ=2", "block_m=128,waves=4,stages=3,occ=2"]):
            run_packed(op, text, ins, offsets.tolist(), offsets.tolist())


def test_sequences_that_share_pages():
    # the same first pages in two tables, and one page twice in a table
    case = ([3, 40], [40, 75], 2, 4, 128, 16)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, C)
    rows, cache, table = paged_inputs(case, 0, 33)
    table[1, :2], table[1, 3] = table[0, :2], table[1, 2]
    keys, _ = keys_of(cache, table, lens, page, 0)
    want, tol = reference(q, lens, f64(rows), keys, True, d ** -0.5)
    for text in S.legal(op, S.ATTENTION_TEXTS):
        check(run_paged(op, text, rows, cache, [ints(starts(q)), ints(lens), ints(table)]), want, tol)


@pytest.mark.parametrize("i8", [0, I8])
def test_a_cache_past_32_bits(i8):
    # pages on both sides of 2^32 elements of K and of V; what is in no page that
    # the table names is not initialised
    hkv, g, d, page, pages, q, lens = 8, 2, 128, 64, 66000, [300, 1], [330, 1000]
    assert pages * hkv * page * d > 2 ** 32
    ids = [pages - 1 - i for i in range(12)] + list(range(10))
    table = np.full((2, 16), -1, np.int64)
    table[0, :6], table[1, :16] = ids[:6], ids[6:]
    dims = (301, 2, hkv, d, page, pages, 16)
    r = np.random.default_rng(40)
    cache = [torch.empty(pages, hkv, page, d, dtype=torch.int8 if i8 else torch.bfloat16, device="cuda") for _ in range(2)]
    if i8:
        cache += [torch.empty(pages, hkv, page, device="cuda") for _ in range(2)]
    where = [ints(starts(lens)).cuda(), ints(lens).cuda(), ints(table).cuda()]
    kv = [bf16(r.standard_normal((sum(lens), hkv, d))).cuda() for _ in range(2)]
    for kind, ins, out in ((rc.RC_OP_KV_WRITE, kv, cache), (rc.RC_OP_KV_READ, cache, [torch.zeros_like(x) for x in kv])):
        op = rc.Op(kind, (sum(lens),) + dims[1:], i8)
        print(f"[gpu] kind={kind} dims={op.dims} flags={i8}", flush=True)
        rc.Plan(op, op.suggest()).launch(ins + where, tuple(out))
        torch.cuda.synchronize()
    want = [f64(x) for x in kv]
    if i8:
        want = [y * s.astype(np.float64)[..., None] for y, s in map(quantised, want)]
    for x, y in zip(out, want):
        assert same(x, f64(bf16(y)))
    at = starts(lens)
    keys = [[x[at[b]:at[b + 1]] for x in want] for b in range(2)]
    rows = bf16(r.standard_normal((301, hkv * g, d)))
    op = rc.Op(rc.RC_OP_ATTENTION_PAGED, (301, 2, hkv * g, hkv, d, page, pages, 16), i8 | C)
    want, tol = reference(q, lens, f64(rows), keys, True, d ** -0.5)
    for text in S.legal(op, ["waves=4,splits=2", "block_m=64,waves=8,stages=3,occ=2,splits=4",
                             "block_m=128,waves=4,stages=3,occ=2,splits=2"]):
        print(f"[gpu] paged dims={op.dims} flags={op.flags} sched={text}", flush=True)
        plan, got = rc.Plan(op, op.from_string(text)), torch.empty(301, hkv * g, d, dtype=torch.bfloat16, device="cuda")
        plan.launch([rows.cuda()] + cache + [ints(starts(q)).cuda()] + where[1:], got, plan.workspace())
        torch.cuda.synchronize()
        check(got, want, tol)


def test_packed_rows_past_32_bits():
    # 140000 sequences of one token: each row of O, of 2^32 bytes and more, is V's
    t, h, hkv, d = 140000, 128, 8, 128
    assert t * h * d * 2 > 2 ** 32
    op = rc.Op(rc.RC_OP_ATTENTION_PACKED, (t, t, t, h, hkv, d), C)
    q, out = (torch.zeros(t, h, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.randn(t, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = torch.arange(t + 1, dtype=torch.int32, device="cuda")
    for text in S.legal(op, ["waves=4"]):
        print(f"[gpu] packed dims={op.dims} flags={op.flags} sched={text}", flush=True)
        plan = rc.Plan(op, op.from_string(text))
        plan.launch([q, k, v, at, at], out.zero_(), plan.workspace())
        for i in range(0, t, 10000):
            part = out[i:i + 10000].view(-1, hkv, h // hkv, d)
            assert bool((part == v[i:i + 10000, :, None]).all())


def test_one_plan_on_two_streams():
    case = ([1] * 6, [3000, 1, 500, 64, 2000, 77], 2, 4, 64, 16)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, C)
    plan = rc.Plan(op, op.suggest())
    assert plan.workspace_bytes > 0
    sets, streams = [paged_inputs(case, 0, 50 + i) for i in range(2)], [torch.cuda.Stream() for _ in range(2)]
    dev = [[x.cuda() for x in [rows] + cache + [ints(starts(q)), ints(lens), ints(table)]] for rows, cache, table in sets]
    outs, ws = [torch.empty_like(x[0]) for x in dev], [plan.workspace() for _ in dev]
    torch.cuda.synchronize()
    for i in (0, 1) * 3:
        plan.launch(dev[i], outs[i], ws[i], streams[i])
    torch.cuda.synchronize()
    for (rows, cache, table), out in zip(sets, outs):
        keys, _ = keys_of(cache, table, lens, page, 0)
        check(out, *reference(q, lens, f64(rows), keys, True, d ** -0.5))


def test_launch_without_allocation():
    case = ([5, 1, 20], [40, 33, 20], 2, 4, 64, 16)
    q, lens, hkv, g, d, page = case
    op = S.paged_op(case, C)
    rows, cache, table = paged_inputs(case, 0, 60)
    ins = [x.cuda() for x in [rows] + cache + [ints(starts(q)), ints(lens), ints(table)]]
    plan = rc.Plan(op, op.from_string("waves=4"))
    outs = [torch.empty_like(ins[0]) for _ in range(2)]
    plan.launch(ins, outs[0], plan.workspace())
    plan.launch_static(ins, outs[1])
    torch.cuda.synchronize()
    assert torch.equal(*outs)


# ---------------------------------------------------------------------------
# The operators together
# ---------------------------------------------------------------------------

class Step:
    """A serving step of `rows` tokens: their K and V into the cache, then their
    attention over it."""

    def __init__(self, b, rows, hkv, g, d, page, width, i8, seed):
        self.dims, self.i8, self.g = (rows, b, hkv, d, page, b * width + 1, width), i8, g
        write = rc.Op(rc.RC_OP_KV_WRITE, self.dims, i8)
        read = rc.Op(rc.RC_OP_ATTENTION_PAGED, (rows, b, hkv * g, hkv, d) + self.dims[4:], i8 | C)
        self.plans = [rc.Plan(op, op.suggest()) for op in (write, read)]
        self.ws = [p.workspace() for p in self.plans]
        r = np.random.default_rng(seed)
        pages = self.dims[5]
        self.table = ints(r.permutation(pages)[:b * width].reshape(b, width)).cuda()
        dtype = torch.int8 if i8 else torch.bfloat16
        self.cache = [torch.zeros(pages, hkv, page, d, dtype=dtype, device="cuda") for _ in range(2)]
        if i8:
            self.cache += [torch.zeros(pages, hkv, page, device="cuda") for _ in range(2)]
        self.q = torch.zeros(rows, hkv * g, d, dtype=torch.bfloat16, device="cuda")
        self.k, self.v = (torch.zeros(rows, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.offsets, self.lens = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (b + 1, b))
        self.out = torch.zeros_like(self.q)
        self.said = [[np.zeros((0, hkv, d))] * 2 for _ in range(b)]
        self.r = r

    def feed(self, counts):
        """New inputs of a step with `counts` tokens of each sequence."""
        rows, b, hkv, d = self.dims[:4]
        for x in (self.q, self.k, self.v):
            x.copy_(bf16(self.r.standard_normal(tuple(x.shape))))
        at = starts(counts)
        new = [f64(self.k), f64(self.v)]
        for i in range(b):
            for j in range(2):
                x = new[j][at[i]:at[i + 1]]
                if self.i8:
                    y, scale = quantised(x)
                    x = y * scale.astype(np.float64)[..., None]
                self.said[i] = list(self.said[i])
                self.said[i][j] = np.concatenate([self.said[i][j], x])
        self.offsets.copy_(ints(at))
        self.lens.copy_(ints([len(s[0]) for s in self.said]))
        self.out.fill_(float("nan"))
        return reference(counts, [len(s[0]) for s in self.said], f64(self.q), self.said, True, d ** -0.5)

    def launch(self, stream=None):
        self.plans[0].launch([self.k, self.v, self.offsets, self.lens, self.table], tuple(self.cache), self.ws[0], stream)
        self.plans[1].launch([self.q] + self.cache + [self.offsets, self.lens, self.table], self.out, self.ws[1], stream)


STEPS = [[7, 0, 1], [1, 1, 6], [3, 4, 1], [8, 0, 0], [1, 1, 1]]


@pytest.mark.parametrize("i8", [0, I8])
def test_steps(i8):
    step = Step(3, 8, 2, 4, 128, 16, 6, i8, 1)
    for counts in STEPS * 2:
        want, tol = step.feed(counts)
        step.launch()
        torch.cuda.synchronize()
        n = sum(counts)
        check(step.out[:n], want[:n], tol[:n])
        assert bool(torch.isnan(step.out[n:]).all())


@pytest.mark.parametrize("i8", [0, I8])
def test_captured_steps(i8):
    # two graphs with a workspace each, replayed on two streams with other
    # lengths each time
    steps = [Step(3, 8, 2, 4, 64, 16, 6, i8, s) for s in (2, 3)]
    graphs, streams = [torch.cuda.CUDAGraph() for _ in steps], [torch.cuda.Stream() for _ in steps]
    for step, graph in zip(steps, graphs):
        step.launch()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step.launch()
    for counts in STEPS * 2:
        want = [step.feed(counts) for step in steps]
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        n = sum(counts)
        for step, (y, tol) in zip(steps, want):
            check(step.out[:n], y[:n], tol[:n])
            eager = step.out.clone()
            step.launch()
            torch.cuda.synchronize()
            assert torch.equal(eager[:n], step.out[:n])


def test_a_prompt_through_the_cache_and_packed():
    # packed attention of prompts, and the same from the cache that they were
    # written to; read back they are what was written
    case = ([33, 100, 1], [33, 100, 1], 2, 4, 128)
    q, k, hkv, g, d = case
    ins = [x.cuda() for x in packed_inputs(case, 7)]
    offsets, lens = ints(starts(q)).cuda(), ints(q).cuda()
    table = ints(np.random.default_rng(0).permutation(30).reshape(3, 10)).cuda()
    cache = [torch.zeros(30, hkv, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    dims = (sum(q), 3, hkv, d, 16, 30, 10)
    outs = [torch.zeros_like(ins[0]) for _ in range(2)]
    back = [torch.zeros_like(x) for x in ins[1:]]

    def launch(kind, dims, flags, inputs, out):
        op = rc.Op(kind, dims, flags)
        plan = rc.Plan(op, op.suggest())
        plan.launch(inputs, out, plan.workspace())

    launch(rc.RC_OP_KV_WRITE, dims, 0, ins[1:] + [offsets, lens, table], tuple(cache))
    launch(rc.RC_OP_KV_READ, dims, 0, cache + [offsets, lens, table], tuple(back))
    launch(rc.RC_OP_ATTENTION_PAGED, (sum(q), 3, hkv * g) + dims[2:], C, ins[:1] + cache + [offsets, lens, table], outs[0])
    launch(rc.RC_OP_ATTENTION_PACKED, (sum(q), sum(k), 3, hkv * g, hkv, d), C, ins + [offsets, offsets], outs[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(back, ins[1:]))
    at = starts(k)
    keys = [[f64(x)[at[b]:at[b + 1]] for x in ins[1:]] for b in range(3)]
    want, tol = reference(q, k, f64(ins[0]), keys, True, d ** -0.5)
    for out in outs:
        check(out, want, tol)


def test_refused_launches():
    case = ([1, 1], [20, 30], 1, 2, 64, 16)
    op = S.paged_op(case, C)
    rows, cache, table = paged_inputs(case, 0, 5)
    plan = rc.Plan(op, op.suggest())
    ins = [x.cuda() for x in [rows] + cache + [ints([0, 1, 2]), ints([20, 30]), ints(table)]]
    out = torch.empty_like(ins[0])
    ws = plan.workspace()
    plan.launch(ins, out, ws)
    for i in range(len(ins)):
        for bad in (ins[i].cpu(), ins[i][:-1], ins[i].to(torch.float64), torch.stack([ins[i]] * 2, -1)[..., 0]):
            with pytest.raises(ValueError):
                plan.launch(ins[:i] + [bad] + ins[i + 1:], out, ws)
    with pytest.raises(rc.RCError) as e:
        plan.launch(ins, ins[0], ws)
    assert e.value.status == rc.RC_ERR_INVALID_ARGUMENT and "overlaps" in str(e.value)
    torch.cuda.synchronize()
