"""GPU tests of the 8-bit integer operators against 64-bit references.

Integers are compared for equality.  Tolerances of the others, with u = 2^-24
(half a step of fp32, relative):
  scale   the norm's sum of squares adds at most n = cols / 64 terms in a
          lane, then 6 + 15 across lanes and waves: (n + 21) u, halved by the
          root; the mean, eps, root, the two divisions and a add 5 u.
  h       exact: the sum of two bf16 is exact in fp32 or within 2^-16 of the
          larger, so its bf16 is that of the true sum.
  product float(acc), sa * sb and their product: 3 u of |acc sa sb|; the
          bias's sum: u of the result and of what went in; the output's
          rounding 2^-8 (bf16, half a step of a value just above a power of
          two) or none (fp32).
  gated   g and u carry 3 u each; SiLU multiplies a relative error of g by at
          most 1 + |g|, and its exponential has |g| u from the product with
          log2 e, 2 u of its own, then a sum, a reciprocal (2 u) and a
          product: (4 |g| + 9) u, the product with u one u more.
"""
import math
import os

import numpy as np
import pytest

from paper_2506_01374_amd import rc

import cases_i8
from cases_i8 import B, F, G, R

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = 2.0 ** -24
BF16 = 2.0 ** -8
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    rc.set_cache_dir(os.path.join(ROOT, "paper_2506_01374_amd", "jit_cache"))
    torch.cuda.set_device(0)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def bf16(a):
    """float64 -> bfloat16 (through fp32, which holds the sum of two)."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.float32).to(torch.bfloat16)


# ---------------------------------------------------------------------------
# Rows to int8
# ---------------------------------------------------------------------------

def rows_reference(x, w=None, r=None, eps=EPS):
    """(q, scale, h) in 64 bits; q of a row whose scale is not finite is 0."""
    h = x if r is None else f64(bf16(x + r))
    with np.errstate(all="ignore"):
        p = h if w is None else h * w
        a = np.abs(p).max(axis=1)
        q = np.rint(127 * p / a[:, None])
        scale = a / 127
        if w is not None:
            ss = (h * h).sum(axis=1)
            scale = scale / np.sqrt(ss / x.shape[1] + eps)
            scale = np.where(ss < 2.0 ** 128, scale, np.nan)
    scale = np.where(a == 0, 0.0, np.where(np.isfinite(a), scale, np.nan))
    q = np.where(np.isfinite(scale)[:, None] & (a > 0)[:, None], q, 0).astype(np.int8)
    return q, scale, h


GUARD = 32


def guarded(shape, dtype):
    """A tensor of `shape` inside a buffer whose ends are checked."""
    n = math.prod(shape)
    buf = torch.full((n + 2 * GUARD,), 77, dtype=dtype, device="cuda")
    t = buf[GUARD:GUARD + n].view(shape)
    return buf, t


def intact(buf):
    return bool((buf[:GUARD] == 77).all()) and bool((buf[-GUARD:] == 77).all())


def run_rows(kind, flags, x, w, r, text=None, eps=EPS, alias=None):
    t, c = x.shape
    op = rc.Op(kind, (t, c), flags, eps=eps if kind == rc.RC_OP_RMSNORM_I8 else None)
    sched = op.from_string(text) if text is not None else op.suggest()
    print(f"[gpu] kind={kind} flags={flags} dims={(t, c)} sched={sched}", flush=True)
    ins = [bf16(x).cuda()] + ([bf16(w).cuda()] if w is not None else []) + ([bf16(r).cuda()] if r is not None else [])
    bufs = [guarded((t, c), torch.int8), guarded((t,), torch.float32)]
    if r is not None:
        bufs.append(guarded((t, c), torch.bfloat16) if alias is None else (None, ins[alias]))
    plan = rc.Plan(op, sched)
    plan.launch(ins, tuple(b[1] for b in bufs), plan.workspace())
    torch.cuda.synchronize()
    for buf, _ in bufs:
        assert buf is None or intact(buf)
    return [b[1] for b in bufs]


def check_rows(kind, flags, x, w=None, r=None, text=None, eps=EPS, alias=None):
    q, scale, h = rows_reference(x, w, r, eps)
    got = run_rows(kind, flags, x, w, r, text, eps, alias)
    assert np.array_equal(got[0].cpu().numpy(), q)
    n = -(-x.shape[1] // 64)
    tol = ((n + 21) / 2 + 5) * U if w is not None else U
    s = f64(got[1])
    assert np.array_equal(np.isnan(s), np.isnan(scale))
    ok = ~np.isnan(s)
    # (a scale below fp32's normal range has its absolute step)
    assert np.all(np.abs(s - scale)[ok] <= tol * scale[ok] + 2.0 ** -149), np.max(np.abs(s - scale)[ok] / scale[ok])
    if r is not None:
        assert np.array_equal(f64(got[2]), h, equal_nan=True)


def rows_inputs(t, c, seed):
    g = np.random.default_rng(seed)
    far = np.where(g.random(c) < 0.02, 20.0, 1.0)
    x, r = (f64(bf16(g.standard_normal((t, c)) * far)) for _ in range(2))
    w = f64(bf16(1 + 0.3 * g.standard_normal(c)))
    return x, w, r


@pytest.mark.parametrize("job", range(len(cases_i8.rows_jobs())))
def test_rows(job):
    (t, c), text = cases_i8.rows_jobs()[job]
    x, w, r = rows_inputs(t, c, 100 + job)
    check_rows(rc.RC_OP_QUANT_I8, 0, x, text=text)
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x, w, text=text)
    check_rows(rc.RC_OP_RMSNORM_I8, R, x, w, r, text=text)


ROWS_EDGE_TEXTS = ["", "vec=8,waves=2,held=1", "vec=8,rows=4,held=2"]


@pytest.mark.parametrize("text", ROWS_EDGE_TEXTS)
def test_rows_of_zeros_nan_and_infinity(text):
    x, w, r = rows_inputs(12, 700, 1)
    x[0] = 0
    x[1, 699], x[2, 3], x[3, 0], x[4, 5] = np.nan, np.inf, -np.inf, 0
    x[5] = 0
    x[5, 100] = -3e-39                      # one value, below the normal range
    x[6, 7] = 3e38                          # the square leaves fp32
    x[7] *= 2.0 ** -130
    x[8] *= 2.0 ** 100
    x = f64(bf16(x))
    check_rows(rc.RC_OP_QUANT_I8, 0, x, text=text)
    ones = np.ones(700)
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x, ones, text=text)
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x, ones, text=text, eps=2.0 ** -100)
    w[:] = 0
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x[9:], w, text=text)
    w[3] = np.inf
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x[9:], w, text=text)
    x, w, r = rows_inputs(3, 700, 2)
    r[0], r[1, 2] = -x[0], np.nan           # the sum is zero; the sum is NaN
    check_rows(rc.RC_OP_RMSNORM_I8, R, x, w, r, text=text)


@pytest.mark.parametrize("text", ROWS_EDGE_TEXTS)
def test_quotients_at_and_next_to_a_half(text):
    # a = 127 m: the quotients are x / m, so that halves are hit exactly (where
    # 127 m has eight bits), and one step of bf16 to either side of them
    rows = []
    for m in (1.0, 2.0, 0.5, 3.0, 1.5, 2.0 ** -70, 2.0 ** 70):
        halves = (np.arange(-126, 127) + 0.5) * m
        x = f64(bf16(halves))
        near = np.concatenate([x, f64(bf16(x * (1 + 2.0 ** -7))), f64(bf16(x * (1 - 2.0 ** -7)))])
        near[np.abs(near) > 127 * m] = 0
        rows.append(np.concatenate([[127 * m], near]))
    x = f64(bf16(np.stack(rows)))           # (127 * 3 has nine bits: the device sees it rounded)
    check_rows(rc.RC_OP_QUANT_I8, 0, x, text=text)
    # a product of two significands has more digits: 127 w x near a half
    g = np.random.default_rng(3)
    w = f64(bf16(1 + g.random(x.shape[1])))
    check_rows(rc.RC_OP_RMSNORM_I8, 0, x[:5], w, text=text)


@pytest.mark.parametrize("alias", [0, 2])
@pytest.mark.parametrize("text", ["", "vec=8,waves=4,held=2", "vec=8", "vec=8,waves=2"])
def test_residual_stream_in_place(alias, text):
    x, w, r = rows_inputs(9, 3000, 4)
    check_rows(rc.RC_OP_RMSNORM_I8, R, x, w, r, text=text, alias=alias)


# ---------------------------------------------------------------------------
# The matrix product
# ---------------------------------------------------------------------------

def gemm_inputs(dims, flags, seed, extreme=False):
    m, n, k = dims
    g = np.random.default_rng(seed)

    def ints(rows):
        if extreme:
            return np.full((rows, k), -128, np.int8)
        return g.integers(-128, 128, (rows, k), dtype=np.int8)

    ins = [ints(m), (0.5 + g.random(m)) / 64, ints(n), (0.5 + g.random(n)) / 512]
    if flags & B:
        ins.append(g.standard_normal(n))
    if flags & G:
        ins += [ints(n), (0.5 + g.random(n)) / 512]
    if flags & G:
        # g from far below to far above zero
        ins[3] *= 8 / max(1.0, math.sqrt(k))
        ins[5] *= 8 / max(1.0, math.sqrt(k))
    return [torch.from_numpy(x if x.dtype == np.int8 else x.astype(np.float32)) for x in ins]


def gemm_reference(ins, flags):
    """The exact result and the bound of its error, in 64 bits."""
    d = [f64(x) for x in ins]
    y = d[0] @ d[2].T * d[1][:, None] * d[3][None, :]
    if flags & G:
        u = d[0] @ d[4].T * d[1][:, None] * d[5][None, :]
        with np.errstate(over="ignore"):
            out = y / (1 + np.exp(-y)) * u
        rel = (4 * np.abs(y) + 9 + 3 * (1 + np.abs(y)) + 3 + 1) * U
        return out, np.abs(out) * (BF16 + 2 * rel)
    err = 3 * U * np.abs(y)
    if flags & B:
        y = y + d[4][None, :]
        err += U * np.abs(y)
    return y, err * 1.01 + (0 if flags & F else BF16 * np.abs(y))


def run_gemm(dims, flags, ins, text=None):
    m, n, k = dims
    op = rc.Op(rc.RC_OP_GEMM_I8, dims, flags)
    sched = op.from_string(text) if text is not None else op.suggest()
    print(f"[gpu] gemm_i8 flags={flags} dims={dims} sched={sched}", flush=True)
    buf, out = guarded((m, n), torch.float32 if flags & F else torch.bfloat16)
    plan = rc.Plan(op, sched)
    plan.launch([x.cuda() for x in ins], out, plan.workspace())
    torch.cuda.synchronize()
    assert intact(buf)
    return out


def check_gemm(dims, flags, seed, text=None, extreme=False):
    ins = gemm_inputs(dims, flags, seed, extreme)
    want, tol = gemm_reference(ins, flags)
    got = f64(run_gemm(dims, flags, ins, text))
    # (a gated value below bf16's normal range has its absolute step)
    assert np.all(np.abs(got - want) <= tol + 2.0 ** -133), np.max(np.abs(got - want) - tol)


@pytest.mark.parametrize("flags", [0, B, F, B | F, G])
@pytest.mark.parametrize("dims", cases_i8.GEMM_DIMS)
def test_gemm(dims, flags):
    for i, (_, text) in enumerate(j for j in cases_i8.gemm_jobs(flags) if j[0] == dims):
        check_gemm(dims, flags, 7 * i + flags, text)


@pytest.mark.parametrize("flags", [0, B | F, G])
def test_gemm_with_half_height_tiles(flags):
    jobs = cases_i8.tail_jobs(flags)
    assert len(jobs) == len(cases_i8.TAIL_DIMS) + len(cases_i8.TAIL_WIDE_DIMS) + 1
    for i, (dims, text) in enumerate(jobs):
        check_gemm(dims, flags, 300 + i, text)


@pytest.mark.parametrize("dims", [(3, 40, 131071), (200, 200, 131056), (20, 70, 131071)])
def test_sums_at_the_limit_of_int32(dims):
    # every product is 128 * 128: 131071 of them are 2^31 - 2^14
    check_gemm(dims, F, 1, extreme=True)
    check_gemm(dims, 0, 2)


@pytest.mark.parametrize("job", range(len(cases_i8.LARGE)))
def test_offsets_past_32_bits(job):
    (m, n, k), knobs = cases_i8.LARGE[job]
    op = rc.Op(rc.RC_OP_GEMM_I8, (m, n, k))
    sched = op.schedule(**knobs)
    assert sched.validate() == "", sched.validate()
    print(f"[gpu] gemm_i8 dims={op.dims} sched={sched}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(job)
    a, b = (torch.randint(-128, 128, (x, k), generator=g, device="cuda", dtype=torch.int8) for x in (m, n))
    sa, sb = (torch.rand(x, generator=g, device="cuda") for x in (m, n))
    out = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    plan = rc.Plan(op, sched)
    plan.launch([a, sa, b, sb], out, plan.workspace())
    torch.cuda.synchronize()
    rows, cols = (torch.tensor(sorted({0, 1, x // 3, x // 2 + 1, x - 2, x - 1})) for x in (m, n))
    ins = [t[i.cuda()].cpu() for t, i in ((a, rows), (sa, rows), (b, cols), (sb, cols))]
    want, tol = gemm_reference(ins, 0)
    assert np.all(np.abs(f64(out[rows.cuda()][:, cols.cuda()]) - want) <= tol)
    # nothing is left out (a product of random rows is never NaN)
    for r in range(0, m, 8192):
        assert not out[r:r + 8192].isnan().any()


def test_rows_past_32_bits():
    t, c, block = 600 * 1024, 8192, 1024
    x, w, r = rows_inputs(block, c, 9)
    q, scale, h = rows_reference(x, w, r)
    dx, dr = (bf16(v).cuda().repeat(t // block, 1) for v in (x, r))
    op = rc.Op(rc.RC_OP_RMSNORM_I8, (t, c), R, eps=EPS)
    plan = rc.Plan(op, op.suggest())
    dq, ds = torch.empty(t, c, dtype=torch.int8, device="cuda"), torch.empty(t, device="cuda")
    print(f"[gpu] rows dims={op.dims}", flush=True)
    plan.launch([dx, bf16(w).cuda(), dr], (dq, ds, dx), None)          # h in place of x
    torch.cuda.synchronize()
    want_q, want_h = torch.from_numpy(q).cuda(), bf16(h).cuda()
    for i in range(0, t, block):
        assert torch.equal(dq[i:i + block], want_q) and torch.equal(dx[i:i + block], want_h)
    assert torch.equal(ds.view(-1, block), ds[:block].expand(t // block, block))
    assert np.all(np.abs(f64(ds[:block]) - scale) <= ((c / 64 + 21) / 2 + 5) * U * scale)


def test_scales_that_are_not_finite_or_zero():
    dims = (40, 70, 200)
    ins = gemm_inputs(dims, F, 5)
    ins[1][3], ins[1][5], ins[1][7], ins[3][9] = float("nan"), float("inf"), 0.0, float("nan")
    got = f64(run_gemm(dims, F, ins))
    d = [f64(x) for x in ins]
    with np.errstate(invalid="ignore"):
        want = (d[0] @ d[2].T) * (d[1][:, None] * d[3][None, :])
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    ok = np.isfinite(want)
    assert np.all(np.abs(got - want)[ok] <= 3.1 * U * np.abs(want)[ok])


# ---------------------------------------------------------------------------
# As they are used
# ---------------------------------------------------------------------------

class Block:
    """The int8 gated MLP of a decoder layer on t tokens: residual and norm,
    gate and up products, quantisation of the hidden rows, down product."""

    def __init__(self, t, hd, inner, seed):
        g = np.random.default_rng(seed)
        self.dims = t, hd, inner
        self.x, self.r = (bf16(g.standard_normal((t, hd))).cuda() for _ in range(2))
        self.w = bf16(1 + 0.2 * g.standard_normal(hd)).cuda()
        self.weights = []
        for rows, k in ((inner, hd), (inner, hd), (hd, inner)):
            f = g.standard_normal((rows, k)) / math.sqrt(k)
            s = np.abs(f).max(1) / 127
            self.weights += [torch.from_numpy(np.rint(f / s[:, None]).astype(np.int8)).cuda(),
                             torch.from_numpy(s.astype(np.float32)).cuda()]
        ops = [rc.Op(rc.RC_OP_RMSNORM_I8, (t, hd), R, eps=EPS), rc.Op(rc.RC_OP_GEMM_I8, (t, inner, hd), G),
               rc.Op(rc.RC_OP_QUANT_I8, (t, inner)), rc.Op(rc.RC_OP_GEMM_I8, (t, hd, inner))]
        self.plans = [rc.Plan(op, op.suggest()) for op in ops]
        self.ws = [p.workspace() for p in self.plans]

        def empty(dtype, *shape):
            return torch.empty(shape, dtype=dtype, device="cuda")

        i8, f32, b16 = torch.int8, torch.float32, torch.bfloat16
        self.q, self.s, self.h = empty(i8, t, hd), empty(f32, t), empty(b16, t, hd)
        self.g, self.gq, self.gs, self.out = empty(b16, t, inner), empty(i8, t, inner), empty(f32, t), empty(b16, t, hd)

    def step(self, stream=None):
        w = self.weights
        norm, up, quant, down = self.plans
        norm.launch([self.x, self.w, self.r], (self.q, self.s, self.h), self.ws[0], stream)
        up.launch([self.q, self.s, *w[:4]], self.g, self.ws[1], stream)
        quant.launch([self.g], (self.gq, self.gs), self.ws[2], stream)
        down.launch([self.gq, self.gs, *w[4:]], self.out, self.ws[3], stream)

    def outputs(self):
        return [self.q, self.s, self.h, self.g, self.gq, self.gs, self.out]

    def check(self):
        """Each step against 64 bits from the values that went into it."""
        q, scale, h = rows_reference(f64(self.x), f64(self.w), f64(self.r))
        assert np.array_equal(self.q.cpu().numpy(), q) and np.array_equal(f64(self.h), h)
        w = [x.cpu() for x in self.weights]
        want, tol = gemm_reference([self.q.cpu(), self.s.cpu(), w[0], w[1], w[2], w[3]], G)
        assert np.all(np.abs(f64(self.g) - want) <= tol)
        gq, gs, _ = rows_reference(f64(self.g))
        assert np.array_equal(self.gq.cpu().numpy(), gq)
        want, tol = gemm_reference([self.gq.cpu(), self.gs.cpu(), w[4], w[5]], 0)
        assert np.all(np.abs(f64(self.out) - want) <= tol)
        # and the whole layer against the float weights' layer, in 64 bits: 8
        # bits leave about a percent
        d = [f64(x) for x in w]
        y = h * f64(self.w) / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
        a, u = (y @ (d[i] * d[i + 1][:, None]).T for i in (0, 2))
        full = (a / (1 + np.exp(-a)) * u) @ (d[4] * d[5][:, None]).T
        assert np.linalg.norm(f64(self.out) - full) <= 0.05 * np.linalg.norm(full)


@pytest.mark.parametrize("t,hd,inner", [(1, 256, 512), (7, 250, 333), (200, 512, 1024)])
def test_a_layer_of_them(t, hd, inner):
    layer = Block(t, hd, inner, t)
    layer.step()
    torch.cuda.synchronize()
    layer.check()


@pytest.mark.parametrize("t", [3, 150])
def test_a_captured_layer(t):
    layer = Block(t, 320, 640, 30 + t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.step()
    g = np.random.default_rng(t)
    for _ in range(3):
        for x in (layer.x, layer.r):
            x.copy_(bf16(g.standard_normal(tuple(x.shape))))
        layer.step()
        want = [x.clone() for x in layer.outputs()]
        for x in layer.outputs():
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(layer.outputs(), want):
            assert torch.equal(x, y)
    layer.check()


def test_two_layers_on_two_streams():
    layers = [Block(t, 320, 640, 60 + t) for t in (40, 70)]
    streams = [torch.cuda.Stream() for _ in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for layer, stream in zip(layers, streams):
            layer.step(stream)
    torch.cuda.synchronize()
    for layer in layers:
        layer.check()


def test_one_plan_on_two_streams():
    dims = (100, 256, 512)
    op = rc.Op(rc.RC_OP_GEMM_I8, dims)
    plan = rc.Plan(op, op.suggest())
    ins = [gemm_inputs(dims, 0, 80 + i) for i in range(2)]
    dev = [[x.cuda() for x in i] for i in ins]
    outs = [torch.empty(dims[:2], dtype=torch.bfloat16, device="cuda") for _ in ins]
    ws = [plan.workspace() for _ in ins]
    streams = [torch.cuda.Stream() for _ in ins]
    torch.cuda.synchronize()
    for i in (0, 1, 0, 1):
        plan.launch(dev[i], outs[i], ws[i], streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        want, tol = gemm_reference(ins[i], 0)
        assert np.all(np.abs(f64(outs[i]) - want) <= tol)


def test_captured_products_of_three_launches():
    # copied rows, the ring on two K splits and their sum: two graphs with a
    # workspace each, replayed on two streams and next to eager launches
    dims, flags = (130, 200, 1001), B
    op = rc.Op(rc.RC_OP_GEMM_I8, dims, flags)
    text = "tile_m=64,tile_n=64,tile_k=128,waves_m=2,waves_n=2,mfma=16,stages=2,order=1,splits=2,pad=1"
    plan = rc.Plan(op, op.from_string(text))
    assert plan.nkernels == 3 and plan.dominant == 1
    sets = []
    for i in range(2):
        ins = gemm_inputs(dims, flags, 90 + i)
        sets.append((ins, [x.cuda() for x in ins], torch.empty(dims[:2], dtype=torch.bfloat16, device="cuda"),
                     plan.workspace(), torch.cuda.CUDAGraph(), torch.cuda.Stream()))
    for _, dev, out, ws, graph, _ in sets:
        plan.launch(dev, out, ws)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            plan.launch(dev, out, ws)
    for turn in range(3):
        for i, (ins, dev, out, ws, _, _) in enumerate(sets):
            ins[:] = gemm_inputs(dims, flags, 100 + 2 * turn + i)
            for x, y in zip(dev, ins):
                x.copy_(y)
            out.zero_()
            ws.fill_(0x55)
        torch.cuda.synchronize()
        for *_, graph, stream in sets:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for ins, dev, out, ws, _, _ in sets:
            want, tol = gemm_reference(ins, flags)
            assert np.all(np.abs(f64(out) - want) <= tol)
            eager = torch.empty_like(out)
            plan.launch(dev, eager, ws)
            torch.cuda.synchronize()
            assert torch.equal(eager, out)


def test_refused_launches():
    op = rc.Op(rc.RC_OP_GEMM_I8, (10, 20, 64))
    plan = rc.Plan(op, op.suggest())
    ins = [x.cuda() for x in gemm_inputs((10, 20, 64), 0, 1)]
    out = torch.empty(10, 20, dtype=torch.bfloat16, device="cuda")
    for bad in ([ins[0].t().contiguous().t(), *ins[1:]], [ins[0].cpu(), *ins[1:]], [ins[0][:9], *ins[1:]], ins[:3],
                [ins[0].to(torch.uint8), *ins[1:]]):
        with pytest.raises(ValueError):
            plan.launch(bad, out, plan.workspace())
        with pytest.raises(ValueError):
            plan.prepare(bad, out, plan.workspace())
        with pytest.raises(ValueError):
            plan.time(bad, out, plan.workspace())
        with pytest.raises(ValueError):
            plan.launch_static(bad, out)
    off = torch.empty(10 * 20 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(10, 20)
    with pytest.raises(rc.RCError) as e:
        plan.launch(ins, off, plan.workspace())
    assert e.value.status == rc.RC_ERR_MISALIGNED
    # an argument block that ends after two outputs, for an operator of three
    op = rc.Op(rc.RC_OP_RMSNORM_I8, (2, 64), R)
    plan = rc.Plan(op, op.suggest())
    x = torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda")
    a = rc.Plan._args([x, x[0], x], (x, x, x))
    a.struct_size -= 16
    assert rc.lib().rc_launch(plan.h, rc.ctypes.byref(a), None, 0, None) == rc.RC_ERR_INVALID_ARGUMENT


def test_static_launch_and_timing():
    dims = (65, 128, 300)
    ins = gemm_inputs(dims, 0, 3)
    want, tol = gemm_reference(ins, 0)
    op = rc.Op(rc.RC_OP_GEMM_I8, dims)
    plan = rc.Plan(op, op.suggest())
    dev = [x.cuda() for x in ins]
    out = torch.empty(dims[:2], dtype=torch.bfloat16, device="cuda")
    plan.launch_static(dev, out)
    torch.cuda.synchronize()
    assert np.all(np.abs(f64(out) - want) <= tol)
    t = plan.time(dev, out, plan.workspace(), warmup=1, repeat=3)
    assert t.median_ms > 0 and t.tflops > 0
