"""Performance cases of the 8-bit integer operators: the root-mean-square norm
with the residual's addition and an int8 output, the quantisation of rows, and
the int8 matrix product with a scale for each token and channel, plain and
gated.

A case is one operator execution on device-resident inputs.  With ``own`` it
runs through the public binding (``rc.Plan.launch``); without, in elementary
torch operations, which is the operators' plain form.  Integers are exact in
both, so they have to be equal.
"""
from __future__ import annotations

import math

import torch

own = False
EPS = 1e-5


def listed():
    return [
        # decode of one token: the norm ahead of a layer, bound by launch and latency
        _norm("norm_t1_h4096_res", 1, 4096, True),
        # prefill of 2048 tokens through the same layer, the largest stream
        _norm("norm_t2048_h4096_res", 2048, 4096, True),
        # a ragged batch of an odd width, no residual (a final norm)
        _norm("norm_t777_h1001", 777, 1001, False),
        # the hidden rows ahead of a down projection: a decode batch and a prefill
        _quant("quant_t16_h14336", 16, 14336),
        _quant("quant_t2048_h14336", 2048, 14336),
        # decode of one token through a down projection: a stream of the weight
        _gemm("gemm_m1_n4096_k14336", 1, 4096, 14336),
        # decode of 16 sequences through a square projection
        _gemm("gemm_m16_n4096_k4096", 16, 4096, 4096),
        # a short prompt of a ragged length, with a bias
        _gemm("gemm_m1000_n4096_k4096_bias", 1000, 4096, 4096, bias=True),
        # sizes that no tile or vector divides, fp32 out (logits of a small vocabulary)
        _gemm("gemm_m777_n1365_k901_f32", 777, 1365, 901, bias=True, f32=True),
        # prefill of 2048 tokens through the down projection
        _gemm("gemm_m2048_n4096_k14336", 2048, 4096, 14336),
        # gate and up products with SiLU(g) * u: a decode batch, and a prefill (the largest case)
        _gemm("gated_m16_n14336_k4096", 16, 14336, 4096, gated=True),
        _gemm("gated_m2048_n14336_k4096", 2048, 14336, 4096, gated=True),
    ]


def _norm(name, t, h, residual):
    return {"name": name, "op": "norm", "t": t, "h": h, "residual": residual}


def _quant(name, t, h):
    return {"name": name, "op": "quant", "t": t, "h": h}


def _gemm(name, m, n, k, bias=False, f32=False, gated=False):
    return {"name": name, "op": "gemm", "m": m, "n": n, "k": k, "bias": bias, "f32": f32, "gated": gated}


def _log(rng, lo, hi, step=1):
    """A multiple of `step` in [lo, hi], uniform in its logarithm."""
    x = math.exp(rng.uniform(math.log(lo), math.log(hi + step)))
    return max(lo, min(hi, int(x) // step * step))


def draw(rng):
    """One more case of the same ranges: single tokens to thousands, widths
    that are whole vectors three times in four and any number otherwise; no
    larger than the listed gated prefill."""
    op = rng.choice(["norm", "quant", "decode", "prefill"])
    step = 16 if rng.random() < 0.75 else 1
    if op in ("norm", "quant"):
        t, h = _log(rng, 1, 8192), _log(rng, 64, 16384, step)
        t = max(1, min(t, (2048 * 16384) // h))
        c = _norm("", t, h, rng.random() < 0.7) if op == "norm" else _quant("", t, h)
    else:
        m = _log(rng, 1, 64) if op == "decode" else _log(rng, 65, 4096)
        n, k = _log(rng, 64, 16384, step), _log(rng, 64, 16384, step)
        gated = rng.random() < 0.3
        most = 2048 * 14336 * 4096 // (1 if gated else 2)     # of m n k
        k = max(64, min(k, most // (m * n) // step * step))
        c = _gemm("", m, n, k, gated=gated, bias=not gated and rng.random() < 0.4,
                  f32=not gated and rng.random() < 0.3)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(1000003 * (int(seed) + 1))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def rows(t, h):
        """Activations: unit normal, some channels ten times as large."""
        return normal(t, h).mul_(torch.where(torch.rand(h, generator=g, device="cuda") < 0.01, 10.0, 1.0))

    def quantised(x):
        a = x.abs().amax(1, keepdim=True)
        return x.mul_(127 / a).round_().to(torch.int8), (a / 127).flatten()

    if case["op"] == "norm":
        t, h = case["t"], case["h"]
        ins = [rows(t, h).to(torch.bfloat16), normal(h).mul_(0.2).add_(1).to(torch.bfloat16)]
        return ins + [rows(t, h).to(torch.bfloat16)] if case["residual"] else ins
    if case["op"] == "quant":
        # SiLU(g) * u of a gated layer: mostly near zero, with far values
        t, h = case["t"], case["h"]
        gate = normal(t, h)
        return [gate.mul_(torch.sigmoid(gate)).mul_(normal(t, h)).to(torch.bfloat16)]
    m, n, k = case["m"], case["n"], case["k"]
    ins = [*quantised(rows(m, k)), *quantised(normal(n, k).mul_(0.02))]
    if case["gated"]:
        ins += quantised(normal(n, k).mul_(0.02))
    if case["bias"]:
        ins.append(normal(n))
    return ins


def _outputs(case):
    def empty(dtype, *shape):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if case["op"] == "gemm":
        return (empty(torch.float32 if case["f32"] else torch.bfloat16, case["m"], case["n"]),)
    t, h = case["t"], case["h"]
    outs = (empty(torch.int8, t, h), empty(torch.float32, t))
    return outs + (empty(torch.bfloat16, t, h),) if case.get("residual") else outs


def _plan(case):
    from paper_2506_01374_amd import rc
    if case["op"] == "norm":
        op = rc.Op(rc.RC_OP_RMSNORM_I8, (case["t"], case["h"]), rc.RC_FLAG_RESIDUAL if case["residual"] else 0, eps=EPS)
    elif case["op"] == "quant":
        op = rc.Op(rc.RC_OP_QUANT_I8, (case["t"], case["h"]))
    else:
        op = rc.Op(rc.RC_OP_GEMM_I8, (case["m"], case["n"], case["k"]),
                   (rc.RC_FLAG_BIAS if case["bias"] else 0) | (rc.RC_FLAG_OUT_F32 if case["f32"] else 0) |
                   (rc.RC_FLAG_GATED if case["gated"] else 0))
    return rc.Plan(op, op.suggest())


def prepare(case, seed):
    state = {"case": case, "inputs": _inputs(case, seed)}
    if own:
        # what a serving program keeps between calls
        plan = _plan(case)
        state.update(plan=plan, outputs=_outputs(case), workspace=plan.workspace())
    return state


# ---------------------------------------------------------------------------
# A pass
# ---------------------------------------------------------------------------

def run(state):
    if own:
        state["plan"].launch(state["inputs"], state["outputs"], state["workspace"])
        return state["outputs"]
    case, ins = state["case"], state["inputs"]
    if case["op"] == "norm":
        return _plain_norm(*ins)
    if case["op"] == "quant":
        p = ins[0].float()
        a = p.abs().amax(1)
        return _plain_round(p, a), a / 127
    return (_plain_gemm(case, ins),)


def _plain_round(p, a):
    # 64 bits: values next to a half go the right way
    q = torch.round(p.double() * 127 / a.double()[:, None])
    return torch.where(a[:, None] > 0, q, 0.0).to(torch.int8)


def _plain_norm(x, w, r=None):
    h = x if r is None else (x.float() + r.float()).to(torch.bfloat16)
    p = h.float() * w.float()
    a = p.abs().amax(1)
    rstd = torch.rsqrt(h.float().square().mean(1) + EPS)
    q, scale = _plain_round(p, a), a * rstd / 127
    return (q, scale) if r is None else (q, scale, h)


def _plain_gemm(case, ins):
    a, sa = ins[0].float(), ins[1][:, None]
    y = (a @ ins[2].float().t()) * (sa * ins[3])
    if case["gated"]:
        u = (a @ ins[4].float().t()) * (sa * ins[5])
        return (y / (1 + torch.exp(-y)) * u).to(torch.bfloat16)
    if case["bias"]:
        y = y + ins[4]
    return y if case["f32"] else y.to(torch.bfloat16)


# ---------------------------------------------------------------------------
# The work and the exact result
# ---------------------------------------------------------------------------

def work(case):
    if case["op"] == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        b = 2 if case["gated"] else 1
        return {"bytes": m * k + b * (n * k + 4.0 * n) + 4.0 * m + (4.0 * n if case["bias"] else 0) +
                (4.0 if case["f32"] else 2.0) * m * n, "flops": 2.0 * b * m * n * k}
    t, h = case["t"], case["h"]
    if case["op"] == "quant":
        return {"bytes": 3.0 * t * h + 4 * t, "flops": 3.0 * t * h}
    return {"bytes": (7.0 if case["residual"] else 3.0) * t * h + 2 * h + 4 * t, "flops": 6.0 * t * h}


def exact(case, seed):
    ins = _inputs(case, seed)
    d = [x.double() for x in ins]
    if case["op"] == "gemm":
        def product(b, s):
            return torch.mm(d[0], b.t()).mul_(d[1].unsqueeze(1)).mul_(s.unsqueeze(0))

        y = product(d[2], d[3])
        if case["gated"]:
            y.mul_(torch.sigmoid(y)).mul_(product(d[4], d[5]))
        elif case["bias"]:
            y.add_(d[4].unsqueeze(0))
        return (y,)
    if case["op"] == "quant":
        y = d[0]
    else:
        # the norm is of the residual stream as it is stored, in bfloat16
        total = d[0] if len(d) == 2 else d[0] + d[2]
        h = total if len(d) == 2 else total.to(torch.bfloat16).double()
        y = h * d[1] / torch.sqrt((h * h).sum(1, keepdim=True) / case["h"] + EPS)
    scale = y.abs().max(1).values / 127
    # the integers are whole numbers: equal to the plain form's, or wrong
    return (None, scale, total) if case.get("residual") else (None, scale)
