"""Performance cases of attention in serving: a paged cache of keys and values,
written (in bf16, or in int8 with a scale for each token and head) and read
back, the attention of new tokens over it, and the attention over whole prompts
packed behind each other.

A case is one operator execution on device-resident inputs.  With ``own`` it
runs through the public binding (``rc.Plan.launch``); without, in elementary
torch operations, which is the operators' plain form.

Sequence b has the packed rows offsets[b] .. offsets[b + 1] - 1, its newest
tokens, and lens[b] tokens in the cache, the newest last.  Position p of it is
slot p % page of page table[b][p / page].
"""
from __future__ import annotations

import math
import random

import torch

own = False


def listed():
    return [
        # a decode step's new tokens into the int8 cache: bound by launch and latency
        _cache("write_i8_b64_h8_d128", "write", "1*64", _spread(64, 64, 8192, 1), 8, 128, 16, True),
        # three prompts of 8000 tokens together, the largest stream into the cache
        _cache("write_i8_t8000_h8_d128", "write", "4000 3001 999", "4000 3001 999", 8, 128, 64, True),
        # sequences leave an int8 cache whole (moved to another place, or read by an operator without pages)
        _cache("read_i8_t16384_h8_d128", "read", "8192 5000 3000 192", "8192 5000 3000 192", 8, 128, 64, True),
        # the last tokens of a few sequences out of a bf16 cache
        _cache("read_bf16_t777_h4_d64", "read", "256 500 21", "1000 500 77", 4, 64, 16, False),
        # decode of one sequence with a long context: nothing but splitting it fills the chip
        _paged("paged_b1_ctx32768_h32_kv8_d128", "1", "32768", 32, 8, 128, 64, False),
        # decode of 64 sequences of very different lengths over the int8 cache
        _paged("paged_i8_b64_h32_kv8_d128", "1*64", _spread(64, 64, 8192, 1), 32, 8, 128, 16, True),
        # five drafted tokens of each of 16 sequences are verified, the other head dimension
        _paged("paged_b16_q5_h16_kv4_d64", "5*16", _spread(16, 300, 4000, 2), 16, 4, 64, 32, False),
        # a chunk of 512 tokens of a long prompt
        _paged("paged_q512_ctx8192_h32_kv8_d128", "512", "8192", 32, 8, 128, 64, False),
        # a step that mixes a chunk with 15 decoding sequences, int8
        _paged("paged_i8_q777_b16_h32_kv8_d128", "777 1*15", "5003 " + _spread(15, 100, 6000, 3), 32, 8, 128, 16, True),
        # short prompts: bound by launch and latency
        _packed("packed_b3_t238_h32_kv8_d128", "1 37 200", 32, 8, 128, True),
        # a batch of prompts of ragged lengths
        _packed("packed_b8_t8192_h32_kv8_d128", "3000 17 1111 801 64 2048 650 501", 32, 8, 128, True),
        # one long prompt: the largest case
        _packed("packed_b1_t16384_h32_kv8_d128", "16384", 32, 8, 128, True),
    ]


def _spread(n, lo, hi, seed):
    """n lengths, uniform in their logarithm, as a text."""
    rng = random.Random(seed)
    return " ".join(str(_log(rng, lo, hi)) for _ in range(n))


def _numbers(text):
    """"5*3 7" is 5, 5, 5, 7."""
    out = []
    for word in text.split():
        x, _, n = word.partition("*")
        out += [int(x)] * int(n or 1)
    return out


def _cache(name, op, q, lens, hkv, d, page, i8):
    return {"name": name, "op": op, "q": q, "lens": lens, "hkv": hkv, "d": d, "page": page, "i8": i8}


def _paged(name, q, lens, h, hkv, d, page, i8, causal=True):
    return {"name": name, "op": "paged", "q": q, "lens": lens, "h": h, "hkv": hkv, "d": d, "page": page, "i8": i8,
            "causal": causal}


def _packed(name, q, h, hkv, d, causal):
    return {"name": name, "op": "packed", "q": q, "lens": q, "h": h, "hkv": hkv, "d": d, "causal": causal}


def _log(rng, lo, hi):
    """A number in [lo, hi], uniform in its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _parts(rng, total, n):
    """n lengths of about `total` together, none empty."""
    w = [rng.uniform(0.05, 1) for _ in range(n)]
    return [max(1, int(total * x / sum(w))) for x in w]


def draw(rng):
    """One more case of the same ranges: any lengths, 1 to 16 query heads for
    each K/V head, three head dimensions, pages of 16 to 256 tokens."""
    op = rng.choice(["write", "read", "decode", "decode", "verify", "chunk", "mixed", "packed", "packed"])
    hkv, d = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 128, 256])
    h = hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
    page, i8 = rng.choice([16, 32, 64, 128, 256]), rng.random() < 0.5
    if op in ("write", "read"):
        q = _parts(rng, _log(rng, 1, 16384), rng.randint(1, 12)) if rng.random() < 0.6 else [1] * _log(rng, 1, 256)
        before = [0 if rng.random() < 0.5 else _log(rng, 1, 2000) for _ in q]
        c = _cache("", op, _text(q), _text(x + y for x, y in zip(q, before)), hkv, d, page, i8)
    elif op in ("decode", "verify"):
        b = _log(rng, 1, 128)
        hi = min(65536, 2 ** 18 // b)
        lens = [_log(rng, 16, hi) for _ in range(b)]
        q = [1 if op == "decode" else min(rng.randint(1, 8), n) for n in lens]
        c = _paged("", _text(q), _text(lens), h, hkv, d, page, i8)
    elif op in ("chunk", "mixed"):
        q = [_log(rng, 16, 2048) for _ in range(rng.randint(1, 3))]
        q += [1] * (rng.randint(1, 24) if op == "mixed" else 0)
        lens = [x + (0 if rng.random() < 0.3 else _log(rng, 1, 8192)) for x in q]
        c = _paged("", _text(q), _text(lens), h, hkv, d, page, i8, rng.random() < 0.85)
    else:
        q = _parts(rng, _log(rng, 1, 8192), rng.randint(1, 8))
        c = _packed("", _text(q), min(h, 32 // hkv * hkv), hkv, d, rng.random() < 0.7)
    del c["name"]
    return c


def _text(numbers):
    return " ".join(str(n) for n in numbers)


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _quantised(x):
    a = x.abs().amax(-1, keepdim=True)
    return x.mul_(127 / a).round_().to(torch.int8), (a / 127).squeeze(-1)


def _inputs(case, seed):
    """The tensors of a call in the operator's order, and what it writes to (the
    cache, for the write)."""
    g = torch.Generator(device="cuda").manual_seed(7919 * (int(seed) + 1))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    def keys(*shape):
        """Keys have a few channels that are far larger than the others."""
        return normal(*shape).mul_(torch.where(torch.rand(shape[-1], generator=g, device="cuda") < 0.03, 4.0, 1.0))

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    q, lens, hkv, d = _numbers(case["q"]), _numbers(case["lens"]), case["hkv"], case["d"]
    t, offsets = sum(q), ints(_starts(q))
    if case["op"] == "packed":
        rows = [normal(t, case["h"], d), keys(t, hkv, d), normal(t, hkv, d)]
        return [x.to(torch.bfloat16) for x in rows] + [offsets, offsets], []
    page = case["page"]
    need = [(n + page - 1) // page for n in lens]
    # the cache's pages are handed out in any order, a few are not in use; a table row is as long as the longest needs
    pages, width = sum(need) + 3, max(need)
    ids = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int64)[:sum(need)].to(torch.int32)
    used = torch.arange(width, device="cuda")[None, :] < ints(need)[:, None]
    table = torch.zeros(len(lens), width, dtype=torch.int32, device="cuda")
    table[used] = ids
    cache = [keys(pages, hkv, page, d), normal(pages, hkv, page, d)]
    if case["i8"]:
        pairs = [_quantised(x) for x in cache]
        cache = [p[0] for p in pairs] + [p[1] for p in pairs]
    else:
        cache = [x.to(torch.bfloat16) for x in cache]
    where = [offsets, ints(lens), table]
    if case["op"] == "write":
        return [keys(t, hkv, d).to(torch.bfloat16), normal(t, hkv, d).to(torch.bfloat16)] + where, cache
    if case["op"] == "read":
        return cache + where, []
    return [normal(t, case["h"], d).to(torch.bfloat16)] + cache + where, []


def _plan(case, inputs, cache):
    from paper_2506_01374_amd import rc
    t, b, hkv, d = sum(_numbers(case["q"])), len(_numbers(case["q"])), case["hkv"], case["d"]
    causal = rc.RC_FLAG_CAUSAL if case.get("causal") else 0
    if case["op"] == "packed":
        op = rc.Op(rc.RC_OP_ATTENTION_PACKED, (t, t, b, case["h"], hkv, d), causal)
        return rc.Plan(op, op.suggest())
    pages = (cache or inputs[1 if case["op"] == "paged" else 0:])[0].shape[0]
    where = (case["page"], pages, inputs[-1].shape[1])
    flags = rc.RC_FLAG_I8_CACHE if case["i8"] else 0
    if case["op"] == "paged":
        op = rc.Op(rc.RC_OP_ATTENTION_PAGED, (t, b, case["h"], hkv, d) + where, flags | causal)
    else:
        op = rc.Op(rc.RC_OP_KV_WRITE if case["op"] == "write" else rc.RC_OP_KV_READ, (t, b, hkv, d) + where, flags)
    return rc.Plan(op, op.suggest())


def prepare(case, seed):
    inputs, cache = _inputs(case, seed)
    state = {"case": case, "inputs": inputs, "cache": cache}
    if own:
        # what a serving program keeps between calls
        t, plan = inputs[0].shape[0], _plan(case, inputs, cache)
        if case["op"] == "read":
            t = sum(_numbers(case["q"]))
            outs = tuple(torch.empty(t, case["hkv"], case["d"], dtype=torch.bfloat16, device="cuda") for _ in range(2))
        else:
            outs = tuple(cache) if cache else (torch.empty_like(inputs[0]),)
        state.update(plan=plan, outputs=outs, workspace=plan.workspace())
    else:
        # the lengths, which the plain form loops over on the host
        state.update(q=_numbers(case["q"]), lens=_numbers(case["lens"]))
    return state


# ---------------------------------------------------------------------------
# A pass
# ---------------------------------------------------------------------------

def run(state):
    if own:
        state["plan"].launch(state["inputs"], state["outputs"], state["workspace"])
        return state["outputs"]
    case, ins = state["case"], state["inputs"]
    if case["op"] == "write":
        return _plain_write(case, ins, state["cache"])
    if case["op"] == "read":
        return _plain_read(case, ins)
    return (_plain_attention(case, ins, state["q"], state["lens"]),)


def _plain_slots(rows, offsets, lens, table, page):
    """Page and slot of each packed row."""
    row = torch.arange(rows, device="cuda")
    b = torch.searchsorted(offsets[1:].contiguous(), row.to(torch.int32), right=True)
    p = lens[b] - offsets[b + 1] + row
    return table[b, p // page].long(), p % page


def _plain_write(case, ins, cache):
    at, slot = _plain_slots(ins[0].shape[0], *ins[2:], case["page"])
    for i, x in enumerate(ins[:2]):
        if not case["i8"]:
            cache[i][at, :, slot] = x
            continue
        # 64 bits: values next to a half go the right way
        a = x.double().abs().amax(-1)
        q = torch.round(x.double() * 127 / a[..., None])
        cache[i][at, :, slot] = torch.where(a[..., None] > 0, q, 0.0).to(torch.int8)
        cache[2 + i][at, :, slot] = (a / 127).float()
    return tuple(cache)


def _plain_read(case, ins):
    offsets, lens, table = ins[-3:]
    at, slot = _plain_slots(sum(_numbers(case["q"])), offsets, lens, table, case["page"])
    x = [c[at, :, slot] for c in ins[:-3]]
    if not case["i8"]:
        return tuple(x)
    return tuple((x[i].float() * x[2 + i][..., None]).to(torch.bfloat16) for i in range(2))


def _plain_attention(case, ins, qs, lens):
    out = torch.empty_like(ins[0])
    t0, k0, group = 0, 0, case["h"] // case["hkv"]
    for b, (n, m) in enumerate(zip(qs, lens)):
        q = ins[0][t0:t0 + n].float().transpose(0, 1)                         # [H][n][D]
        if case["op"] == "packed":
            k, v = (x[k0:k0 + m].float().transpose(0, 1) for x in ins[1:3])   # [Hkv][m][D]
        else:
            k, v = _plain_pages(case, ins, b, m)
        # (pieces of at most 2^28 scores)
        step = max(1, 2 ** 28 // (case["h"] * m))
        for i in range(0, n, step):
            r = min(n, i + step) - i
            # the query heads of a K/V head are rows of one product
            s = torch.matmul(q[:, i:i + r].reshape(-1, group * r, case["d"]), k.transpose(1, 2)) / math.sqrt(case["d"])
            s = s.unflatten(1, (group, r))
            if case["causal"]:
                last = torch.arange(i, i + r, device="cuda") + (m - n)
                s.masked_fill_(torch.arange(m, device="cuda")[None, :] > last[:, None], -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True)).flatten(1, 2)
            o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
            out[t0 + i:t0 + i + r] = o.view(-1, r, case["d"]).transpose(0, 1).to(torch.bfloat16)
        t0, k0 = t0 + n, k0 + m
    return out


def _plain_pages(case, ins, b, m):
    cache, table, page = ins[1:-3], ins[-1], case["page"]
    at = table[b, :(m + page - 1) // page].long()
    x = [c[at].transpose(0, 1).flatten(1, 2)[:, :m].float() for c in cache]
    if case["i8"]:
        return x[0] * x[2][..., None], x[1] * x[3][..., None]
    return x[0], x[1]


# ---------------------------------------------------------------------------
# The work and the exact result
# ---------------------------------------------------------------------------

def work(case):
    q, lens, hkv, d = _numbers(case["q"]), _numbers(case["lens"]), case["hkv"], case["d"]
    t = sum(q)
    token = (2.0 * d + 8 if case.get("i8") else 4.0 * d) * hkv            # cache bytes of a token
    if case["op"] in ("write", "read"):
        return {"bytes": t * (token + 4.0 * d * hkv), "flops": 6.0 * t * hkv * d if case["i8"] else 0.0}
    if case["causal"]:
        pairs = sum(n * m - n * (n - 1) / 2 for n, m in zip(q, lens))
    else:
        pairs = sum(n * m for n, m in zip(q, lens))
    return {"bytes": 4.0 * t * case["h"] * d + token * sum(lens), "flops": 4.0 * case["h"] * d * pairs}


def exact(case, seed):
    ins, cache = _inputs(case, seed)
    qs, lens = _numbers(case["q"]), _numbers(case["lens"])
    if case["op"] in ("write", "read"):
        # (page, slot) of each row, on the host
        page, table = case["page"], ins[-1].tolist()
        places = [(table[b][p // page], p % page) for b, (n, m) in enumerate(zip(qs, lens)) for p in range(m - n, m)]
        at, slot = (torch.tensor(x, device="cuda") for x in zip(*places))
        if case["op"] == "read":
            out = [c.double()[at, :, slot] for c in ins[:-3]]
            return (out[0] * out[2].unsqueeze(2), out[1] * out[3].unsqueeze(2)) if case["i8"] else tuple(out)
        if not case["i8"]:
            out = [c.double() for c in cache]
            for i in (0, 1):
                out[i][at, :, slot] = ins[i].double()
            return tuple(out)
        scales = [c.double() for c in cache[2:]]
        for i in (0, 1):
            scales[i][at, :, slot] = ins[i].double().abs().max(dim=2).values / 127
        # the integers are whole numbers: equal to the plain form's, or wrong
        return (None, None, scales[0], scales[1])
    rows, row = [], 0
    for b, (n, m) in enumerate(zip(qs, lens)):
        query = ins[0][row:row + n].double()
        if case["op"] == "packed":
            k, v = (x[sum(lens[:b]):sum(lens[:b]) + m].double() for x in ins[1:3])
        else:
            index = ins[-1][b].long()
            kv = [c.index_select(0, index).double() for c in ins[1:3]]
            if case["i8"]:
                kv = [x * c.index_select(0, index).double().unsqueeze(3) for x, c in zip(kv, ins[3:5])]
            k, v = (x.permute(0, 2, 1, 3).reshape(-1, case["hkv"], case["d"])[:m] for x in kv)
        heads = []
        for h in range(case["h"]):
            kh, vh = (x[:, h * case["hkv"] // case["h"]].contiguous() for x in (k, v))
            pieces = []
            for piece in torch.arange(n, device="cuda").split(max(1, 2 ** 27 // m)):
                score = query[piece, h] @ kh.T * case["d"] ** -0.5
                if case["causal"]:
                    hidden = torch.arange(m, device="cuda").unsqueeze(0) > (piece + m - n).unsqueeze(1)
                    score = torch.where(hidden, -math.inf, score)
                pieces.append(torch.softmax(score, dim=1) @ vh)
            heads.append(torch.cat(pieces))
        rows.append(torch.stack(heads, dim=1))
        row += n
    return (torch.cat(rows),)
