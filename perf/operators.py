"""Attention without its n x m matrix: the cases that its speed is measured on.

Five operators: attention of packed rows (`apply`), its gradient in a training step (`grad`), and
what serving needs: block tables and slots from the requests' lengths (`map`), new rows into a
cache of 8-bit blocks (`append`) and attention of the newest rows over that cache (`cache`).

Every case is a dict of plain values; "op" is one of the five names, the others are that
operator's sizes and options.  Lengths of documents and requests follow from the sizes alone.
"""
from __future__ import annotations

import math
import random

import torch

own = False

LIMIT = 10 ** 9  # bytes the library may keep beside inputs and outputs


# ---- cases ----------------------------------------------------------------------------------

def _apply(name, op, n, m, docs, hq, hkv, d, dtype, causal=True, prefix=False, cap=0.0, slopes=False):
    return {"name": name, "op": op, "n": n, "m": m, "docs": docs, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype,
            "causal": causal, "prefix": prefix, "cap": cap, "slopes": slopes}


def _cache(name, batch, longest, nq, hq, hkv, d, block, dtype, code, cap=0.0, slopes=False):
    return {"name": name, "op": "cache", "batch": batch, "longest": longest, "nq": nq, "hq": hq, "hkv": hkv, "d": d,
            "block": block, "dtype": dtype, "code": code, "cap": cap, "slopes": slopes}


def _append(name, batch, new, hkv, d, block, dtype, code):
    return {"name": name, "op": "append", "batch": batch, "new": new, "hkv": hkv, "d": d, "block": block, "dtype": dtype,
            "code": code}


def _map(name, batch, longest, new, block):
    return {"name": name, "op": "map", "batch": batch, "longest": longest, "new": new, "block": block}


def listed():
    return [
        # one long sequence through a layer with shared heads: the largest forward pass
        _apply("apply_long", "apply", 8192, 8192, 1, 32, 8, 128, "bf16"),
        # ragged documents packed into one row axis, each with a part that sees itself whole
        # (a prompt), scores capped
        _apply("apply_packed", "apply", 5003, 5003, 7, 16, 16, 64, "f16", prefix=True, cap=30.0),
        # a few new rows against a long resident sequence: work has to be split along the keys
        _apply("apply_few_rows", "apply", 3, 50_021, 1, 16, 2, 128, "bf16", slopes=True),
        # a training step's forward and backward pass
        _apply("grad_train", "grad", 4096, 4096, 1, 32, 8, 128, "bf16", slopes=True),
        # a small batch of short documents, rows that are not a power of two wide
        _apply("grad_packed", "grad", 1201, 1201, 5, 8, 2, 80, "f16", prefix=True, cap=50.0),
        # a service's step: 64 requests of very different lengths, one new row each
        _cache("cache_batch", 64, 8192, 1, 32, 8, 128, 64, "bf16", "int8"),
        # one request with a very long history in small blocks
        _cache("cache_long", 1, 200_003, 1, 32, 8, 128, 16, "f16", "e4m3", cap=50.0),
        # a handful of short requests, three rows each (a drafted continuation): latency
        _cache("cache_small", 4, 500, 3, 8, 4, 64, 32, "bf16", "e4m3", slopes=True),
        # a step's new rows, one a request
        _append("append_step", 64, 1, 8, 128, 16, "bf16", "int8"),
        # prompts go into the cache
        _append("append_prompts", 8, 2048, 8, 128, 64, "bf16", "e4m3"),
        # a step's bookkeeping, and that of many prompts at once
        _map("map_step", 64, 8192, 1, 16),
        _map("map_prompts", 256, 4096, 512, 64),
    ]


def _log(rng, low, high):
    """A whole number between low and high, its logarithm uniform."""
    return int(min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))))


def draw(rng):
    """One more call of the same ranges."""
    op = rng.choice(("apply", "apply", "few", "grad", "grad", "cache", "cache", "append", "map"))
    dtype = rng.choice(("bf16", "f16"))
    hkv = rng.choice((1, 2, 4, 8, 16))
    hq = hkv * rng.choice([g for g in (1, 2, 3, 4, 8) if hkv * g <= 32])
    d = rng.choice((64, 128, 64, 128, 8 * rng.randint(4, 16)))
    cap = rng.choice((0.0, 0.0, 30.0, 50.0))
    slopes = rng.random() < 0.3
    if op == "few":
        n = _log(rng, 1, 64)
        m = _log(rng, 5_000, 100_000)
        case = _apply("", "apply", n, m, 1, hq, hkv, d, dtype, rng.random() < 0.8, False, cap, slopes)
    elif op in ("apply", "grad"):
        docs = rng.choice((1, 1, 2, 5, 16))
        causal = rng.random() < 0.8  # where not, twice the pairs are seen
        n = _log(rng, 200, (4_000 if op == "grad" else 8_000) if causal else (2_800 if op == "grad" else 5_600))
        m = n if causal or rng.random() < 0.5 else _log(rng, 200, 2_800)
        case = _apply("", op, n, m, docs, hq, hkv, d, dtype, causal, causal and rng.random() < 0.4, cap, slopes)
    elif op == "cache":
        batch = _log(rng, 1, 64)
        longest = _log(rng, 100, min(200_000, 500_000 // batch))
        case = _cache("", batch, longest, rng.choice((1, 1, 1, 2, 4)), hq, hkv, d, rng.choice((16, 32, 64)), dtype,
                      rng.choice(("int8", "e4m3")), cap, slopes)
    elif op == "append":
        new = rng.choice((1, 1, _log(rng, 2, 2_000)))
        batch = _log(rng, 1, 8 if new > 1 else 128)
        case = _append("", batch, new, min(hkv, 8), d, rng.choice((16, 32, 64)), dtype, rng.choice(("int8", "e4m3")))
    else:
        case = _map("", _log(rng, 1, 256), _log(rng, 600, 8_000), rng.choice((1, _log(rng, 2, 500))),
                    rng.choice((16, 32, 64)))
    del case["name"]
    return case


# ---- lengths that follow from a case --------------------------------------------------------

def _cuts(total, parts):
    """`parts` lengths that add up to `total`, uneven; some may be zero."""
    rng = random.Random(1000 * total + parts)
    at = sorted(rng.randint(0, total) for _ in range(parts - 1))
    return [b - a for a, b in zip([0] + at, at + [total])]


def _documents(case):
    """(query rows, key rows, rows of the prefix) of each document."""
    nq = _cuts(case["n"], case["docs"])
    nk = nq if case["m"] == case["n"] else _cuts(case["m"], case["docs"])
    rng = random.Random(case["n"])
    return [(a, b, rng.randint(0, b // 2) if case["prefix"] else 0) for a, b in zip(nq, nk)]


def _lengths(batch, longest):
    """Rows of each request, from a sixteenth of the longest to the longest, which is among them."""
    rng = random.Random(1000 * longest + batch)
    return [longest] + [rng.randint(max(1, longest // 16), longest) for _ in range(batch - 1)]


def _news(case):
    """(rows before, new rows) of each request of an append or a map."""
    rng = random.Random(1000 * case["batch"] + case["new"])
    new = [case["new"] if case["new"] == 1 else rng.randint(1, case["new"]) for _ in range(case["batch"])]
    if case["op"] == "append":
        return [(rng.randint(0, 3 * case["block"]), n) for n in new]
    return [(rng.randint(0, case["longest"] - n), n) for n in new]


def _starts(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device="cuda")


def _words(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- inputs ---------------------------------------------------------------------------------

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
_MOST = {"int8": 127.0, "e4m3": 448.0}  # the largest code


def _normal(gen, shape, dtype, size=1.0):
    return (size * torch.randn(shape, generator=gen, device="cuda")).to(_TYPES[dtype])


def _slopes(case):
    if not case["slopes"]:
        return None
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / case["hq"]) for h in range(case["hq"])], device="cuda")


def _row(d):
    return (d + 63) // 64 * 64  # entries of a row in the cache; those behind d are zero


def _codes(gen, blocks, case):
    """A cache in use: codes as a normal distribution gives them, scales of a factor of two."""
    hkv, d, block = case["hkv"], case["d"], case["block"]
    made = []
    for _ in range(2):
        x = torch.randn(blocks, hkv, block, _row(d), generator=gen, device="cuda", dtype=torch.bfloat16)
        x = (x * (_MOST[case["code"]] / 4)).clamp_(-_MOST[case["code"]], _MOST[case["code"]])
        x[..., d:] = 0
        made.append((x.round_() if case["code"] == "int8" else x).to(_TYPES[case["code"]]))
        del x
    scales = [(1 + torch.rand(blocks, hkv, generator=gen, device="cuda")) * (4 / _MOST[case["code"]]) for _ in range(2)]
    return {"k": made[0], "v": made[1].transpose(2, 3).contiguous(), "k_scale": scales[0], "v_scale": scales[1]}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    state = {"case": case}
    if case["op"] in ("apply", "grad"):
        n, m, hq, hkv, d = (case[a] for a in ("n", "m", "hq", "hkv", "d"))
        docs = _documents(case)
        # capped scores are large ones: the cap has to act
        state["Q"] = _normal(gen, (n, hq, d), case["dtype"], 6.0 if case["cap"] else 1.0)
        state["K"] = _normal(gen, (m, hkv, d), case["dtype"])
        state["V"] = _normal(gen, (m, hkv, d), case["dtype"])
        state["dO"] = _normal(gen, (n, hq, d), case["dtype"]) if case["op"] == "grad" else None
        state["slopes"] = _slopes(case)
        one = case["docs"] == 1
        state["starts"] = None if one and not case["prefix"] else _starts([a for a, _, _ in docs])
        state["k_starts"] = None if state["starts"] is None else _starts([b for _, b, _ in docs])
        state["prefix"] = _words([p for _, _, p in docs]) if case["prefix"] else None
        return state
    batch, block = case["batch"], case["block"]
    if case["op"] == "cache":
        lengths = _lengths(batch, case["longest"])
        width = -(-case["longest"] // block)
        held = [-(-n // block) for n in lengths]
        order = torch.randperm(sum(held) + 3, generator=gen, device="cuda").to(torch.int32)
        table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
        at = 0
        for i, h in enumerate(held):
            table[i, :h] = order[at:at + h]
            at += h
        state |= _codes(gen, sum(held) + 3, case)
        state["table"], state["lengths"] = table, _words(lengths)
        state["Q"] = _normal(gen, (batch, case["nq"], case["hq"], case["d"]), case["dtype"], 6.0 if case["cap"] else 1.0)
        state["slopes"] = _slopes(case)
        return state
    if case["op"] == "append":
        slots, blocks = [], 0
        for before, new in _news(case):
            rest = before % block  # rows that the request's last block holds already
            slots += [blocks * block + rest + t for t in range(new)]
            blocks += -(-(rest + new) // block)
        # the request's blocks lie in no order
        order = torch.randperm(blocks, generator=gen, device="cuda")
        slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
        state["slots"] = order[slots // block] * block + slots % block
        state |= _codes(gen, blocks, case)
        shape = (slots.numel(), case["hkv"], case["d"])
        state["K"], state["V"] = _normal(gen, shape, case["dtype"], 1.5), _normal(gen, shape, case["dtype"], 1.5)
        return state
    news = _news(case)
    width = -(-case["longest"] // block)
    held = [-(-b // block) for b, _ in news]
    order = torch.randperm(batch * (width + 1), generator=gen, device="cuda").to(torch.int32)
    table = torch.full((batch, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, h in enumerate(held):
        table[i, :h] = order[at:at + h]
        at += h
    state["table"], state["free"] = table, order[at:].clone()
    state["lengths"], state["news"] = _words([b + n for b, n in news]), _words([n for _, n in news])
    # slots of a padded step: the program's own buffer is a little longer than this step's rows
    state["slots"] = sum(n for _, n in news) + 5
    return state


# ---- one pass -------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        import paper_2206_14148_amd as knn
        if c["op"] in ("apply", "grad"):
            options = {"causal": c["causal"], "cap": c["cap"], "slopes": state["slopes"], "starts": state["starts"],
                       "k_starts": state["k_starts"], "prefix": state["prefix"]}
            O, lse = knn.attn_apply(state["Q"], state["K"], state["V"], LIMIT, **options)
            if c["op"] == "apply":
                return O, lse
            return (O,) + tuple(knn.attn_grad(state["Q"], state["K"], state["V"], O, lse, state["dO"], LIMIT, **options))
        if c["op"] == "map":
            return knn.attn_cache_map(state["lengths"], state["news"], state["table"], state["free"], c["block"],
                                      state["slots"])
        cache = knn.AttnCache(state["k"], state["v"], state["k_scale"], state["v_scale"], c["d"])
        if c["op"] == "cache":
            return knn.attn_cache_apply(state["Q"], cache, state["table"], state["lengths"], LIMIT, cap=c["cap"],
                                        slopes=state["slopes"])
        knn.attn_cache_append(cache, state["K"], state["V"], state["slots"])
        return _values(state["k"], state["v"], state["k_scale"], state["v_scale"])
    if c["op"] in ("apply", "grad"):
        return _plain_attention(state, c["op"] == "grad")
    if c["op"] == "map":
        return _plain_map(state)
    if c["op"] == "cache":
        return _plain_cache(state)
    return _plain_append(state)


def _values(k, v, k_scale, v_scale):
    """What a cache's codes stand for."""
    return k.float() * k_scale[:, :, None, None], v.float() * v_scale[:, :, None, None]


def _spread(x, hq):
    """[rows, hkv, d] as [hq, rows, d] in 32 bits, a head for each query head."""
    return x.float().transpose(0, 1).repeat_interleave(hq // x.shape[1], 0)


def _seen(state):
    """Which key each row sees, and how far it is: two [n, m] tensors."""
    c = state["case"]
    n, m = c["n"], c["m"]
    starts, k_starts = state["starts"], state["k_starts"]
    if starts is None:
        starts, k_starts = _words([0, n]), _words([0, m])
    i, j = (torch.arange(x, device="cuda", dtype=torch.int32) for x in (n, m))
    di = torch.searchsorted(starts, i, right=True) - 1
    dj = torch.searchsorted(k_starts, j, right=True) - 1
    # both counted from the first key of the row's document
    p = i - starts[di] + (k_starts[di + 1] - k_starts[di]) - (starts[di + 1] - starts[di])
    q = j - k_starts[dj]
    seen = di[:, None] == dj[None, :]
    if c["causal"]:
        hi = p + 1
        if state["prefix"] is not None:
            hi = torch.maximum(hi, state["prefix"][di])
        seen &= q[None, :] < hi[:, None]
    return seen, (p[:, None] - q[None, :]).abs()


def _softmax(u, seen, away, cap, slopes):
    """(probabilities, their log-sums, tanh(u / cap)) of scores u [h, n, m]."""
    t = None
    if cap:
        t = torch.tanh(u / cap)
        u = cap * t
    if slopes is not None:
        u = u - slopes[:, None, None] * away
    u = u.masked_fill(~seen, -math.inf)
    top = u.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    e = torch.exp(u - top)
    total = e.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).squeeze(-1)
    return e / torch.where(total == 0, torch.ones_like(total), total), lse, t


def _plain_attention(state, grad):
    c = state["case"]
    hq, hkv, d, scale = c["hq"], c["hkv"], c["d"], 1.0 / math.sqrt(c["d"])
    Q, K, V = state["Q"].float().transpose(0, 1).contiguous(), _spread(state["K"], hq), _spread(state["V"], hq)
    seen, away = _seen(state)
    P, lse, t = _softmax(scale * torch.bmm(Q, K.transpose(1, 2).contiguous()), seen, away, c["cap"], state["slopes"])
    O = torch.bmm(P, V)
    out = O.transpose(0, 1).to(state["Q"].dtype)
    if not grad:
        return out, lse
    dO = state["dO"].float().transpose(0, 1).contiguous()
    dV = torch.bmm(P.transpose(1, 2).contiguous(), dO)
    dS = P * (torch.bmm(dO, V.transpose(1, 2).contiguous()) - (dO * O).sum(-1, keepdim=True))
    if t is not None:
        dS = dS * (1 - t * t)
    dQ = scale * torch.bmm(dS, K)
    dK = scale * torch.bmm(dS.transpose(1, 2).contiguous(), Q)
    dK, dV = (x.view(hkv, hq // hkv, c["m"], d).sum(1) for x in (dK, dV))
    return (out,) + tuple(x.transpose(0, 1).to(state["Q"].dtype) for x in (dQ, dK, dV))


def _plain_cache(state):
    c = state["case"]
    batch, nq, hq, hkv, d = (c[a] for a in ("batch", "nq", "hq", "hkv", "d"))
    table, lengths = state["table"].clamp(min=0).long(), state["lengths"]
    K = state["k"][table].float() * state["k_scale"][table][..., None, None]
    V = state["v"][table].float() * state["v_scale"][table][..., None, None]
    K = K.permute(0, 2, 1, 3, 4).reshape(batch * hkv, -1, K.shape[-1])[..., :d]
    V = V.permute(0, 2, 1, 4, 3).reshape(batch * hkv, -1, V.shape[3])[..., :d]
    g, m = hq // hkv, K.shape[1]
    Q = state["Q"].float().view(batch, nq, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(batch * hkv, g * nq, d)
    u = torch.bmm(Q, K.transpose(1, 2).contiguous()).view(batch, hq, nq, m) / math.sqrt(d)
    j = torch.arange(m, device="cuda")
    p = lengths[:, None] - nq + torch.arange(nq, device="cuda")
    seen = (j <= p[..., None]) & (j < lengths[:, None, None])
    away = (p[..., None] - j).abs()
    slopes = state["slopes"]
    P = _softmax(u.view(batch * hq, nq, m), seen.repeat_interleave(hq, 0), away.repeat_interleave(hq, 0) if slopes is not None else None,
                 c["cap"], None if slopes is None else slopes.repeat(batch))[0]
    O = torch.bmm(P.view(batch * hkv, g * nq, m), V.contiguous())
    return O.view(batch, hq, nq, d).transpose(1, 2).to(state["Q"].dtype)


def _nearest(x, code):
    """The codes nearest to 64-bit numbers, as numbers; of two as near the even one."""
    x = x.clamp(-_MOST[code], _MOST[code])
    if code == "int8":
        return torch.round(x)
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)  # of e4m3: three bits behind the first
    return torch.round(x / step) * step


def _plain_append(state):
    c = state["case"]
    block, most = c["block"], _MOST[c["code"]]
    at, offset = state["slots"] // block, state["slots"] % block
    fresh = torch.zeros(state["k"].shape[0], device="cuda").index_fill_(0, at[offset == 0], 1.0)[:, None]
    found = []
    for codes, scales, x in ((state["k"], state["k_scale"], state["K"]), (state["v"].transpose(2, 3), state["v_scale"], state["V"])):
        x = x.double()
        grown = (x.abs().amax(-1) / most).float()
        before = scales * (1 - fresh)
        after = before.index_reduce(0, at, grown, "amax")
        q = codes.double()
        ratio = before.double() / after
        kept = _nearest(q * ratio[:, :, None, None], c["code"])
        kept = torch.where((after > before)[:, :, None, None], kept, q)
        kept[at, :, offset, :c["d"]] = _nearest(x / after.double()[at][..., None], c["code"])
        found.append((kept.float() * after[:, :, None, None]))
    return found[0], found[1].transpose(2, 3).contiguous()


def _plain_map(state):
    block, table, free = state["case"]["block"], state["table"].long(), state["free"].long()
    lengths, news = state["lengths"].long(), state["news"].long()
    before = lengths - news
    held, need = (before + block - 1) // block, (lengths + block - 1) // block
    take = need - held
    first = torch.cumsum(take, 0) - take
    j = torch.arange(table.shape[1], device="cuda")
    from_free = first[:, None] + j - held[:, None]
    taken = torch.where(from_free < free.numel(), free[from_free.clamp(0, free.numel() - 1)], -1)
    table = torch.where((j >= held[:, None]) & (j < need[:, None]), taken, table)
    starts = torch.nn.functional.pad(torch.cumsum(news, 0), (1, 0))
    t = torch.arange(state["slots"], device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    inside = r < news.numel()
    r = r.clamp(max=news.numel() - 1)
    at = before[r] + t - starts[r]
    where = table[r, (at // block).clamp(max=table.shape[1] - 1)]
    slots = torch.where(inside & (where >= 0), where * block + at % block, -1)
    return table.int(), starts.int(), slots, take.sum().int().view(1)


# ---- what a pass cannot do without ----------------------------------------------------------

def _pairs(case):
    total = 0
    for nq, nk, prefix in _documents(case):
        if not case["causal"]:
            total += nq * nk
        else:
            total += sum(min(nk, max(t + nk - nq + 1, prefix, 0)) for t in range(nq))
    return total


def work(case):
    if case["op"] in ("apply", "grad"):
        n, m, hq, hkv, d = (case[a] for a in ("n", "m", "hq", "hkv", "d"))
        pairs = _pairs(case) * hq
        if case["op"] == "apply":  # two products; Q, O and K, V in 16 bits, the log-sums in 32
            return {"bytes": 4 * d * (n * hq + m * hkv) + 4 * n * hq, "flops": 4 * d * pairs}
        # two products forward, and five backward, the scores among them once more
        return {"bytes": 2 * d * (4 * n * hq + 4 * m * hkv), "flops": 14 * d * pairs}
    if case["op"] == "cache":
        rows = sum(_lengths(case["batch"], case["longest"]))
        asked = case["batch"] * case["nq"] * case["hq"] * case["d"]
        return {"bytes": 2 * rows * case["hkv"] * case["d"] + 4 * asked,
                "flops": 4 * rows * case["nq"] * case["hq"] * case["d"]}
    news = _news(case)
    rows = sum(n for _, n in news)
    if case["op"] == "append":
        # the new rows read and their codes written; the values that are looked at, 4 bytes each
        block, entries = case["block"], case["hkv"] * case["d"]
        held = sum(-(-(b % block + n) // block) for b, n in news) * block
        return {"bytes": rows * entries * 4 + held * entries * 8, "flops": 4 * rows * entries}
    tables = case["batch"] * -(-case["longest"] // case["block"])
    return {"bytes": 8 * rows + 8 * tables + 12 * case["batch"], "flops": 8 * rows}


# ---- the same in 64 bits --------------------------------------------------------------------

def exact(case, seed):
    """What `run` returns from the definitions in 64 bits, head by head and request by request."""
    state = prepare(case, seed)
    if case["op"] == "map":
        return None
    if case["op"] == "append":
        return _exact_append(case, state)
    if case["op"] == "cache":
        return _exact_cache(case, state)
    n, m, hq, hkv, d = (case[a] for a in ("n", "m", "hq", "hkv", "d"))
    wide = {a: state[a].double() for a in ("Q", "K", "V")}
    out = torch.zeros(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((hq, n), -math.inf, dtype=torch.float64, device="cuda")
    dQ, dK, dV = torch.zeros_like(out), torch.zeros_like(wide["K"]), torch.zeros_like(wide["V"])
    i0 = j0 = 0
    for nq, nk, prefix in _documents(case):
        if nq and nk:
            p = torch.arange(nq, device="cuda")[:, None] + (nk - nq)
            j = torch.arange(nk, device="cuda")[None, :]
            hidden = (j > p) & (j >= prefix) if case["causal"] else torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
            empty = hidden.all(1)
            rows, keys = slice(i0, i0 + nq), slice(j0, j0 + nk)
            for h in range(hq):
                f = h // (hq // hkv)
                q, k, v = wide["Q"][rows, h], wide["K"][keys, f], wide["V"][keys, f]
                s = q @ k.T * d ** -0.5
                slope = torch.ones((), dtype=torch.float64, device="cuda")
                if case["cap"]:
                    th = torch.tanh(s / case["cap"])
                    s, slope = th * case["cap"], 1 - th ** 2
                if case["slopes"]:
                    s = s - state["slopes"][h].double() * (p - j).abs()
                s[hidden] = -math.inf
                lse[h, rows] = torch.logsumexp(s, 1)
                w = torch.exp(s - lse[h, rows][:, None])
                w[empty] = 0
                out[rows, h] = w @ v
                if case["op"] == "grad":
                    g = state["dO"][rows, h].double()
                    dV[keys, f] += w.T @ g
                    ds = w * (g @ v.T - (g * out[rows, h]).sum(1, keepdim=True)) * slope
                    dQ[rows, h] = ds @ k * d ** -0.5
                    dK[keys, f] += ds.T @ q * d ** -0.5
        i0, j0 = i0 + nq, j0 + nk
    return (out, lse) if case["op"] == "apply" else (out, dQ, dK, dV)


def _exact_cache(case, state):
    nq, hq, hkv, d, block = (case[a] for a in ("nq", "hq", "hkv", "d", "block"))
    out = torch.zeros(state["Q"].shape, dtype=torch.float64, device="cuda")
    for b, length in enumerate(_lengths(case["batch"], case["longest"])):
        mine = state["table"][b, : -(-length // block)].long()
        k = (state["k"][mine].double() * state["k_scale"][mine].double()[..., None, None])
        v = (state["v"][mine].double() * state["v_scale"][mine].double()[..., None, None])
        k = k.transpose(0, 1).reshape(hkv, -1, k.shape[-1])[:, :length, :d]
        v = v.permute(1, 0, 3, 2).reshape(hkv, -1, v.shape[2])[:, :length, :d]
        p = torch.arange(length - nq, length, device="cuda")[:, None]
        j = torch.arange(length, device="cuda")[None, :]
        for h in range(hq):
            s = state["Q"][b, :, h].double() @ k[h // (hq // hkv)].T * d ** -0.5
            if case["cap"]:
                s = case["cap"] * torch.tanh(s / case["cap"])
            if case["slopes"]:
                s = s - state["slopes"][h].double() * (p - j).abs()
            out[b, :, h] = torch.softmax(s.masked_fill(j > p, -math.inf), 1).nan_to_num(0.0) @ v[h // (hq // hkv)]
    return out


def _exact_append(case, state):
    """Block by block: a scale is a 32-bit number, a code the nearest to a quotient of real numbers."""
    d, block, most = case["d"], case["block"], _MOST[case["code"]]
    values = []
    slots = state["slots"].tolist()
    mine = {}
    for t, s in enumerate(slots):
        mine.setdefault(s // block, []).append((s % block, t))
    if case["code"] == "e4m3":
        whole = torch.arange(127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn).double()
    else:
        whole = torch.arange(128, device="cuda").double()
    between = (whole[1:] + whole[:-1]) / 2
    up = torch.nextafter(between, torch.full_like(between, math.inf))

    def code(y):
        a = y.abs()
        low = torch.bucketize(a, torch.where(torch.arange(between.numel(), device="cuda") % 2 == 0, up, between), right=True)
        return torch.copysign(whole[low], y)

    for codes, scales, x in ((state["k"], state["k_scale"], state["K"]),
                             (state["v"].transpose(2, 3), state["v_scale"], state["V"])):
        held = codes.double()
        now = scales.clone()
        x = x.double()
        for b, rows in mine.items():
            offsets = torch.tensor([o for o, _ in rows], device="cuda")
            new = x[torch.tensor([t for _, t in rows], device="cuda")]  # [rows, hkv, d]
            s0 = torch.zeros_like(now[b]) if any(o == 0 for o, _ in rows) else now[b]
            s1 = torch.maximum(s0, (new.abs().amax((0, 2)) / most).float())
            moved = code(held[b] * s0.double()[:, None, None] / s1.double()[:, None, None])
            held[b] = torch.where((s1 > s0)[:, None, None], moved, held[b])
            held[b][:, offsets, :d] = code(new.transpose(0, 1) / s1.double()[:, None, None])
            now[b] = s1
        values.append(held * now.double()[:, :, None, None])
    return values[0], values[1].transpose(2, 3).contiguous()
