"""The operators that bring prompts into a transformer's paged cache, as cases that can be timed and compared.

A case is one pass through one operator: `page_tables` (pages for prompts of given lengths), `page_slots` (where the tokens of a packed
batch stand and go), `rotary` (queries and keys turned by their positions, keys and values into the cache) or `attend_prompts` (causal
attention of packed prompts, also behind tokens that the cache holds already).  Widths are those of this repository's models and examples
or generic ones; inputs are synthetic, as everywhere here.

`run` computes the plain form in elementary torch operations, or, with `own` set, calls the framework.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

TABLES = dict(op="tables", none=0)
SLOTS = dict(op="slots", past=0, pad=0)
ROTARY = dict(op="rotary", cache=False, page=0, interleaved=False, factor=1.0)
ATTEND = dict(op="attend", past_lo=0, past_hi=0, page=0, pad=0)


def listed():
    return [
        # one batch of eight utterances' prompts, five hypotheses each: a call of latency
        dict(TABLES, name="tables_8_prompts", prompts=8, beams=5, page=16, lo=10, hi=200, room=64),
        # many requests at once, every eleventh place without one
        dict(TABLES, name="tables_4096_prompts", prompts=4096, beams=4, page=16, lo=0, hi=4000, room=100, none=11),
        # N-best lists of eight utterances, some tokens of padding behind them
        dict(SLOTS, name="slots_40_prompts", prompts=40, page=16, lo=0, hi=60, pad=48),
        # a million tokens of prompts, each behind what the cache holds of it
        dict(SLOTS, name="slots_1000_prompts", prompts=1000, page=64, lo=100, hi=1999, past=3000),
        # the single token of five hypotheses: latency
        dict(ROTARY, name="rotary_5_tokens_f32", tokens=5, heads=8, kv=2, dim=64, rot=64, far=60, dtype="f32"),
        # prompts of a model with long contexts, keys and values into the cache
        dict(ROTARY, name="rotary_8000_tokens_bf16", tokens=8000, heads=32, kv=8, dim=128, rot=128, far=131071, dtype="bf16", cache=True, page=64, factor=8.0),
        # neighbouring dimensions as pairs, a part of the head
        dict(ROTARY, name="rotary_3001_tokens_f16", tokens=3001, heads=20, kv=4, dim=80, rot=32, far=8000, dtype="f16", interleaved=True, cache=True, page=16),
        # one hypothesis of 37 tokens under the example's small model: latency
        dict(ATTEND, name="prompts_1_short_f32", prompts=1, heads=8, kv=2, dim=32, lo=37, hi=37, dtype="f32"),
        # N-best lists of eight utterances, five hypotheses each, rescored together, padded to a fixed size
        dict(ATTEND, name="prompts_40_nbest_bf16", prompts=40, heads=8, kv=8, dim=64, lo=0, hi=60, dtype="bf16", pad=48),
        # a batch of ragged prompts, a head of odd size, three query heads to a key head
        dict(ATTEND, name="prompts_16_ragged_f16", prompts=16, heads=24, kv=8, dim=80, lo=1, hi=2047, dtype="f16"),
        # two long prompts
        dict(ATTEND, name="prompts_2_long_bf16", prompts=2, heads=32, kv=8, dim=128, lo=7001, hi=16000, dtype="bf16"),
        # a chunk each of four prompts whose beginnings the cache holds
        dict(ATTEND, name="prompts_4_chunks_bf16", prompts=4, heads=32, kv=4, dim=128, lo=100, hi=512, dtype="bf16", past_lo=20001, past_hi=60000, page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("tables", "slots", "rotary", "rotary", "attend", "attend", "attend"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    page = rng.choice((1, 8, 16, 32, 48, 64, 128))
    if op == "tables":
        while True:
            prompts, beams, hi, room = _log_int(rng, 1, 4096), rng.choice((1, 1, 2, 4, 5, 8, 16)), _log_int(rng, 1, 8000), _log_int(rng, 1, 500)
            if prompts * beams * ((hi + room) // page + 1) <= 4096 * 4 * 257:
                break
        return dict(TABLES, prompts=prompts, beams=beams, page=page, lo=rng.choice((0, hi // 2, hi)), hi=hi, room=room, none=rng.choice((0, 0, 7)))
    if op == "slots":
        while True:
            prompts, hi = _log_int(rng, 1, 4096), _log_int(rng, 1, 20000)
            if prompts * hi <= 1999 * 1000:
                break
        return dict(SLOTS, prompts=prompts, page=page, lo=rng.choice((0, hi // 2, hi)), hi=hi, past=rng.choice((0, 0, 777)), pad=rng.choice((0, 100)))
    kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 2, 3, 4, 8))
    dim = rng.choice((32, 64, 80, 96, 128, 128, 256))
    if op == "rotary":
        while True:
            tokens = _log_int(rng, 1, 16000)
            if tokens * kv * (group + 1) * dim * BYTES[dtype] <= 8000 * 48 * 128 * 2:
                break
        return dict(ROTARY, tokens=tokens, heads=kv * group, kv=kv, dim=dim, rot=rng.choice((dim, dim, dim // 2, dim // 4, 2 * rng.randint(1, dim // 2))),
                    far=_log_int(rng, 1, 1000000), dtype=dtype, cache=rng.random() < 0.5, page=page, interleaved=rng.random() < 0.4, factor=rng.choice((1.0, 1.0, 4.0)))
    while True:
        prompts, hi = _log_int(rng, 1, 64), _log_int(rng, 1, 16000)
        past = rng.choice((0, 0, 1)) * _log_int(rng, 1, 60000)
        c = dict(ATTEND, prompts=prompts, heads=kv * group, kv=kv, dim=dim, lo=rng.choice((0, hi // 2, hi)), hi=hi, dtype=dtype, past_lo=past // 2, past_hi=past,
                 page=page, pad=rng.choice((0, 0, 77)))
        if prompts * hi * (hi + past) * kv * group * dim <= (1 if dtype != "f32" else 0.1) * 16000 * 16000 * 32 * 128 and prompts * (hi + past) * kv * dim <= 240000 * 512:
            return c


# ---------------------------------------------------------------- what a program has in hand

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32 if dtype == torch.float32 else torch.float16)
    return x.mul_(scale).to(dtype)


def _spread(lo, hi, n):
    """Lengths evenly over [lo, hi], the longest not last."""
    x = np.linspace(lo, hi, n).round().astype(np.int64) if n > 1 else np.array([hi], np.int64)
    return np.roll(x, n // 3)


def _int32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def _pages(lens, page, seed):
    """Page tables of prompts that share nothing, pages in no order, -1 behind a prompt's last one."""
    need = -(-lens // page)
    width = max(1, int(need.max()))
    order = np.random.default_rng(seed).permutation(int(need.sum()))
    tables = np.full((len(lens), width), -1, np.int32)
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = order[at:at + n]
        at += int(n)
    return tables, max(1, at)


def _lengths(c):
    lens = _spread(c["lo"], c["hi"], c["prompts"])
    return lens, np.roll(_spread(c["past_lo"], c["past_hi"], c["prompts"]), 1)


def _frequencies(c):
    """Radians a position of every pair: base 10000, or, for long contexts, base 500000 with the slow ones slower by `factor`: pairs that turn less than
    once in 8192 / 1 positions wholly, those that turn more than four times not at all, in between by their number of turns."""
    half = c["rot"] // 2
    at = torch.arange(half, dtype=torch.float64) / half
    f = (10000.0 if c["factor"] == 1.0 else 500000.0) ** -at
    if c["factor"] != 1.0:
        keep = ((8192 * f / (2 * math.pi) - 1) / 3).clamp(0, 1)
        f = f * (keep + (1 - keep) / c["factor"])
    return f.cuda()


def prepare(case, seed):
    c, r = case, np.random.default_rng(seed)
    if c["op"] == "tables":
        lens = r.permutation(_spread(c["lo"], c["hi"], c["prompts"]))
        if c["none"]:
            lens[c["none"] - 1::c["none"]] = -1
        width = (c["hi"] + c["room"]) // c["page"] + 1
        most = int(((np.maximum(lens, 0) + c["room"]) // c["page"] + 1).sum()) * c["beams"]
        return dict(case=c, lens=_int32(lens), width=width, free=_int32(r.permutation(most + 100)), taken=_int32([r.integers(0, 100)]))
    if c["op"] == "slots":
        lens = r.permutation(_spread(c["lo"], c["hi"], c["prompts"]))
        past = r.integers(0, c["past"] + 1, c["prompts"])
        tables, _ = _pages(lens + past, c["page"], seed)
        return dict(case=c, lens=_int32(lens), past=_int32(past) if c["past"] else None, tables=torch.from_numpy(tables).cuda(), tokens=int(lens.sum()) + c["pad"])
    gen, dt = _gen(seed), DTYPES[c["dtype"]]
    heads, kv, dim = c["heads"], c["kv"], c["dim"]
    if c["op"] == "rotary":
        qkv = _randn(gen, (c["tokens"], heads + 2 * kv, dim), dt)   # as one product makes them
        s = dict(case=c, q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:], freqs=_frequencies(c),
                 positions=_int32(r.integers(0, c["far"] + 1, c["tokens"])))
        if c["cache"]:
            pages = -(-c["tokens"] * 5 // (4 * c["page"]))
            slots = r.permutation(pages * c["page"])[:c["tokens"]].astype(np.int64)
            slots[::50] = -1   # tokens that have no place
            s.update(slots=torch.from_numpy(slots).cuda(), k_cache=_randn(gen, (pages, c["page"], kv, dim), dt), v_cache=_randn(gen, (pages, c["page"], kv, dim), dt))
        return s
    lens, past = _lengths(c)
    tokens = int(lens.sum())
    qkv = _randn(gen, (tokens + c["pad"], heads + 2 * kv, dim), dt)
    s = dict(case=c, q=qkv[:, :heads].contiguous(), k=qkv[:, heads:heads + kv].contiguous(), v=qkv[:, heads + kv:],   # (queries and keys come from `rotary`)
             starts=_int32(np.concatenate([[0], np.cumsum(lens)])), lens=lens.tolist(), had=past.tolist(), past=None, k_cache=None, v_cache=None, tables=None)
    if c["past_hi"]:
        tables, pages = _pages(past, c["page"], seed)
        s.update(past=_int32(past), tables=torch.from_numpy(tables).cuda(), k_cache=_randn(gen, (pages, c["page"], kv, dim), dt),
                 v_cache=_randn(gen, (pages, c["page"], kv, dim), dt))
    return s


# ---------------------------------------------------------------- one pass

def run(state):
    return {"tables": _tables, "slots": _slots, "rotary": _rotary, "attend": _attend}[state["case"]["op"]](state)


def _tables(s):
    c = s["case"]
    beams, page, width = c["beams"], c["page"], s["width"]
    if own:
        from paper_2302_14357_amd import page_tables
        return page_tables(s["lens"], page=page, width=width, beams=beams, room=c["room"], free=s["free"], taken=s["taken"])
    n = s["lens"].long()
    whole, need = n // page, (n + c["room"] + page - 1) // page
    live = (n >= 0) & (need <= width)
    count = torch.where(live, whole + beams * (need - whole), 0)
    end = s["taken"].long() + torch.cumsum(count, 0)
    fits = live & ((end <= len(s["free"])) | (count == 0))
    base = end - count
    col = torch.arange(width, device=n.device)[None, None, :]
    row = torch.arange(beams, device=n.device)[None, :, None]
    n3, whole3, base3 = (need[:, None, None], whole[:, None, None], base[:, None, None])
    at = torch.where(col < whole3, base3 + col, base3 + whole3 + row * (n3 - whole3) + col - whole3)
    there = (col < n3) & fits[:, None, None]
    tables = torch.where(there, s["free"][torch.where(there, at, 0)], -1)
    lens = torch.where(fits[:, None] & (row[..., 0] == 0), n[:, None], -1)
    return tables.reshape(-1, width).int(), lens.reshape(-1).int(), (s["taken"] + torch.where(fits, count, 0).sum()).int()


def _slots(s):
    c, tokens, page = s["case"], s["tokens"], s["case"]["page"]
    if own:
        from paper_2302_14357_amd import page_slots
        return page_slots(s["lens"], s["tables"], page=page, tokens=tokens, past=s["past"])
    ends = torch.cumsum(s["lens"].long(), 0)
    starts = torch.cat([torch.zeros_like(ends[:1]), ends]).clamp(max=tokens)
    t = torch.arange(tokens, device=ends.device)
    prompt = torch.searchsorted(ends, t, right=True)
    inside = prompt < len(ends)
    prompt = prompt.clamp(max=len(ends) - 1)
    at = t - starts[prompt]
    if s["past"] is not None:
        at = at + s["past"][prompt]
    column = at // page
    entry = s["tables"][prompt, column.clamp(max=s["tables"].shape[1] - 1)].long()
    there = inside & (column < s["tables"].shape[1]) & (entry >= 0)
    return starts.int(), torch.where(inside, at, -1).int(), torch.where(there, entry * page + at % page, -1)


def _turn(x, cos, sin, interleaved):
    """x [tokens, heads, dim], cos and sin [tokens, pairs]."""
    half = cos.shape[1]
    y = x.float() if x.dtype != torch.float64 else x.clone()
    pairs = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    a, b = y[..., pairs[0]], y[..., pairs[1]]
    c, d = cos[:, None, :], sin[:, None, :]
    a, b = a * c - b * d, b * c + a * d
    y = y.clone()
    y[..., pairs[0]], y[..., pairs[1]] = a, b
    return y


def _rotary(s):
    c = s["case"]
    if own:
        from paper_2302_14357_amd import rotary
        if not c["cache"]:
            return rotary(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"])
        q, k = rotary(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"], v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], slots=s["slots"])
        return q, k, s["k_cache"], s["v_cache"]
    angle = s["positions"].double()[:, None] * s["freqs"]   # (radians of 10^6 positions leave 32 bits four digits)
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q, k = (_turn(s[x], cos, sin, c["interleaved"]).to(s["q"].dtype) for x in ("q", "k"))
    if not c["cache"]:
        return q, k
    there = s["slots"] >= 0
    into = s["slots"][there]
    s["k_cache"].view(-1, c["kv"], c["dim"])[into] = k[there]
    s["v_cache"].view(-1, c["kv"], c["dim"])[into] = s["v"][there]
    return q, k, s["k_cache"], s["v_cache"]


def _attend(s):
    c = s["case"]
    if own:
        from paper_2302_14357_amd import attend_prompts
        return attend_prompts(s["q"], s["k"], s["v"], s["starts"], past=s["past"], k_cache=s["k_cache"], v_cache=s["v_cache"], tables=s["tables"])
    kv, dim, group = c["kv"], c["dim"], c["heads"] // c["kv"]
    out = torch.zeros_like(s["q"])   # rows of no prompt
    at = 0
    for i, (n, past) in enumerate(zip(s["lens"], s["had"])):   # (a program knows the lengths it has packed)
        if n == 0:
            continue
        k, v = (s[x][at:at + n].float() for x in ("k", "v"))
        if past:
            pages = s["tables"][i, :-(-past // c["page"])].long()
            k, v = (torch.cat([s[x][pages].reshape(-1, kv, dim)[:past].float(), y]) for x, y in (("k_cache", k), ("v_cache", v)))
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()
        for j in range(0, n, 1024):   # the scores of all queries at once would not fit
            m = min(1024, n - j)
            seen = past + j + m
            q = s["q"][at + j:at + j + m].float().reshape(m, kv, group, dim).permute(1, 0, 2, 3).reshape(kv, m * group, dim)
            a = torch.matmul(q, k[:, :, :seen]).reshape(kv, m, group, seen) / math.sqrt(dim)
            later = torch.arange(seen, device=a.device)[None, :] > past + j + torch.arange(m, device=a.device)[:, None]
            a = a.masked_fill(later[None, :, None, :], -math.inf)
            p = torch.exp(a - a.amax(-1, keepdim=True))
            o = torch.matmul(p.reshape(kv, m * group, seen), v[:, :seen]) / p.reshape(kv, m * group, seen).sum(-1, keepdim=True)
            out[at + j:at + j + m] = o.reshape(kv, m, group, dim).permute(1, 0, 2, 3).reshape(m, c["heads"], dim).to(out.dtype)
        at += n
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c = case
    if c["op"] == "tables":
        lens = _spread(c["lo"], c["hi"], c["prompts"])
        live = (np.arange(len(lens)) + 1) % c["none"] != 0 if c["none"] else np.ones(len(lens), bool)
        whole, need = lens // c["page"], -(-(lens + c["room"]) // c["page"])
        pages = int(((whole + c["beams"] * (need - whole)) * live).sum())
        rows, width = c["prompts"] * c["beams"], (c["hi"] + c["room"]) // c["page"] + 1
        return {"bytes": 4 * (len(lens) + pages + rows * (width + 1) + 2), "flops": 0}
    if c["op"] == "slots":
        lens = _spread(c["lo"], c["hi"], c["prompts"])
        tokens, pages = int(lens.sum()), int((-(-lens // c["page"])).sum())
        return {"bytes": 12 * (tokens + c["pad"]) + 4 * (2 * len(lens) + 1 + (len(lens) if c["past"] else 0) + pages), "flops": 0}
    b = BYTES[c["dtype"]]
    if c["op"] == "rotary":
        elements = 2 * (c["heads"] + c["kv"]) + (3 * c["kv"] if c["cache"] else 0)   # a cache: keys once more, values read and written
        return {"bytes": c["tokens"] * (elements * c["dim"] * b + 4 + (8 if c["cache"] else 0)) + 8 * (c["rot"] // 2), "flops": 3 * c["tokens"] * (c["heads"] + c["kv"]) * c["rot"]}
    lens, past = _lengths(c)
    past = np.where(lens > 0, past, 0)
    tokens, had, width = int(lens.sum()), int(past.sum()), c["heads"] * c["dim"]
    seen = int((lens * past + lens * (lens + 1) // 2).sum())
    return {"bytes": b * (2 * tokens + c["pad"]) * width + 2 * b * (tokens + had) * c["kv"] * c["dim"] + 4 * (len(lens) + 1), "flops": 4 * seen * width}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c = case
    if c["op"] in ("tables", "slots"):
        return None
    s = prepare(case, seed)
    if c["op"] == "rotary":
        angle = s["positions"].double()[:, None] * s["freqs"]
        unit = torch.polar(torch.ones_like(angle), angle)[:, None, :]
        half, out = c["rot"] // 2, []
        for x in (s["q"].double(), s["k"].double()):
            head, tail = x[..., :2 * half], x[..., 2 * half:]
            pairs = head.unflatten(-1, (half, 2)) if c["interleaved"] else head.unflatten(-1, (2, half)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
            out.append(torch.cat([(z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2), tail], -1))
        if not c["cache"]:
            return tuple(out)
        cache = s["k_cache"].double().flatten(0, 1)
        there = (s["slots"] >= 0).nonzero()[:, 0]
        cache.index_copy_(0, s["slots"][there], out[1][there])
        return out[0], out[1], cache.view_as(s["k_cache"]), None
    if work(c)["flops"] > 6e12:
        return None
    kv, dim = c["kv"], c["dim"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    edges = s["starts"].tolist()
    for i, (first, end) in enumerate(zip(edges, edges[1:])):
        had = s["had"][i]
        for h in range(kv if end > first else 0):
            k, v = s["k"][first:end, h].double(), s["v"][first:end, h].double()
            if had:
                pages = s["tables"][i].long().clamp(min=0)
                k = torch.cat([s["k_cache"][pages, :, h].double().flatten(0, 1)[:had], k])
                v = torch.cat([s["v_cache"][pages, :, h].double().flatten(0, 1)[:had], v])
            kt = k.t().contiguous()
            for head in range(h * (c["heads"] // kv), (h + 1) * (c["heads"] // kv)):
                for j in range(first, end, 4096):
                    rows = s["q"][j:min(j + 4096, end), head].double()
                    n = had + j - first + len(rows)
                    a = (rows @ kt[:, :n]) * dim ** -0.5
                    a = a + torch.full_like(a, -math.inf).triu(had + j - first + 1)
                    out[j:j + len(rows), head] = torch.log_softmax(a, -1).exp() @ v[:n]
    return out
