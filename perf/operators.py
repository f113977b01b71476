"""The operators of one step of a transformer's beam decode, as cases that can be timed and compared.

A case is one pass through one operator: `linear` (product with bias, activation and residual), `attend_paged` (one new
token over a paged cache of keys and values), `beam_select` (the best of beams x vocabulary) or `beam_reorder` (page tables,
lengths and partly filled pages follow the chosen hypotheses).  Widths are those of this repository's models (512, 640, 1024;
vocabularies of 1024 and 4096) or generic ones; inputs are synthetic, as everywhere here.

`run` computes the plain form in elementary torch operations, or, with `own` set, calls the framework.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}

LINEAR = dict(op="linear", act="none", bias=True, residual=False)
ATTEND = dict(op="attend", tail=0, done=0)
SELECT = dict(op="select", done=0)
REORDER = dict(op="reorder")


def listed():
    return [
        # five hypotheses of one utterance through the first product of a feed-forward block: a call of latency
        dict(LINEAR, name="linear_5_640_2560_bf16", m=5, k=640, n=2560, dtype="bf16", act="relu"),
        # the second product of the block for 64 utterances of five hypotheses, with its residual, in single precision
        dict(LINEAR, name="linear_320_2048_512_f32", m=320, k=2048, n=512, dtype="f32", residual=True),
        # a batch of rows as a prompt has them
        dict(LINEAR, name="linear_8000_1024_4096_bf16", m=8000, k=1024, n=4096, dtype="bf16", act="gelu", residual=True),
        # one utterance of five hypotheses, eight heads of 64, a short history: latency
        dict(ATTEND, name="attend_5_rows_f32", utts=1, beams=5, heads=8, kv=8, dim=64, page=16, lo=50, hi=50, dtype="f32", tail=10),
        # 64 utterances of five hypotheses, ragged histories from no token on, every seventh hypothesis finished
        dict(ATTEND, name="attend_320_rows_bf16", utts=64, beams=5, heads=8, kv=8, dim=64, page=16, lo=0, hi=400, dtype="bf16", tail=30, done=7),
        # four long histories, eight query heads to a key head: split over the length
        dict(ATTEND, name="attend_4_long_bf16", utts=4, beams=1, heads=32, kv=4, dim=128, page=64, lo=100001, hi=131071, dtype="bf16"),
        # 32 utterances of eight hypotheses that share a long prompt's pages
        dict(ATTEND, name="attend_256_shared_f16", utts=32, beams=8, heads=32, kv=8, dim=128, page=32, lo=1500, hi=4000, dtype="f16", tail=77),
        # the small vocabulary, one utterance
        dict(SELECT, name="select_5_1024_f32", utts=1, beams=5, vocab=1024, dtype="f32"),
        # 64 utterances, a word-piece vocabulary of odd size, some hypotheses finished
        dict(SELECT, name="select_320_32001_bf16", utts=64, beams=5, vocab=32001, dtype="bf16", done=9),
        # a wide beam over a large vocabulary
        dict(SELECT, name="select_512_131000_f32", utts=32, beams=16, vocab=131000, dtype="f32"),
        # one utterance, a model of four layers
        dict(REORDER, name="reorder_5_rows_4_layers", utts=1, beams=5, layers=4, kv=8, dim=64, page=16, lo=50, hi=50, extra=2, dtype="f32"),
        # 64 utterances of eight hypotheses, twelve layers, pages of 64 tokens
        dict(REORDER, name="reorder_512_rows_12_layers", utts=64, beams=8, layers=12, kv=8, dim=128, page=64, lo=30, hi=250, extra=4, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "attend", "attend", "select", "reorder"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    if op == "linear":
        while True:
            m, k, n = _log_int(rng, 1, 8000), _log_int(rng, 16, 5000), _log_int(rng, 16, 5000)
            if rng.random() < 0.5:   # widths of whole pieces as well as odd ones
                k, n = (k + 63) // 64 * 64, (n + 63) // 64 * 64
            if m * k * n <= (8000 * 1024 * 4096 if dtype != "f32" else 1000 * 1024 * 4096):
                break
        return dict(LINEAR, m=m, k=k, n=n, dtype=dtype, act=rng.choice(("none", "relu", "gelu", "silu", "tanh")),
                    bias=rng.random() < 0.7, residual=rng.random() < 0.5)
    if op == "attend":
        while True:
            beams, utts = rng.choice((1, 1, 2, 5, 8)), _log_int(rng, 1, 64)
            kv, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 2, 3, 4, 8, 16))
            dim, page, hi = rng.choice((32, 64, 80, 96, 128, 128, 256)), rng.choice((8, 16, 32, 48, 64, 128)), _log_int(rng, 1, 131071)
            if utts * beams * hi * kv * dim * BYTES[dtype] <= 4 * 115536 * 4 * 128 * 2:
                break
        return dict(ATTEND, utts=utts, beams=beams, heads=kv * group, kv=kv, dim=dim, page=page, lo=rng.choice((0, hi // 2, hi)), hi=hi,
                    dtype=dtype, tail=rng.randint(0, 100), done=rng.choice((0, 0, 5)))
    if op == "select":
        while True:
            beams, utts, vocab = rng.randint(1, 32), _log_int(rng, 1, 256), _log_int(rng, 2, 262144)
            if utts * beams * vocab * BYTES[dtype] <= 512 * 131000 * 4:
                break
        return dict(SELECT, utts=utts, beams=beams, vocab=vocab, dtype=dtype, done=rng.choice((0, 0, 4)))
    beams = rng.randint(1, 16)
    while True:
        utts, layers, hi = _log_int(rng, 1, 64), rng.randint(1, 24), _log_int(rng, 1, 500)
        kv, dim, page = rng.choice((1, 4, 8)), rng.choice((64, 128)), rng.choice((8, 16, 48, 64))
        if utts * beams * layers * 2 * kv * dim * (hi + 2 * page) * BYTES[dtype] <= 512 * 24 * 8 * 128 * 256 * 2:
            break
    return dict(REORDER, utts=utts, beams=beams, layers=layers, kv=kv, dim=dim, page=page, lo=rng.choice((0, hi // 2, hi)), hi=hi,
                extra=rng.randint(0, beams - 1), dtype=dtype)


# ---------------------------------------------------------------- what a program has in hand

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, shape, dtype, scale=1.0):
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32 if dtype == torch.float32 else torch.float16)
    return x.mul_(scale).to(dtype)


def _lengths(c):
    """Tokens of every utterance: evenly over [lo, hi], the longest not last."""
    x = np.linspace(c["lo"], c["hi"], c["utts"]).round().astype(np.int64) if c["utts"] > 1 else np.array([c["hi"]], np.int64)
    return np.roll(x, c["utts"] // 3)


def _layout(c):
    """(tokens of each utterance, whole pages its beams share, pages of a row): a prompt is shared, the last tokens are a row's own."""
    lens = _lengths(c)
    shared = np.maximum(lens - c["tail"], 0) // c["page"] if c["beams"] > 1 else np.zeros_like(lens)
    return lens, shared, int(lens.max()) // c["page"] + 1


def _tables(c, seed):
    """Page tables [rows, pages of a row] over pages in no order; -1 where a row has none yet."""
    lens, shared, width = _layout(c)
    need = lens // c["page"] + 1
    counts = shared + c["beams"] * (need - shared)
    order = np.random.default_rng(seed).permutation(int(counts.sum()))
    tables = np.full((c["utts"], c["beams"], width), -1, np.int32)
    at = 0
    for u in range(c["utts"]):
        s, n = int(shared[u]), int(need[u])
        tables[u, :, :s] = order[at:at + s]
        tables[u, :, s:n] = order[at + s:at + s + c["beams"] * (n - s)].reshape(c["beams"], n - s)
        at += int(counts[u])
    return lens, tables.reshape(-1, width), int(counts.sum())


def _row_lengths(c, lens):
    rows = np.repeat(lens, c["beams"])
    if c["done"]:
        rows[c["done"] - 1::c["done"]] = ~rows[c["done"] - 1::c["done"]]   # finished hypotheses take no part
    return rows.astype(np.int32)


def prepare(case, seed):
    c, gen = case, _gen(seed)
    dt = DTYPES[c["dtype"]]
    if c["op"] == "linear":
        a = math.sqrt(6.0 / (c["k"] + c["n"]))
        w = (torch.rand((c["n"], c["k"]), generator=gen, device="cuda") * (2 * a) - a).to(dt)
        return dict(case=c, x=_randn(gen, (c["m"], c["k"]), dt), w=w,
                    bias=torch.rand(c["n"], generator=gen, device="cuda") * 0.1 - 0.05 if c["bias"] else None,
                    residual=_randn(gen, (c["m"], c["n"]), dt) if c["residual"] else None)
    if c["op"] == "attend":
        lens, tables, pages = _tables(c, seed)
        rows = len(tables)
        cache = (pages, c["page"], c["kv"], c["dim"])
        return dict(case=c, q=_randn(gen, (rows, c["heads"], c["dim"]), dt), k_new=_randn(gen, (rows, c["kv"], c["dim"]), dt),
                    v_new=_randn(gen, (rows, c["kv"], c["dim"]), dt), k=_randn(gen, cache, dt), v=_randn(gen, cache, dt),
                    tables=torch.from_numpy(tables).cuda(), lens=torch.from_numpy(_row_lengths(c, lens)).cuda(), max_len=int(lens.max()) + 1)
    if c["op"] == "select":
        rows = c["utts"] * c["beams"]
        done = torch.zeros(rows, dtype=torch.bool, device="cuda")
        if c["done"]:
            done[c["done"] - 1::c["done"]] = True
        # scores of hypotheses that have survived some steps: some nats apart
        return dict(case=c, logits=_randn(gen, (rows, c["vocab"]), dt, 3.0), done=done,
                    scores=-40.0 - 3.0 * torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64))
    lens = _lengths(c)
    rows, width = c["utts"] * c["beams"], (int(lens.max()) + 1) // c["page"] + 1
    r = np.random.default_rng(seed)
    tables = r.permutation(rows * width).astype(np.int32).reshape(rows, width)   # a row's pages are reserved ahead
    # `extra` children of every utterance have a parent that another child has already
    parents = np.stack([r.permutation(np.concatenate([k := r.permutation(c["beams"])[:c["beams"] - c["extra"]], r.choice(k, c["extra"])]))
                        for _ in range(c["utts"])]).astype(np.int32)
    cache = (rows * width, c["page"], c["kv"], c["dim"])
    return dict(case=c, tables=torch.from_numpy(tables).cuda(), lens=torch.from_numpy(np.repeat(lens, c["beams"]).astype(np.int32)).cuda(),
                parents=torch.from_numpy(parents.reshape(-1)).cuda(), done=torch.zeros(rows, dtype=torch.bool, device="cuda"),
                caches=[_randn(gen, cache, dt) for _ in range(2 * c["layers"])])


# ---------------------------------------------------------------- one pass

def run(state):
    return {"linear": _linear, "attend": _attend, "select": _select, "reorder": _reorder}[state["case"]["op"]](state)


def _linear(s):
    c = s["case"]
    if own:
        from paper_2302_14357_amd import linear
        return linear(s["x"], s["w"], s["bias"], act=c["act"], residual=s["residual"])
    y = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        y = y + s["bias"]
    y = {"none": lambda t: t, "relu": lambda t: t.clamp(min=0), "gelu": lambda t: 0.5 * t * (1 + torch.erf(t * math.sqrt(0.5))),
         "silu": lambda t: t / (1 + torch.exp(-t)), "tanh": torch.tanh}[c["act"]](y)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _attend(s):
    c = s["case"]
    if own:
        from paper_2302_14357_amd import attend_paged
        out = attend_paged(s["q"], s["k"], s["v"], s["tables"], s["lens"], k_new=s["k_new"], v_new=s["v_new"], beams=c["beams"],
                           max_len=s["max_len"])
        return out, s["k"], s["v"]
    rows, heads, dim = s["q"].shape
    kv, page = c["kv"], c["page"]
    live = s["lens"] >= 0
    at = s["lens"].clamp(min=0).long()
    into = s["tables"].gather(1, (at // page)[:, None])[:, 0].long()
    s["k"][into[live], (at % page)[live]] = s["k_new"][live]
    s["v"][into[live], (at % page)[live]] = s["v_new"][live]
    n = torch.where(live, at + 1, 0)
    pages = s["tables"].clamp(min=0).long()
    length = pages.shape[1] * page
    k = s["k"][pages].float().reshape(rows, length, kv, dim).permute(0, 2, 3, 1).contiguous()
    v = s["v"][pages].float().reshape(rows, length, kv, dim).permute(0, 2, 1, 3).contiguous()
    a = torch.matmul(s["q"].float().reshape(rows, kv, heads // kv, dim), k) / math.sqrt(dim)
    seen = torch.arange(length, device=a.device)[None, :] < n[:, None]
    a = a.masked_fill(~seen[:, None, None, :], -math.inf)
    p = torch.exp(a - a.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.reshape(rows, heads, dim).to(s["q"].dtype), s["k"], s["v"]


def _select(s):
    c = s["case"]
    beams, eos = c["beams"], c["vocab"] - 1
    if own:
        from paper_2302_14357_amd import beam_select
        return beam_select(s["logits"], s["scores"], beams=beams, finished=s["done"], eos=eos)
    # 64 bits: candidates of two hypotheses can lie closer than 32 bits tell apart
    m = min(beams, c["vocab"])
    l, token = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    l, token = l[:, :m].double(), token[:, :m]
    x = s["logits"].double()
    top = x.amax(1, keepdim=True)
    score = s["scores"][:, None] + (l - (top + torch.log(torch.exp(x - top).sum(1, keepdim=True))))
    alone = torch.arange(m, device=l.device)[None, :] == 0
    done = s["done"][:, None]
    score = torch.where(done, torch.where(alone, s["scores"][:, None], -math.inf), score)
    token = torch.where(done, eos, token)
    score = torch.nan_to_num(score, nan=-math.inf, neginf=-math.inf, posinf=math.inf).reshape(c["utts"], beams * m)
    best, order = torch.sort(score, dim=1, descending=True, stable=True)
    best, order = best[:, :beams], order[:, :beams]
    none = best == -math.inf
    parent = torch.where(none, -1, order // m)
    token = torch.where(none, -1, token.reshape(c["utts"], beams * m).gather(1, order))
    ended = none | (token == eos) | s["done"].reshape(c["utts"], beams).gather(1, parent.clamp(min=0))
    return best.reshape(-1), token.reshape(-1).int(), parent.reshape(-1).int(), ended.reshape(-1)


def _reorder(s):
    c = s["case"]
    beams, page = c["beams"], c["page"]
    if own:
        from paper_2302_14357_amd import beam_reorder
        tables, lens = beam_reorder(s["parents"], s["tables"], s["lens"], s["caches"], beams=beams, finished=s["done"])
        return [tables, lens] + s["caches"]
    parent = s["parents"].reshape(-1, beams).long()
    same = parent[:, :, None] == parent[:, None, :]
    index = torch.arange(beams, device=parent.device)
    first = ~(same & (index[None, :, None] > index[None, None, :])).any(2)
    childless = ~(parent[:, :, None] == index).any(1)
    # the k-th child that needs a row's tail takes that of the k-th row without children
    giver = torch.argsort((~childless).int(), dim=1, stable=True).gather(1, (torch.cumsum((~first).int(), 1) - 1).clamp(min=0))
    base = (torch.arange(parent.shape[0], device=parent.device) * beams)[:, None]
    rows = (parent + base).reshape(-1)
    tail = torch.where(first, parent, giver).add(base).reshape(-1)
    lens = s["lens"][rows] + 1
    full = (lens // page).long()[:, None]
    tables = torch.where(torch.arange(s["tables"].shape[1], device=parent.device)[None, :] < full, s["tables"][rows], s["tables"][tail])
    # the tokens of a partly filled page that two rows would go on writing; others copy a page of their own onto itself
    at = full.clamp(max=s["tables"].shape[1] - 1)
    into, source = tables.gather(1, at)[:, 0].long(), torch.where(first.reshape(-1), tables.gather(1, at)[:, 0], s["tables"][rows].gather(1, at)[:, 0]).long()
    part = (torch.arange(page, device=parent.device)[None, :] < (lens % page)[:, None])[:, :, None, None]
    for cache in s["caches"]:
        cache[into] = torch.where(part, cache[source], cache[into])
    return [tables, torch.where(s["done"], ~lens, lens)] + s["caches"]


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    c, b = case, BYTES[case["dtype"]]
    if c["op"] == "linear":
        m, k, n = c["m"], c["k"], c["n"]
        return {"bytes": b * (m * k + n * k + m * n * (2 if c["residual"] else 1)) + 4 * n * c["bias"], "flops": 2 * m * n * k}
    if c["op"] == "attend":
        lens, shared, width = _layout(c)
        rows = _row_lengths(c, lens)
        live = (rows >= 0).reshape(c["utts"], c["beams"])
        tokens = int((np.where(live.any(1), shared * c["page"], 0) + live.sum(1) * (lens - shared * c["page"])).sum())
        d, n = c["dim"], int(live.sum())
        return {"bytes": b * (2 * tokens * c["kv"] * d + n * (2 * c["heads"] + 4 * c["kv"]) * d) + 4 * n * width,
                "flops": 4 * int((rows[rows >= 0] + 1).sum()) * c["heads"] * d}
    rows = c["utts"] * c["beams"]
    if c["op"] == "select":
        live = rows - (rows // c["done"] if c["done"] else 0)
        return {"bytes": b * live * c["vocab"] + 34 * rows, "flops": 4 * live * c["vocab"]}
    lens = _lengths(c) + 1
    tokens = int((lens % c["page"]).sum()) * c["extra"]
    return {"bytes": 2 * b * tokens * 2 * c["layers"] * c["kv"] * c["dim"] + 8 * rows * (int(lens.max()) // c["page"] + 1) + 13 * rows, "flops": 0}


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "linear":
        w, out = s["w"].double(), []
        for x in s["x"].split(1024):
            y = torch.nn.functional.linear(x.double(), w, None if s["bias"] is None else s["bias"].double())
            if c["act"] == "relu":
                y = torch.where(y > 0, y, 0.0)
            elif c["act"] == "gelu":
                y = y * torch.special.ndtr(y)
            elif c["act"] == "silu":
                y = y * torch.special.expit(y)
            elif c["act"] == "tanh":
                y = 1 - 2 / (torch.exp(2 * y) + 1)
            out.append(y)
        y = torch.cat(out)
        return y if s["residual"] is None else y + s["residual"].double()
    if c["op"] == "attend":
        rows = []
        for r, n in enumerate(s["lens"].tolist()):
            q = s["q"][r].double().reshape(c["kv"], -1, c["dim"])
            if n < 0:
                rows.append(torch.zeros_like(q).reshape(-1, c["dim"]))
                continue
            pages = s["tables"][r, :-(-n // c["page"])].long()
            k, v = (torch.cat([s[x][pages].reshape(-1, c["kv"], c["dim"])[:n], s[y][r][None]]).double().transpose(0, 1).contiguous()
                    for x, y in (("k", "k_new"), ("v", "v_new")))
            a = torch.log_softmax((q @ k.transpose(1, 2).contiguous()) * c["dim"] ** -0.5, -1)
            rows.append((a.exp() @ v).reshape(-1, c["dim"]))
        return torch.stack(rows), None, None
    if c["op"] == "select":
        best = []
        for u in range(c["utts"]):
            at = slice(u * c["beams"], (u + 1) * c["beams"])
            all_ = s["scores"][at, None] + torch.log_softmax(s["logits"][at].double(), 1)
            all_[s["done"][at]] = -math.inf
            every = torch.cat([all_.reshape(-1), s["scores"][at][s["done"][at]]])
            got = torch.sort(every, descending=True).values[:c["beams"]]
            best.append(torch.cat([got, got.new_full((c["beams"] - len(got),), -math.inf)]))
        return torch.cat(best), None, None, None
    return None
