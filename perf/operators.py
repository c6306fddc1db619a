"""Operators of a serving worker's decode step: what a program that runs one has them do.

The scheduler places requests on workers; these are the operators of the worker itself, over the requests
that it holds. Keys and values lie in pages of a pool, a table names each request's pages, and every pass
works on all requests of the worker at once:

* ``attend``: attention of a step's new tokens over the cached tokens of their requests. The new tokens of
  a request form a tree of drafted tokens (one token: plain decoding; a chain: a piece of a prompt); a token
  sees its request's cached tokens, its ancestors and itself. Query heads share key heads in groups.
* ``accept``: the drafted tokens that the verification kept enter the cache, and the attention weight that
  their rows gave every cached token is added to that token's accumulated weight.
* ``evict``: requests over their budget drop, per key head, the cached tokens of least accumulated weight
  outside a window of recent positions; the survivors behind the budget move into the holes before it.
* ``logprobs``: log probabilities of given tokens, with the entropy, the rank and the top alternatives.

Lengths follow the package's workload recipe: lognormal prompts, generated tokens uniform below a lognormal
prediction, at most 8,192 tokens a request; longer contexts where a case says so (131,072 tokens is the KV
capacity of the recipe's larger workers). Head counts, vocabularies and page sizes are generic.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HEADS = [(32, 8), (32, 32), (64, 8), (28, 4), (8, 1), (16, 2), (12, 12)]
VOCABS = [32000, 50257, 128256]
#: a drawn case's floor in seconds at 7 TB/s and 2 PFLOP/s, and the scores of its padded plain form
MOST_SECONDS, MOST_SCORES = 1.3e-4, 1.2e9


def _cache_case(name, op, requests, ctx, most, heads, dim, page, kind, lens, **more):
    """``ctx``, ``most``: mean and largest cached length; ``tree``: most drafted tokens a request; ``lens``
    seeds the lengths, so that a case has the same ones on every input; ``rows``: the pool's order, pages of
    ``hnd`` (head, token, channel) or ``nhd`` (token, head, channel)."""
    case = dict(op=op, requests=requests, ctx=ctx, most=most, q_heads=heads[0], kv_heads=heads[1], dim=dim,
                page=page, kind=kind, lens=lens, tree=1, rows="hnd", weigh=True, budget=0, recent=0)
    case.update(more)
    if name:
        case["name"] = name
    return case


def _logit_case(name, rows, vocab, kind, top):
    case = dict(op="logprobs", rows=rows, vocab=vocab, kind=kind, top=top)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One request alone on a worker, one new token: the smallest step, where latency counts.
        _cache_case("attend_one", "attend", 1, 640, 1000, (32, 8), 128, 64, "bf16", 3),
        # A decode step of a worker of the recipe: 128 requests of a few hundred tokens each.
        _cache_case("attend_128", "attend", 128, 640, 8192, (32, 8), 128, 64, "bf16", 4),
        # Verification of drafted trees of up to 64 tokens: products count as much as bytes.
        _cache_case("attend_trees", "attend", 24, 3000, 8192, (64, 8), 128, 32, "f16", 5, tree=64),
        # Odd groups and an odd head dimension, short chains, a pool in token-major order.
        _cache_case("attend_odd", "attend", 37, 1500, 5001, (28, 4), 96, 16, "bf16", 6, tree=5, rows="nhd"),
        # Few long requests without shared heads: one long axis, split and joined.
        _cache_case("attend_long", "attend", 2, 60000, 65536, (32, 32), 64, 16, "f16", 7),
        # Every request of a worker keeps one token a step and adds up its attention weight.
        _cache_case("accept_128", "accept", 128, 640, 8192, (32, 8), 128, 64, "bf16", 4),
        # A few tokens of every tree are kept; long requests, shared heads.
        _cache_case("accept_trees", "accept", 24, 3000, 8192, (64, 8), 128, 32, "f16", 5, tree=12),
        # A worker at its budget: every request is one token over it.
        _cache_case("evict_step", "evict", 64, 1025, 1025, (32, 8), 128, 64, "bf16", 8, budget=1024, recent=128),
        # Long requests cut down to a quarter.
        _cache_case("evict_long", "evict", 3, 60000, 65536, (32, 8), 128, 16, "f16", 9, budget=15001, recent=512),
        # One token's answer: the smallest vocabulary, five alternatives.
        _logit_case("logprobs_one", 1, 32000, "f32", 5),
        # A verification step: the rows of every drafted token, twenty alternatives each.
        _logit_case("logprobs_trees", 777, 128256, "bf16", 20),
        # A prompt is scored: its tokens' probabilities, an odd vocabulary, no alternatives.
        _logit_case("logprobs_prompt", 2049, 50257, "f32", 0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dear(case):
    w = work(case)
    if max(w["bytes"] / 7e12, w["flops"] / 2e15) > MOST_SECONDS:
        return True
    if case["op"] == "logprobs":
        return False
    return case["requests"] * case["q_heads"] * case["tree"] * max(_lengths(case)) > MOST_SCORES


def draw(rng):
    op = rng.choice(["attend", "attend", "accept", "evict", "logprobs"])
    while True:
        if op == "logprobs":
            case = _logit_case("", _log_int(rng, 1, 4000), rng.choice(VOCABS + [_log_int(rng, 100, 200000)]),
                               rng.choice(["bf16", "f16", "f32"]), rng.choice([0, 1, 5, 20, 64]))
        else:
            ctx = _log_int(rng, 40, 60000)
            case = _cache_case("", op, _log_int(rng, 1, 200), ctx, int(ctx * rng.uniform(1.0, 2.5)) + 1, rng.choice(HEADS),
                               rng.choice([64, 64, 96, 128, 128, 128, 256]), rng.choice([16, 32, 64, 128]),
                               rng.choice(["bf16", "f16"]), rng.randrange(1 << 30), rows=rng.choice(["hnd", "hnd", "nhd"]))
            if op == "evict":
                case["budget"] = max(1, int(ctx * rng.uniform(0.2, 1.0)))
                case["recent"] = int(case["budget"] * rng.uniform(0.0, 0.5))
            else:
                case["tree"] = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
                case["weigh"] = rng.random() < 0.8
        if not _dear(case):
            return case


# ---------------------------------------------------------------------------------------------------------
# The lengths of a case and what it cannot do without.

def _lengths(case):
    """Cached tokens of every request: lognormal of mean ``ctx`` up to ``most``; where several requests share
    the worker the second has no cached token yet, and the third's tokens end with a page."""
    rng = np.random.default_rng(case["lens"])
    n, s = case["requests"], 0.6
    x = np.rint(rng.lognormal(math.log(case["ctx"]) - 0.5 * s * s, s, n))
    x = np.clip(x, 1, case["most"]).astype(np.int64)
    if case["most"] == case["ctx"]:
        x[:] = case["ctx"]
    elif n > 3:
        x[1] = 0
        x[2] = max(case["page"], x[2] // case["page"] * case["page"])
    return x.tolist()


def _counts(case):
    """Drafted tokens of every request (up to ``tree``), and how many of them are kept."""
    rng = np.random.default_rng(case["lens"] + 1)
    n, t = case["requests"], case["tree"]
    toks = rng.integers((t + 1) // 2, t + 1, n)
    return toks.tolist(), np.minimum(toks, 1 + rng.integers(0, min(t, 6), n)).tolist()


def _width(case):
    """Entries of a row of the page table."""
    return -(-(max(_lengths(case)) + case["tree"]) // case["page"])


def work(case):
    if case["op"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        return {"bytes": n * v * (4 if case["kind"] == "f32" else 2) + n * (16 + 8 * case["top"]), "flops": 4 * n * v}
    lens, (toks, kept) = _lengths(case), _counts(case)
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    if case["op"] == "attend":
        n = sum(toks)
        return {"bytes": 4 * d * hk * (sum(lens) + n) + n * hq * (4 * d + 4),
                "flops": 4 * d * hq * sum(t * (c + 1) for t, c in zip(toks, lens))}
    if case["op"] == "accept":
        n = sum(kept)
        moved = 8 * d * hk * n
        if not case["weigh"]:
            return {"bytes": moved + 8 * hk * n, "flops": 1}
        return {"bytes": moved + hk * (2 * d + 8) * sum(lens) + n * hq * (2 * d + 4),
                "flops": 2 * d * hq * sum(t * (c + 1) for t, c in zip(kept, lens))}
    over = [c for c in lens if c > case["budget"]]
    b, r = case["budget"], case["recent"]
    # what lies behind the budget and stays: its recent tokens, of the others as many as chance has there
    move = sum(min(c - b, r) + max(0, c - b - r) * (b - r) / max(1, c - r) for c in over)
    return {"bytes": int(hk * (8 * sum(over) + move * (8 * d + 8))), "flops": hk * sum(over) + 1}


# ---------------------------------------------------------------------------------------------------------
# What a worker's program has in hand.

def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    kind = TYPES[case["kind"]]

    def normal(*shape, scale=1.0, kind=kind):
        return torch.randn(shape, generator=g, device=dev, dtype=kind).mul_(scale)

    def ints(x):
        return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(dev)

    if case["op"] == "logprobs":
        n, v = case["rows"], case["vocab"]
        logits = normal(n, v, scale=2.5)
        # a few tokens stand out, and the given one is often among them
        peak = torch.randint(0, v, (n, 8), generator=g, device=dev)
        logits.scatter_add_(1, peak, (6.0 + 3.0 * torch.randn((n, 8), generator=g, device=dev)).to(kind))
        pick = torch.randint(0, v, (n,), generator=g, device=dev)
        token = torch.where(torch.rand((n,), generator=g, device=dev) < 0.7, peak[:, 0], pick).to(torch.int32)
        return {"case": case, "logits": logits, "token": token}

    lens, (toks, kept) = _lengths(case), _counts(case)
    n, width, page = case["requests"], _width(case), case["page"]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    # every request has pages for its cached and its new tokens, in any order; entries behind are unused
    need = [-(-(c + t) // page) for c, t in zip(lens, toks)]
    pages = sum(need) + 3
    order = rng.permutation(pages)
    table = np.full((n, width), -1, np.int32)
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = order[at:at + m]
        at += m
    shape = (pages, page, hk, d) if case["rows"] == "nhd" else (pages, hk, page, d)
    k, v = normal(*shape), normal(*shape)
    if case["rows"] == "nhd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    # accumulated weights: most tokens have little; positions count what was cached, some dropped since
    meta = torch.empty((2, pages, hk, page), device=dev, dtype=torch.int32)
    u = torch.rand((pages, hk, page), generator=g, device=dev)
    meta[0] = (u ** 8 * 20).view(torch.int32)
    slot = torch.zeros(pages, dtype=torch.int64)
    for r, m in enumerate(need):
        slot[torch.as_tensor(table[r, :m].astype(np.int64))] = torch.arange(m) * page
    meta[1] = (slot.to(dev)[:, None, None] + torch.arange(page, device=dev)).to(torch.int32)
    rows = ints(np.stack([lens, lens]))  # cached tokens, next position
    off = np.concatenate([[0], np.cumsum(toks)])
    acc_off = np.concatenate([[0], np.cumsum(kept)])
    # trees whose first `kept` tokens are a path from the root, the rest hang anywhere on what came before
    parent, path = [], []
    for t, a in zip(toks, kept):
        p = rng.integers(-1, np.arange(t))
        p[:a] = np.arange(a) - 1
        parent.extend(p.tolist())
        path.extend(range(a))
    # queries, keys and values of the new tokens as one projection leaves them
    fused = normal(int(off[-1]), hq + 2 * hk, d)
    q, kn, vn = fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]
    q.mul_(1.5)
    state = {"case": case, "k": k, "v": v, "table": ints(table), "meta": meta, "rows": rows, "off": ints(off),
             "parent": ints(parent), "q": q, "k_new": kn, "v_new": vn, "acc_off": ints(acc_off), "acc": ints(path),
             "scale": d ** -0.5, "budget": ints([case["budget"]] * n), "longest": max(lens)}
    if case["op"] == "accept" and case["weigh"]:
        state["lse"] = _attend(state)[1]  # the step's attention left it
    return state


# ---------------------------------------------------------------------------------------------------------
# The plain forms: padded to the longest request, in 32 bits.

def _of_tokens(off, count):
    """Request and place in its request of each of ``count`` tokens in rows [off[r], off[r + 1])."""
    i = torch.arange(count, device=off.device)
    r = (i[:, None] >= off[None, 1:]).sum(1)
    return r, i - off[r]


def _cached(pool, table):
    """[request, head, slot, channel] of a pool in 32 bits."""
    x = pool[table.long().clamp(min=0)].transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1]).float()


def _padded(x, off, most):
    """[request, place, head, channel] in 32 bits of rows in request order."""
    i = off[:-1, None].long() + torch.arange(most, device=off.device)
    return x[i.clamp(max=x.shape[0] - 1)].float()


def _attend(s):
    case, off = s["case"], s["off"].long()
    b, t, hk, d = case["requests"], case["tree"], case["kv_heads"], case["dim"]
    grp, n = case["q_heads"] // hk, s["q"].shape[0]
    r, place = _of_tokens(off, n)
    q = _padded(s["q"], off, t).view(b, t, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * t, d)
    # tokens that a token descends from: powers of the tree's step matrix
    step = torch.zeros((b, t, t), device=q.device)
    up = s["parent"].long()
    step[r, place, up.clamp(min=0)] = (up >= 0).float()
    sees = torch.matrix_power(step + torch.eye(t, device=q.device), 64) > 0
    old = q @ _cached(s["k"], s["table"]).transpose(2, 3) * s["scale"]
    new = (q @ _padded(s["k_new"], off, t).permute(0, 2, 3, 1) * s["scale"]).view(b, hk, grp, t, t)
    held = torch.arange(old.shape[3], device=q.device) < s["rows"][0][:, None]
    old = old.masked_fill(~held[:, None, None], -math.inf)
    new = new.masked_fill(~sees[:, None, None], -math.inf).reshape(b, hk, grp * t, t)
    x = torch.cat([old, new], 3)
    top = x.amax(3, keepdim=True)
    x = (x - top).exp_()
    total = x.sum(3, keepdim=True)
    x = x / total
    out = x[..., :old.shape[3]] @ _cached(s["v"], s["table"])
    out = out + x[..., old.shape[3]:] @ _padded(s["v_new"], off, t).permute(0, 2, 1, 3)
    lse = (top + total.log()).view(b, hk * grp, t)
    out = out.view(b, hk * grp, t, d)
    return out[r, :, place].to(s["q"].dtype), lse[r, :, place]


def _accept(s):
    case, off = s["case"], s["acc_off"].long()
    b, hk, d, page = case["requests"], case["kv_heads"], case["dim"], case["page"]
    grp, n, a = case["q_heads"] // hk, s["acc"].shape[0], min(6, case["tree"])
    meta, rows = s["meta"].clone(), s["rows"].clone()
    weight = meta[0].view(torch.float32)
    r, i = _of_tokens(off, n)
    tok = s["off"].long()[r] + s["acc"].long()
    kept = off[1:] - off[:-1]
    slot = rows[0].long()[r] + i
    at = s["table"].long()[r, slot // page]
    s["k"][at, :, slot % page] = s["k_new"][tok]
    s["v"][at, :, slot % page] = s["v_new"][tok]
    weight[at, :, slot % page] = 0.0
    meta[1][at, :, slot % page] = (rows[1][r] + i).to(torch.int32)[:, None].expand(-1, hk)
    if case["weigh"]:
        q = _padded(s["q"][tok], off, a).view(b, a, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * a, d)
        lse = _padded(s["lse"][tok][:, :, None], off, a).view(b, a, hk, grp).permute(0, 2, 3, 1)
        x = (q @ _cached(s["k"], s["table"]).transpose(2, 3) * s["scale"]).view(b, hk, grp, a, -1)
        key, row = torch.arange(x.shape[4], device=x.device), torch.arange(a, device=x.device)
        sees = (key <= rows[0][:, None, None] + row[:, None]) & (row[:, None] < kept[:, None, None])
        x = torch.where(sees[:, None, None], (x - lse[..., None]).exp(), 0.0).sum((2, 3))
        x = x.view(b, hk, -1, page).transpose(1, 2).reshape(-1, hk, page)
        weight.index_add_(0, s["table"].long().clamp(min=0).flatten(), x)
    rows += kept.to(torch.int32)
    return s["k"], s["v"], weight, meta[1], rows[0], rows[1]


def _evict(s):
    case = s["case"]
    hk, d, page = case["kv_heads"], case["dim"], case["page"]
    meta, rows = s["meta"].clone(), s["rows"].clone()
    weight, pos = meta[0].view(torch.float32), meta[1]
    table = s["table"].long().clamp(min=0)
    held, budget = rows[0].long(), s["budget"].long()
    most = max(1, s["longest"] - case["budget"])  # tokens behind the budget
    w = weight[table].transpose(1, 2).reshape(table.shape[0], hk, -1)
    p = pos[table].transpose(1, 2).reshape(w.shape)
    slot = torch.arange(w.shape[2], device=w.device)
    live = slot < held[:, None, None]
    w = torch.where(p >= rows[1][:, None, None] - case["recent"], math.inf, w)
    w = torch.where(live, w, -math.inf)
    order = w.sort(dim=2, descending=True, stable=True)[1]
    keep = torch.empty_like(order).scatter_(2, order, slot.expand_as(order)) < budget[:, None, None]
    keep = (keep | (held <= budget)[:, None, None]) & live
    behind = live & (slot >= budget[:, None, None])
    holes = (~(live & ~behind & ~keep)).long().sort(dim=2, stable=True)[1]
    movers = torch.where(behind & keep, 0, torch.where(behind, 1, 2)).sort(dim=2, stable=True)[1]
    count = (behind & keep).sum(2, keepdim=True)
    over = (held - budget).clamp(min=0)
    i = torch.minimum(torch.arange(most, device=w.device), (over - 1).clamp(min=0)[:, None]).view(-1, 1, most)
    i = i.expand(-1, hk, -1)
    src = movers.gather(2, i)
    dst = torch.where(i < count, holes.gather(2, i), src)  # the others stay where they are
    req = torch.arange(table.shape[0], device=w.device)[:, None, None]
    head = torch.arange(hk, device=w.device)[:, None]
    there, here = (table[req, dst // page], head, dst % page), (table[req, src // page], head, src % page)
    for pool in (s["k"], s["v"], weight, pos):
        pool[there] = pool[here]
    rows[0] = torch.minimum(held, budget).to(torch.int32)
    return s["k"], s["v"], weight, pos, rows[0], rows[1]


def _logprobs(s):
    x, token, k = s["logits"].float(), s["token"].long()[:, None], s["case"]["top"]
    place = torch.arange(x.shape[1], device=x.device)
    top = x.amax(1, keepdim=True)
    e = (x - top).exp()
    total = e.sum(1, keepdim=True)
    lse = top + total.log()
    mine = x.gather(1, token)
    rank = (x > mine).sum(1) + ((x == mine) & (place < token)).sum(1)
    logprob, entropy = (mine - lse)[:, 0], (lse - (e / total * x).sum(1, keepdim=True))[:, 0]
    if not k:
        return logprob, entropy, rank.to(torch.int32)
    bits = (x + 0.0).view(torch.int32).long()  # whole numbers in the order of the values, lower places first
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    best = ((bits << 32) + (x.shape[1] - place)).topk(k, 1)[1]
    return logprob, entropy, rank.to(torch.int32), best.to(torch.int32), x.gather(1, best) - lse


# ---------------------------------------------------------------------------------------------------------
# The framework's operators.

_workers = {}


def _worker(case):
    """The handle that a worker's program keeps: one for a model's shape and a stream."""
    from paper_2405_06856_gb300 import aladdin as A
    shape = (case.get("kind", "bf16"), case["q_heads"], case["kv_heads"], case["dim"], case["page"]) \
        if case["op"] != "logprobs" else ("bf16", 1, 1, 64, 16)
    key = shape + (torch.cuda.current_stream().cuda_stream,)
    if key not in _workers:
        _workers[key] = A.Worker(*shape)
    return A, _workers[key]


def _run_own(s):
    case = s["case"]
    A, worker = _worker(case)
    if case["op"] == "logprobs":
        got = worker.logprobs(s["logits"], s["token"], case["top"])
        return got if case["top"] else got[:3]
    if case["op"] == "attend":
        kv = A.make_kv(s["k"], s["v"], s["table"], s["rows"][0])
        return worker.attend(kv, A.make_tokens(s["off"], s["q"], s["k_new"], s["v_new"], s["parent"]), s["scale"])
    meta, rows = s["meta"].clone(), s["rows"].clone()
    weight = meta[0].view(torch.float32)
    if case["op"] == "accept":
        kv = A.make_kv(s["k"], s["v"], s["table"], rows[0], weight, meta[1], rows[1])
        toks = A.make_tokens(s["off"], s["q"], s["k_new"], s["v_new"], s["parent"])
        worker.accept(kv, toks, s["scale"], s["lse"] if case["weigh"] else None, s["acc_off"], s["acc"])
    else:
        kv = A.make_kv(s["k"], s["v"], s["table"], rows[0], weight, meta[1], rows[1])
        worker.evict(kv, s["budget"], case["recent"])
    return s["k"], s["v"], weight, meta[1], rows[0], rows[1]


def run(state):
    """One pass. The accumulated weights, positions and lengths of ``accept`` and ``evict`` are copied first,
    so that a pass finds the state that the one before it found."""
    if own:
        return _run_own(state)
    return {"attend": _attend, "accept": _accept, "evict": _evict, "logprobs": _logprobs}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------
# The definitions, request by request, in 64 bits.

def _slots(s, r, count):
    i = torch.arange(count, device=s["k"].device)
    return s["table"][r].long()[i // s["case"]["page"]], i % s["case"]["page"]


def _exact_attend(s):
    case = s["case"]
    lens, off, parent = _lengths(case), s["off"].tolist(), s["parent"].tolist()
    grp = case["q_heads"] // case["kv_heads"]
    outs, sums = [], []
    for r, held in enumerate(lens):
        pg, sl = _slots(s, r, held)
        lo, hi = off[r], off[r + 1]
        keys = torch.cat([s["k"][pg, :, sl].double(), s["k_new"][lo:hi].double()]).transpose(0, 1)
        vals = torch.cat([s["v"][pg, :, sl].double(), s["v_new"][lo:hi].double()]).transpose(0, 1)
        sees = torch.zeros((hi - lo, held + hi - lo), dtype=torch.bool)
        sees[:, :held] = True
        for t in range(hi - lo):
            up = t
            while up >= 0:
                sees[t, held + up] = True
                up = parent[lo + up]
        q = s["q"][lo:hi].double().view(hi - lo, -1, grp, case["dim"]).permute(1, 2, 0, 3)
        x = torch.einsum("hgtd,hkd->hgtk", q, keys) * s["scale"]
        x = x.masked_fill(~sees.to(x.device), -math.inf)
        sums.append(torch.logsumexp(x, 3).flatten(0, 1).transpose(0, 1))
        outs.append(torch.einsum("hgtk,hkd->hgtd", torch.softmax(x, 3), vals).flatten(0, 1).transpose(0, 1))
    return torch.cat(outs), torch.cat(sums)


def _exact_accept(s):
    case = s["case"]
    lens, off, acc_off, acc = _lengths(case), s["off"].tolist(), s["acc_off"].tolist(), s["acc"].tolist()
    grp = case["q_heads"] // case["kv_heads"]
    k, v = s["k"].double(), s["v"].double()
    weight, pos, rows = s["meta"][0].view(torch.float32).double(), s["meta"][1].clone(), s["rows"].clone()
    for r, held in enumerate(lens):
        toks = [off[r] + a for a in acc[acc_off[r]:acc_off[r + 1]]]
        for i, t in enumerate(toks):
            pg, sl = int(s["table"][r, (held + i) // case["page"]]), (held + i) % case["page"]
            k[pg, :, sl], v[pg, :, sl] = s["k_new"][t].double(), s["v_new"][t].double()
            weight[pg, :, sl], pos[pg, :, sl] = 0.0, held + i
        if case["weigh"]:
            pg, sl = _slots(s, r, held + len(toks))
            for i, t in enumerate(toks):
                n = held + i + 1
                q = s["q"][t].double().view(-1, grp, case["dim"])
                x = torch.einsum("hgd,khd->hgk", q, k[pg[:n], :, sl[:n]]) * s["scale"]
                # the weights a full softmax over these tokens gives: what the row attended to
                weight[pg[:n], :, sl[:n]] += torch.softmax(x, 2).sum(1).transpose(0, 1)
        rows[:, r] += len(toks)
    return k, v, weight, pos, rows[0], rows[1]


def _exact_evict(s):
    case = s["case"]
    k, v = s["k"].double(), s["v"].double()
    weight, pos, rows = s["meta"][0].view(torch.float32).double(), s["meta"][1].clone(), s["rows"].clone()
    for r, held in enumerate(_lengths(case)):
        b = case["budget"]
        if held <= b:
            continue
        rows[0, r] = b
        pg, sl = _slots(s, r, held)
        for h in range(case["kv_heads"]):
            w = weight[pg, h, sl].cpu().numpy().copy()
            w[pos[pg, h, sl].cpu().numpy() >= held - case["recent"]] = np.inf
            stay = np.zeros(held, bool)
            stay[np.lexsort((np.arange(held), -w))[:b]] = True
            to = torch.as_tensor(np.flatnonzero(~stay[:b])).to(pg.device)
            of = torch.as_tensor(b + np.flatnonzero(stay[b:])).to(pg.device)
            for x in (k, v, weight, pos):
                x[pg[to], h, sl[to]] = x[pg[of], h, sl[of]]
    return k, v, weight, pos, rows[0], rows[1]


def _exact_logprobs(s):
    n, v = s["logits"].shape
    got = []
    for lo in range(0, n, 256):
        x, t = s["logits"][lo:lo + 256].double(), s["token"][lo:lo + 256].long()
        lp = torch.log_softmax(x, 1)
        order = (-x).sort(dim=1, stable=True)[1]
        rank = (order == t[:, None]).int().argmax(1).int()
        top = order[:, :s["case"]["top"]]
        got.append((lp.gather(1, t[:, None])[:, 0], -(lp.exp() * lp).sum(1), rank, top.int(), lp.gather(1, top)))
    got = tuple(torch.cat(x) for x in zip(*got))
    return got if s["case"]["top"] else got[:3]


def exact(case, seed):
    s = prepare(case, seed)
    return {"attend": _exact_attend, "accept": _exact_accept, "evict": _exact_evict,
            "logprobs": _exact_logprobs}[case["op"]](s)
