"""Operators of a serving worker between its projections and its cache: rotary positions, the cache's growth, and
attention over a cache of 8 bits.

A layer's decode step rotates the queries and keys of its tokens to their positions, attends over what its requests
hold, and appends the tokens that stay; a prompt's queries are rotated, and its keys on their way into the cache:

* ``rotate``: rotary positions on queries and keys, half or interleaved pairs, the whole head or its first channels,
  plain frequencies or ones scaled for long contexts. A request's tokens are a piece of text or a tree of drafted
  tokens; a token's position is its request's next one and its depth.
* ``append``: keys, rotated on the way, and values enter a paged cache of 16 bits.
* ``append8``: the same into a cache of 8 bits (e4m3) with a scale for each block of tokens and head. The scale is a
  power of two, the least under which the block's largest value is at most 448; a block that has tokens keeps
  its scale where that is larger, and its old codes are rounded again where the new one is.
* ``attend8``: attention of a step's new tokens, of 16 bits, over the cached tokens of their requests, of 8 bits.
  Drafted tokens form trees; a token sees its request's cached tokens, its ancestors and itself.

Lengths follow the package's workload recipe: lognormal prompts, at most 8,192 tokens a request; longer contexts where a
case says so (131,072 tokens is the KV capacity of the recipe's larger workers). Head counts and page sizes are generic.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
HEADS = [(32, 8), (32, 32), (64, 8), (28, 4), (8, 1), (16, 2), (12, 12)]
#: a drawn case's floor in seconds at 7 TB/s and 2 PFLOP/s, and the scores and values of its padded plain form
MOST_SECONDS, MOST_SCORES, MOST_VALUES, MOST_BLOCKS = 7e-5, 1.2e9, 1.6e8, 30000


def _case(name, op, requests, ctx, most, heads, dim, page, kind, lens, **more):
    """``ctx``, ``most``: mean and largest cached length (or position); ``lens`` seeds the lengths, so that a case has
    the same ones on every input; ``new``: most new tokens a request; ``tree``: whether they form trees; ``rows``: the
    pool's order, pages of ``hnd`` (head, token, channel) or ``nhd`` (token, head, channel); ``block``: tokens that
    share a scale; ``turn``: rotated channels; ``keep``: whether only the first few of a request's tokens are appended."""
    case = dict(op=op, requests=requests, ctx=ctx, most=most, q_heads=heads[0], kv_heads=heads[1], dim=dim, page=page,
                kind=kind, lens=lens, new=1, tree=False, rows="hnd", block=16, turn=dim, layout="half", base=10000.0,
                scaling="none", factor=1.0, keep=False)
    case.update(more)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One request alone on a worker, one new token: the smallest step, where latency counts.
        _case("rotate_one", "rotate", 1, 640, 1000, (32, 8), 128, 64, "bf16", 3),
        # Drafted trees of up to 64 tokens: positions from the trees.
        _case("rotate_trees", "rotate", 24, 3000, 8192, (64, 8), 128, 32, "bf16", 5, new=64, tree=True),
        # Pieces of long prompts, far positions, scaled frequencies, two thirds of an odd head.
        _case("rotate_prompt", "rotate", 9, 60000, 131072, (28, 4), 96, 16, "f16", 6, new=2500, turn=64,
              layout="interleaved", scaling="parts", factor=16.0),
        # A decode step of a worker of the recipe: one token each of 128 requests.
        _case("append_step", "append", 128, 640, 8192, (32, 8), 128, 64, "bf16", 4),
        # Prompts enter a cache in token-major order, behind what their requests hold.
        _case("append_prompt", "append", 21, 640, 8192, (32, 8), 128, 64, "bf16", 7, new=1300, rows="nhd"),
        # The decode step with a cache of 8 bits: the new token may raise the scale of what its block holds.
        _case("append8_step", "append8", 128, 640, 8192, (32, 8), 128, 64, "bf16", 4),
        # Prompts into 8 bits, odd lengths, scales for 64 tokens, half of the head rotated.
        _case("append8_prompt", "append8", 21, 640, 8192, (28, 4), 96, 128, "f16", 8, new=2100, block=64, turn=48,
              layout="interleaved", scaling="linear", factor=4.0),
        # One request alone on a worker, one new token: the smallest step, where latency counts.
        _case("attend8_one", "attend8", 1, 640, 1000, (32, 8), 128, 64, "bf16", 3),
        # A decode step of a worker of the recipe: 128 requests of a few hundred tokens each.
        _case("attend8_128", "attend8", 128, 640, 8192, (32, 8), 128, 64, "bf16", 4),
        # Verification of drafted trees of up to 64 tokens: products count as much as bytes.
        _case("attend8_trees", "attend8", 24, 3000, 8192, (64, 8), 128, 32, "bf16", 5, new=64, tree=True, block=32),
        # Odd groups and an odd head dimension, short trees, a pool in token-major order.
        _case("attend8_odd", "attend8", 37, 1500, 5001, (28, 4), 96, 16, "f16", 6, new=5, tree=True, rows="nhd"),
        # Few long requests without shared heads: one long axis, split and joined.
        _case("attend8_long", "attend8", 2, 60000, 65536, (32, 32), 64, 64, "f16", 7, block=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _dear(case):
    w = work(case)
    if max(w["bytes"] / 7e12, w["flops"] / 2e15) > MOST_SECONDS:
        return True
    if case["op"] == "attend8":
        return case["requests"] * case["q_heads"] * case["new"] * max(_lengths(case)) > MOST_SCORES
    if case["op"] == "append8" and case["requests"] * case["new"] > MOST_BLOCKS * case["block"]:
        return True  # (its definition goes block by block)
    heads = case["q_heads"] + case["kv_heads"] if case["op"] == "rotate" else case["kv_heads"]
    return case["requests"] * (case["new"] + case["block"]) * heads * case["dim"] > MOST_VALUES


def draw(rng):
    op = rng.choice(["rotate", "append", "append8", "append8", "attend8", "attend8", "attend8"])
    while True:
        ctx = _log_int(rng, 40, 60000)
        dim = rng.choice([64, 64, 96, 128, 128, 128, 256])
        page = rng.choice([16, 32, 64, 128, 256])
        case = _case("", op, _log_int(rng, 1, 200), ctx, int(ctx * rng.uniform(1.0, 2.5)) + 1, rng.choice(HEADS), dim, page,
                     rng.choice(["bf16", "f16"]), rng.randrange(1 << 30), rows=rng.choice(["hnd", "hnd", "nhd"]),
                     block=rng.choice([b for b in (16, 16, 32, 64, 128, 256) if b <= page]),
                     turn=rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)]),
                     layout=rng.choice(["half", "interleaved"]), base=rng.choice([10000.0, 500000.0]),
                     scaling=rng.choice(["none", "none", "linear", "base", "parts"]))
        if case["scaling"] != "none":
            case["factor"] = float(rng.choice([2, 4, 8, 32]))
        if case["scaling"] == "base" and case["turn"] == 2:
            case["scaling"], case["factor"] = "none", 1.0
        if op == "attend8":
            case["new"] = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 64)])
            case["tree"] = True
        else:
            case["tree"] = op != "append" and rng.random() < 0.3
            case["new"] = rng.choice([1, _log_int(rng, 2, 64)]) if case["tree"] else rng.choice([1, _log_int(rng, 2, 4000)])
            case["keep"] = op != "rotate" and case["tree"]
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
    if n > 3:
        x[1] = 0
        x[2] = max(case["page"], x[2] // case["page"] * case["page"])
    return x.tolist()


def _counts(case):
    """New tokens of every request (up to ``new``), and how many of them are appended."""
    rng = np.random.default_rng(case["lens"] + 1)
    n, t = case["requests"], case["new"]
    toks = rng.integers((t + 1) // 2, t + 1, n)
    kept = np.minimum(toks, 1 + rng.integers(0, min(t, 6), n)) if case["keep"] else toks
    return toks.tolist(), kept.tolist()


def _width(case):
    """Entries of a row of the page table."""
    return -(-(max(_lengths(case)) + case["new"]) // case["page"])


def _blocks(case, lens, kept):
    """Blocks that new tokens enter."""
    return sum(-(-(c + t) // case["block"]) - c // case["block"] for c, t in zip(lens, kept) if t)


def work(case):
    lens, (toks, kept) = _lengths(case), _counts(case)
    hq, hk, d, n = case["q_heads"], case["kv_heads"], case["dim"], sum(toks)
    if case["op"] == "rotate":
        return {"bytes": 4 * d * (hq + hk) * n, "flops": 3 * case["turn"] * (hq + hk) * n}
    if case["op"] == "append":
        return {"bytes": 8 * d * hk * sum(kept), "flops": 3 * case["turn"] * hk * sum(kept)}
    if case["op"] == "append8":
        return {"bytes": hk * (6 * d * sum(kept) + 16 * _blocks(case, lens, kept)),
                "flops": (3 * case["turn"] + 4 * d) * hk * sum(kept)}
    return {"bytes": hk * (2 * d * sum(lens) + 8 * sum(-(-c // case["block"]) for c in lens) + 4 * d * n) + n * hq * (4 * d + 4),
            "flops": 4 * d * hq * sum(t * (c + 1) for t, c in zip(toks, lens))}


# ---------------------------------------------------------------------------------------------------------
# What a worker's program has in hand.

def _quantised(x, block):
    """Codes and scales of [page, head, token, channel]."""
    p, h, t, d = x.shape
    x = x.float().view(p, h, t // block, block, d)
    scale = _scale_of(x.abs().amax((3, 4)))
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn).view(p, h, t, d), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    kind = TYPES[case["kind"]]

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=dev, dtype=kind).mul_(scale)

    def ints(x):
        return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(dev)

    lens, (toks, kept) = _lengths(case), _counts(case)
    n, page = case["requests"], case["page"]
    hq, hk, d = case["q_heads"], case["kv_heads"], case["dim"]
    off = np.concatenate([[0], np.cumsum(toks)])
    parent = None
    if case["tree"]:  # the first `kept` tokens are a path from the root, the rest hang anywhere on what came before
        parent = []
        for t, a in zip(toks, kept):
            p = rng.integers(-1, np.arange(t))
            if case["keep"]:
                p[:a] = np.arange(a) - 1
            parent.extend(p.tolist())
    # queries, keys and values of the new tokens as one projection leaves them; a few channels of keys are large
    fused = normal(int(off[-1]), hq + 2 * hk, d)
    large = 1.0 + 5.0 * (torch.rand((hk, d), generator=g, device=dev) < 0.03).to(kind)
    fused[:, hq:hq + hk].mul_(large)
    q, kn, vn = fused[:, :hq], fused[:, hq:hq + hk], fused[:, hq + hk:]
    q.mul_(1.2)
    state = {"case": case, "off": ints(off), "parent": None if parent is None else ints(parent), "q": q, "k_new": kn,
             "v_new": vn, "rows": ints(np.stack([lens, lens])),  # cached tokens, next position
             "scale": d ** -0.5, "acc_off": None, "acc": None}
    if case["op"] == "rotate":
        return state
    if case["keep"]:
        state["acc_off"] = ints(np.concatenate([[0], np.cumsum(kept)]))
        state["acc"] = ints(np.concatenate([np.arange(a) for a in kept]))
    # every request has pages for its cached and its new tokens, in any order; entries behind are unused
    need = [-(-(c + t) // page) for c, t in zip(lens, toks)]
    pages = sum(need) + 3
    order = rng.permutation(pages)
    table = np.full((n, _width(case)), -1, np.int32)
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = order[at:at + m]
        at += m
    state["table"] = ints(table)

    def pool(large):
        """Values of the pool's shape; blocks differ in size."""
        x = normal(pages, hk, page, d).mul_(large)
        if case["op"] == "append":
            return (x,)
        b = case["block"]
        size = (0.5 + torch.rand((pages, hk, page // b), generator=g, device=dev)).to(kind)
        x.view(pages, hk, page // b, b, d).mul_(size[..., None, None])
        return _quantised(x, b)

    for name, more in (("k", large[:, None]), ("v", 1.0)):
        x, *scale = pool(more)
        if case["rows"] == "nhd":
            x = x.transpose(1, 2).contiguous().transpose(1, 2)
        state[name] = x
        if scale:
            state[name + "_scale"] = scale[0]
    return state


# ---------------------------------------------------------------------------------------------------------
# The plain forms: padded to the longest request, in 32 bits.

def _scale_of(most):
    """The least power of two, 2^-126 at least, of which ``most`` is 448 times at most."""
    m, e = torch.frexp(most)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    e = torch.where(most > 0, e, -126).clamp(min=-126)
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)  # (ldexp is not exact on every device)


def _of_tokens(off, count):
    """Request and place in its request of each of ``count`` tokens in rows [off[r], off[r + 1])."""
    i = torch.arange(count, device=off.device)
    r = torch.searchsorted(off[1:].contiguous(), i, right=True)
    return r, i - off[r]


def _padded(x, off, most):
    """[request, place, head, channel] in 32 bits of rows in request order."""
    i = off[:-1, None].long() + torch.arange(most, device=off.device)
    return x[i.clamp(max=x.shape[0] - 1)].float()


def _sees(s, r, place):
    """[request, token, token]: what a token descends from, and itself: powers of the tree's step matrix."""
    b, t = s["case"]["requests"], s["case"]["new"]
    step = torch.zeros((b, t, t), device=r.device)
    up = s["parent"].long() if s["parent"] is not None else place - 1
    step[r, place, up.clamp(min=0)] = (up >= 0).float()
    return torch.matrix_power(step + torch.eye(t, device=r.device), 64) > 0


def _frequencies(case, device):
    """Radians a position of every pair, in 64 bits, and the factor of rotated channels."""
    i = torch.arange(case["turn"] // 2, device=device, dtype=torch.float64)
    base, factor, turn = case["base"], case["factor"], case["turn"]
    if case["scaling"] == "base":
        base = base * factor ** (turn / (turn - 2))
    freq = base ** (-2.0 * i / turn)
    if case["scaling"] == "linear":
        return freq / factor, 1.0
    if case["scaling"] == "parts":
        part = ((8192 * freq / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        return freq * (part + (1.0 - part) / factor), 0.1 * math.log(factor) + 1.0
    return freq, 1.0


def _rotated(case, x, pos):
    """[token, head, channel] in 32 bits, rotated to the positions; angles in 64 bits."""
    freq, factor = _frequencies(case, x.device)
    angle = pos.double()[:, None, None] * freq
    cos, sin = (factor * angle.cos()).float(), (factor * angle.sin()).float()
    x, turn = x.float(), case["turn"]
    a, b = (slice(0, turn, 2), slice(1, turn, 2)) if case["layout"] == "interleaved" else \
        (slice(0, turn // 2), slice(turn // 2, turn))
    out = x.clone()
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., a] * sin + x[..., b] * cos
    return out


def _rotate(s):
    case, off = s["case"], s["off"].long()
    r, depth = _of_tokens(off, s["q"].shape[0])
    if s["parent"] is not None:
        depth = _sees(s, r, depth)[r, depth].sum(1) - 1
    pos = s["rows"][1].long()[r] + depth
    return _rotated(case, s["q"], pos).to(s["q"].dtype), _rotated(case, s["k_new"], pos).to(s["q"].dtype)


def _kept(s):
    """Of the appended tokens: request, place behind the cached ones, index among the new ones."""
    off = s["off"].long()
    if s["acc"] is None:
        r, i = _of_tokens(off, s["q"].shape[0])
        return r, i, torch.arange(r.shape[0], device=r.device)
    r, i = _of_tokens(s["acc_off"].long(), s["acc"].shape[0])
    return r, i, off[r] + s["acc"].long()


def _append(s):
    case, page, rows = s["case"], s["case"]["page"], s["rows"].clone()
    r, i, tok = _kept(s)
    slot = rows[0].long()[r] + i
    at = s["table"].long()[r, slot // page]
    s["k"][at, :, slot % page] = _rotated(case, s["k_new"][tok], rows[1].long()[r] + i).to(s["k"].dtype)
    s["v"][at, :, slot % page] = s["v_new"][tok]
    off = s["off"] if s["acc_off"] is None else s["acc_off"]
    rows += off[1:] - off[:-1]
    return s["k"], s["v"], rows[0], rows[1]


def _append8(s):
    case, page, b, rows = s["case"], s["case"]["page"], s["case"]["block"], s["rows"].clone()
    r, i, tok = _kept(s)
    held = rows[0].long()
    n, hk, d = case["requests"], case["kv_heads"], case["dim"]
    off = (s["off"] if s["acc_off"] is None else s["acc_off"]).long()
    count = off[1:] - off[:-1]
    most = min(case["new"], 6) if case["keep"] else case["new"]
    nb = (b - 1 + most + b - 1) // b  # blocks that a request's new tokens enter, at most
    slot = (held // b * b)[:, None] + torch.arange(nb * b, device=held.device)
    old = slot < held[:, None]
    live = slot < (held + count)[:, None]
    pages = s["table"].long().gather(1, (slot // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    new = {"k": _rotated(case, s["k_new"][tok], rows[1].long()[r] + i), "v": s["v_new"][tok].float()}
    first = slot[:, ::b]  # of every block
    enters = (first < (held + count)[:, None]) & (count > 0)[:, None]
    has = first < held[:, None]
    where = live & (count > 0)[:, None]
    for name in ("k", "v"):
        codes, scales = s[name].view(torch.uint8), s[name + "_scale"]
        x = torch.zeros((n, nb * b, hk, d), device=held.device)
        x[r, held[r] % b + i] = new[name]
        most_of = x.abs().view(n, nb, b, hk, d).amax((2, 4))
        block_at = (pages[:, ::b, None], torch.arange(hk, device=held.device), (first % page // b)[:, :, None])
        before = scales[block_at]
        scale = _scale_of(most_of)
        scale = torch.where(has[..., None], torch.maximum(scale, before), scale)
        x = x / scale.repeat_interleave(b, 1)[..., None]
        again = codes[pages, :, slot % page].view(torch.float8_e4m3fn).float() * (before / scale).repeat_interleave(b, 1)[..., None]
        x = torch.where(old[..., None, None], again, x).to(torch.float8_e4m3fn).view(torch.uint8)
        rw, sw = where.nonzero(as_tuple=True)
        codes[pages[rw, sw], :, slot[rw, sw] % page] = x[rw, sw]
        rb, sb = enters.nonzero(as_tuple=True)
        scales[pages[:, ::b][rb, sb], :, (first % page // b)[rb, sb]] = scale[rb, sb]
    rows += count.to(torch.int32)
    return s["k"], s["v"], s["k_scale"], s["v_scale"], rows[0], rows[1]


def _cached(s, name):
    """[request, head, slot, channel] of a pool of 8 bits in 32 bits."""
    at = s["table"].long().clamp(min=0)
    x = s[name].view(torch.uint8)[at].view(torch.float8_e4m3fn).float()
    x = x * s[name + "_scale"][at].repeat_interleave(s["case"]["block"], 3)[..., None]
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _attend8(s):
    case, off = s["case"], s["off"].long()
    b, t, hk, d = case["requests"], case["new"], case["kv_heads"], case["dim"]
    grp, n = case["q_heads"] // hk, s["q"].shape[0]
    r, place = _of_tokens(off, n)
    q = _padded(s["q"], off, t).view(b, t, hk, grp, d).permute(0, 2, 3, 1, 4).reshape(b, hk, grp * t, d)
    old = q @ _cached(s, "k").transpose(2, 3) * s["scale"]
    new = (q @ _padded(s["k_new"], off, t).permute(0, 2, 3, 1) * s["scale"]).view(b, hk, grp, t, t)
    held = torch.arange(old.shape[3], device=q.device) < s["rows"][0][:, None]
    old = old.masked_fill(~held[:, None, None], -math.inf)
    new = new.masked_fill(~_sees(s, r, place)[:, None, None], -math.inf).reshape(b, hk, grp * t, t)
    x = torch.cat([old, new], 3)
    top = x.amax(3, keepdim=True)
    x = (x - top).exp_()
    total = x.sum(3, keepdim=True)
    x = x / total
    out = x[..., :old.shape[3]] @ _cached(s, "v")
    out = out + x[..., old.shape[3]:] @ _padded(s["v_new"], off, t).permute(0, 2, 1, 3)
    lse = (top + total.log()).view(b, hk * grp, t)
    out = out.view(b, hk * grp, t, d)
    return out[r, :, place].to(s["q"].dtype), lse[r, :, place]


# ---------------------------------------------------------------------------------------------------------
# The framework's operators.

_handles = {}


def _worker(case):
    """The handles that a worker's program keeps: one for a model's shape and a stream, and its rotation."""
    from paper_2405_06856_gb300 import aladdin as A
    shape = (case["kind"], case["q_heads"], case["kv_heads"], case["dim"], case["page"])
    turn = (case["turn"], case["base"], case["layout"], case["scaling"], case["factor"])
    key = shape + turn + (torch.cuda.current_stream().cuda_stream,)
    if key not in _handles:
        scaling = None if case["scaling"] == "none" else case["scaling"]
        _handles[key] = A.Worker(*shape), A.make_rope(case["turn"], case["base"], case["layout"], scaling, case["factor"], 8192)
    return (A,) + _handles[key]


def _run_own(s):
    case = s["case"]
    A, worker, rope = _worker(case)
    tok = A.make_tokens(s["off"], s["q"], s["k_new"], s["v_new"], s["parent"])
    if case["op"] == "rotate":
        return worker.rotate(rope, tok, s["rows"][1])
    if case["op"] == "attend8":
        kv = A.make_kv8(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], s["rows"][0])
        return worker.attend(kv, tok, s["scale"])
    rows = s["rows"].clone()
    if case["op"] == "append":
        worker.append(A.make_kv(s["k"], s["v"], s["table"], rows[0], next_pos=rows[1]), tok, rope, s["acc_off"], s["acc"])
        return s["k"], s["v"], rows[0], rows[1]
    kv = A.make_kv8(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"], rows[0], rows[1])
    worker.append(kv, tok, rope, s["acc_off"], s["acc"])
    return s["k"], s["v"], s["k_scale"], s["v_scale"], rows[0], rows[1]


def run(state):
    """One pass. The lengths and next positions of ``append`` and ``append8`` are copied first, so that a pass finds the
    state that the one before it found. The cache of 8 bits comes back as its e4m3 values and their blocks' scales."""
    if own:
        return _run_own(state)
    return {"rotate": _rotate, "append": _append, "append8": _append8, "attend8": _attend8}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------
# The definitions, request by request, in 64 bits.

def _exact_rotation(case, x, positions):
    """[token, head, channel] turned pair by pair."""
    x = x.double()
    out, turn, factor = x.clone(), case["turn"], 1.0
    pos = torch.tensor(positions, dtype=torch.float64, device=x.device)[:, None]
    for i in range(turn // 2):
        freq = math.exp(-2.0 * i / turn * math.log(case["base"]))
        if case["scaling"] == "linear":
            freq /= case["factor"]
        elif case["scaling"] == "base":
            freq = math.exp(-2.0 * i / turn * (math.log(case["base"]) + turn / (turn - 2) * math.log(case["factor"])))
        elif case["scaling"] == "parts":
            turns = 8192 * freq / (2 * math.pi)  # within the context that the model was made for
            whole = 0.0 if turns < 1.0 else 1.0 if turns > 32.0 else (turns - 1.0) / 31.0
            freq = freq * whole + freq / case["factor"] * (1.0 - whole)
            factor = 1.0 + 0.1 * math.log(case["factor"])
        a, b = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + turn // 2)
        z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.full_like(pos, factor), pos * freq)
        out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_rotate(s):
    off, start = s["off"].tolist(), s["rows"][1].tolist()
    parent = None if s["parent"] is None else s["parent"].tolist()
    pos = []
    for r, first in enumerate(start):
        for t in range(off[r + 1] - off[r]):
            depth = t
            if parent is not None:
                depth, up = 0, parent[off[r] + t]
                while up >= 0:
                    depth, up = depth + 1, parent[off[r] + up]
            pos.append(first + depth)
    return _exact_rotation(s["case"], s["q"], pos), _exact_rotation(s["case"], s["k_new"], pos)


def _tokens_kept(s, r):
    off = s["off"].tolist()
    if s["acc"] is None:
        return list(range(off[r], off[r + 1]))
    lo, hi = s["acc_off"].tolist()[r:r + 2]
    return [off[r] + a for a in s["acc"].tolist()[lo:hi]]


def _exact_append(s):
    case, page = s["case"], s["case"]["page"]
    k, v, rows = s["k"].double(), s["v"].double(), s["rows"].clone()
    for r, held in enumerate(_lengths(case)):
        toks = _tokens_kept(s, r)
        if toks:
            slot = torch.arange(held, held + len(toks), device=k.device)
            at = s["table"][r].long()[slot // page]
            k[at, :, slot % page] = _exact_rotation(case, s["k_new"][toks], list(range(held, held + len(toks))))
            v[at, :, slot % page] = s["v_new"][toks].double()
        rows[:, r] += len(toks)
    return k, v, rows[0], rows[1]


def _nearest8(x):
    """The nearest numbers of e4m3, the even one of two; |x| at most 448."""
    e = torch.frexp(x)[1].clamp(min=-5)  # a step of 2^-9 below 2^-6, else 8 steps a power of two
    step = torch.exp2(e.double() - 4)
    return torch.round(x / step) * step


def _exact_append8(s):
    case, page, b = s["case"], s["case"]["page"], s["case"]["block"]
    k, v = s["k"].view(torch.uint8).view(torch.float8_e4m3fn).double(), s["v"].view(torch.uint8).view(torch.float8_e4m3fn).double()
    ks, vs, rows = s["k_scale"].double(), s["v_scale"].double(), s["rows"].clone()
    table = s["table"].tolist()
    for r, held in enumerate(_lengths(case)):
        toks = _tokens_kept(s, r)
        if toks:
            new = (_exact_rotation(case, s["k_new"][toks], list(range(held, held + len(toks)))), s["v_new"][toks].double())
        for first in range(held // b * b, held + len(toks), b) if toks else ():
            lo, hi = max(first, held), min(first + b, held + len(toks))
            p, at, bl = table[r][first // page], first % page, first % page // b
            for x, codes, scales in ((new[0], k, ks), (new[1], v, vs)):
                y = x[lo - held:hi - held].transpose(0, 1)  # [head, token, channel]
                most = y.abs().amax((1, 2))
                m, j = torch.frexp(most / 448.0)
                j = torch.where(m == 0.5, j - 1, j).clamp(min=-126)
                scale = torch.where(most > 0, torch.exp2(j.double()), 2.0 ** -126)
                if lo > first:
                    scale = torch.maximum(scale, scales[p, :, bl])
                    old = codes[p, :, at:at + lo - first] * scales[p, :, bl, None, None]
                    codes[p, :, at:at + lo - first] = _nearest8(old / scale[:, None, None])
                codes[p, :, at + lo - first:at + hi - first] = _nearest8(y / scale[:, None, None])
                scales[p, :, bl] = scale
        rows[:, r] += len(toks)
    return k, v, ks, vs, rows[0], rows[1]


def _exact_attend8(s):
    case = s["case"]
    lens, off, page, b = _lengths(case), s["off"].tolist(), case["page"], case["block"]
    parent = list(range(-1, off[-1] - 1)) if s["parent"] is None else s["parent"].tolist()
    grp = case["q_heads"] // case["kv_heads"]
    outs, sums = [], []
    for r, held in enumerate(lens):
        i = torch.arange(held, device=s["k"].device)
        pg, sl = s["table"][r].long()[i // page], i % page
        lo, hi = off[r], off[r + 1]
        both = []
        for name in ("k", "v"):
            x = s[name].view(torch.uint8)[pg, :, sl].view(torch.float8_e4m3fn).double()
            x = x * s[name + "_scale"][pg, :, sl // b].double()[..., None]
            both.append(torch.cat([x, s[name + "_new"][lo:hi].double()]).transpose(0, 1))
        sees = torch.zeros((hi - lo, held + hi - lo), dtype=torch.bool)
        sees[:, :held] = True
        for t in range(hi - lo):
            up = t
            while up >= 0:
                sees[t, held + up] = True
                up = parent[lo + up] if s["parent"] is not None else up - 1
        q = s["q"][lo:hi].double().view(hi - lo, -1, grp, case["dim"]).permute(1, 2, 0, 3)
        x = torch.einsum("hgtd,hkd->hgtk", q, both[0]) * s["scale"]
        x = x.masked_fill(~sees.to(x.device), -math.inf)
        sums.append(torch.logsumexp(x, 3).flatten(0, 1).transpose(0, 1))
        outs.append(torch.einsum("hgtk,hkd->hgtd", torch.softmax(x, 3), both[1]).flatten(0, 1).transpose(0, 1))
    return torch.cat(outs), torch.cat(sums)


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "append": _exact_append, "append8": _exact_append8,
            "attend8": _exact_attend8}[case["op"]](s)
