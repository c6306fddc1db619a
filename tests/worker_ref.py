"""The worker step's operators in 64 bits on the CPU, token by token, from their definitions: shared by the
tests. No code of the library."""
import math

import numpy as np


def ancestors(parent, t):
    seen = []
    while t >= 0:
        seen.append(t)
        t = int(parent[t])
    return seen


def slots(case, r, count):
    i = np.arange(count)
    return case["table"][r][i // case["page"]], i % case["page"]


def attend(case):
    """out [tokens, q_heads, dim], lse [tokens, q_heads] of float64 arrays k, v [pages, heads, page, dim], q,
    k_new, v_new [tokens, heads, dim], lists table, len, off, parent (None: chains)."""
    q, hk = case["q"], case["k"].shape[1]
    grp = q.shape[1] // hk
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
    for r, held in enumerate(case["len"]):
        lo, hi = case["off"][r], case["off"][r + 1]
        pg, sl = slots(case, r, held)
        parent = np.arange(hi - lo) - 1 if case["parent"] is None else case["parent"][lo:hi]
        for t in range(hi - lo):
            new = lo + np.array(sorted(ancestors(parent, t)))
            for h in range(hk):
                keys = np.concatenate([case["k"][pg, h, sl], case["k_new"][new, h]])
                vals = np.concatenate([case["v"][pg, h, sl], case["v_new"][new, h]])
                for g in range(grp):
                    with np.errstate(invalid="ignore"):
                        s = keys @ q[lo + t, h * grp + g] * case["scale"]
                        m = s.max()
                        if m == -math.inf:
                            out[lo + t, h * grp + g], lse[lo + t, h * grp + g] = 0.0, -math.inf
                            continue
                        e = np.exp(s - m)
                        out[lo + t, h * grp + g] = e @ vals / e.sum()
                        lse[lo + t, h * grp + g] = m + np.log(e.sum())
    return out, lse


def accept(case, acc_off, acc, lse=None):
    """k, v, weight, pos, len, next after the tokens were kept, and by how much weights grew."""
    k, v = case["k"].copy(), case["v"].copy()
    weight, pos = case["weight"].copy(), case["pos"].copy()
    length, nxt = list(case["len"]), list(case["next"])
    hk, page = k.shape[1], case["page"]
    grp = case["q"].shape[1] // hk
    for r, held in enumerate(case["len"]):
        toks = [case["off"][r] + a for a in acc[acc_off[r]:acc_off[r + 1]]]
        for i, t in enumerate(toks):
            p, s = case["table"][r][(held + i) // page], (held + i) % page
            k[p, :, s], v[p, :, s] = case["k_new"][t], case["v_new"][t]
            weight[p, :, s], pos[p, :, s] = 0.0, nxt[r] + i
        if lse is not None:
            pg, sl = slots(case, r, held + len(toks))
            for i, t in enumerate(toks):
                n = held + i + 1
                for h in range(hk):
                    for g in range(grp):
                        s = k[pg[:n], h, sl[:n]] @ case["q"][t, h * grp + g] * case["scale"]
                        weight[pg[:n], h, sl[:n]] += np.exp(s - lse[t, h * grp + g])
        length[r] += len(toks)
        nxt[r] += len(toks)
    return k, v, weight, pos, length, nxt


def evict(case, budget, recent):
    k, v = case["k"].copy(), case["v"].copy()
    weight, pos, length = case["weight"].copy(), case["pos"].copy(), list(case["len"])
    for r, held in enumerate(case["len"]):
        b = budget[r]
        if held <= b:
            continue
        pg, sl = slots(case, r, held)
        for h in range(k.shape[1]):
            order = []
            for s in range(held):
                w = float(weight[pg[s], h, sl[s]])
                if pos[pg[s], h, sl[s]] >= case["next"][r] - recent:
                    w = math.inf
                order.append((1 if math.isnan(w) else 0, 0.0 if math.isnan(w) else -w, s))
            stay = {s for _, _, s in sorted(order)[:b]}
            holes = [s for s in range(b) if s not in stay]
            movers = [s for s in range(b, held) if s in stay]
            assert len(holes) == len(movers)
            for d, s in zip(holes, movers):
                for x in (k, v, weight, pos):
                    x[pg[d], h, sl[d]] = x[pg[s], h, sl[s]]
        length[r] = b
    return k, v, weight, pos, length


def logprobs(x, token, top):
    """logprob, entropy, rank, top_id, top_logprob of float64 logits x [rows, vocab]."""
    n, vocab = x.shape
    lp, ent = np.full(n, np.nan), np.full(n, np.nan)
    rank = np.full(n, -2)
    ids, tlp = np.zeros((n, top), int), np.full((n, top), np.nan)
    for r in range(n):
        row = x[r]
        order = sorted(range(vocab), key=lambda i: (math.isnan(row[i]), 0.0 if math.isnan(row[i]) else -row[i], i))
        ids[r] = order[:top]
        if 0 <= token[r] < vocab:
            rank[r] = order.index(token[r])
        if np.isnan(row).any() or (row == math.inf).any():
            continue
        m = row.max()
        if m == -math.inf:
            ent[r], tlp[r] = 0.0, -math.inf
            if 0 <= token[r] < vocab:
                lp[r] = -math.inf
            continue
        e = np.exp(row - m)
        lse = m + math.log(e.sum())
        p = e / e.sum()
        ent[r] = -sum(a * math.log(a) for a in p[p > 0])
        tlp[r] = row[ids[r]] - lse
        if 0 <= token[r] < vocab:
            lp[r] = row[token[r]] - lse
    return lp, ent, rank, ids, tlp
