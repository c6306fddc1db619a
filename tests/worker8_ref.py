"""Rotary positions, appending and the cache of 8 bits in 64 bits on the CPU, token by token, from their definitions:
shared by the tests. No code of the library."""
import math

import numpy as np

import worker_ref as ref


def depths(off, parent):
    """Depth of every token in its request's tree (its index, for chains)."""
    out = np.zeros(off[-1], int)
    for r in range(len(off) - 1):
        for t in range(off[r + 1] - off[r]):
            out[off[r] + t] = t if parent is None else len(ref.ancestors(parent[off[r]:off[r + 1]], t)) - 1
    return out


def rotate(x, pos, freq, layout, scale=1.0):
    """x [tokens, heads, channels] at positions pos [tokens]."""
    out = x.copy()
    n = len(freq)
    for c in range(n):
        a, b = (2 * c, 2 * c + 1) if layout == "interleaved" else (c, c + n)
        t = np.array([math.fmod(float(p) * freq[c], 2 * math.pi) for p in pos])[:, None]
        with np.errstate(invalid="ignore"):
            out[..., a] = scale * (x[..., a] * np.cos(t) - x[..., b] * np.sin(t))
            out[..., b] = scale * (x[..., a] * np.sin(t) + x[..., b] * np.cos(t))
    return out


#: the numbers of e4m3 by code 0 .. 126 (127: NaN), and the others by their sign
VALUES = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def code(x):
    """The nearest code of every |x| <= 448, the even one of two; NaN: 127."""
    y = np.abs(np.where(np.isfinite(x), x, 0.0))
    hi = np.clip(np.searchsorted(VALUES, y), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = VALUES[hi] - y, y - VALUES[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(np.isfinite(x), c, 127)
    return (c + 128 * np.signbit(x)).astype(np.uint8)


def value(c):
    c = np.asarray(c)
    v = np.append(VALUES, np.nan)[c & 127]
    return np.where(c & 128, -v, v)


def scale_of(most):
    """The least power of two, 2^-126 at least, of which most is 448 times at most."""
    j = -126
    while most > 448.0 * 2.0 ** j:
        j += 1
    return 2.0 ** j


def kept(case, r, acc_off, acc):
    lo, hi = case["off"][r], case["off"][r + 1]
    return list(range(lo, hi)) if acc_off is None else [lo + a for a in acc[acc_off[r]:acc_off[r + 1]]]


def append8(case, rotated, acc_off=None, acc=None, skip=()):
    """Codes and scales (dict k, v, k_scale, v_scale) after the tokens of case entered them; rotated: the keys at their
    positions. case: codes k, v [pages, heads, page, dim], scales [pages, heads, page / block], len, off, table, page."""
    got = {x: case[x].copy() for x in ("k", "v", "k_scale", "v_scale")}
    page = case["page"]
    block = page // case["k_scale"].shape[2]
    for r, held in enumerate(case["len"]):
        toks = kept(case, r, acc_off, acc)
        if r in skip or not toks:
            continue
        for first in range(held // block * block, held + len(toks), block):
            p, at = case["table"][r][first // page], first % page
            if not 0 <= p < len(case["k"]):
                continue
            lo, hi = max(first, held), min(first + block, held + len(toks))
            for name, x in (("k", rotated), ("v", case["v_new"])):
                for h in range(x.shape[1]):
                    y = x[toks[lo - held:hi - held], h]
                    fin = np.abs(y[np.isfinite(y)])
                    s = scale_of(fin.max(initial=0.0))
                    held_s = got[name + "_scale"][p, h, at // block]
                    if lo > first:
                        if s > held_s:
                            c = got[name][p, h, at:at + lo - first]
                            got[name][p, h, at:at + lo - first] = code(value(c) * (held_s / s))
                        else:
                            s = held_s
                    got[name][p, h, at + lo - first:at + hi - first] = code(y / s)
                    got[name + "_scale"][p, h, at // block] = s
    return got


def dequantised(case, name):
    """[pages, heads, page, dim] of a cache of 8 bits."""
    with np.errstate(invalid="ignore"):
        s = np.repeat(case[name + "_scale"].astype(np.float64), case["page"] // case[name + "_scale"].shape[2], 2)
        return value(case[name]) * s[..., None]


def attend8(case):
    """As worker_ref.attend, over dequantised keys and values, a request and key head at a time."""
    k, v, q = dequantised(case, "k"), dequantised(case, "v"), case["q"]
    hk = k.shape[1]
    grp = q.shape[1] // hk
    out, lse = np.full(q.shape, np.nan), np.full(q.shape[:2], np.nan)
    for r, held in enumerate(case["len"]):
        lo, hi = case["off"][r], case["off"][r + 1]
        n = hi - lo
        if n <= 0:
            continue
        pg, sl = ref.slots(case, r, held)
        parent = np.arange(n) - 1 if case["parent"] is None else case["parent"][lo:hi]
        sees = np.zeros((n, n), bool)
        for t in range(n):
            sees[t, ref.ancestors(parent, t)] = True
        for h in range(hk):
            rows = q[lo:hi, h * grp:(h + 1) * grp].reshape(n * grp, -1)
            see = np.repeat(sees, grp, 0)
            with np.errstate(invalid="ignore", over="ignore"):
                old = rows @ k[pg, h, sl].T * case["scale"]
                new = np.where(see, rows @ case["k_new"][lo:hi, h].T * case["scale"], -math.inf)
                s = np.concatenate([old, new], 1)
                m = s.max(1)
                none = m == -math.inf
                e = np.exp(s - np.where(none, 0.0, m)[:, None])
                total = e.sum(1)
                o = e[:, :held] @ v[pg, h, sl]
                for t in range(n):  # (what a row does not see has no part, finite or not)
                    at = see[:, t]
                    o[at] += e[at, held + t, None] * case["v_new"][lo + t, h]
                o = np.where(none[:, None], 0.0, o / np.where(none, 1.0, total)[:, None])
                z = np.where(none, -math.inf, m + np.log(np.where(none, 1.0, total)))
            out[lo:hi, h * grp:(h + 1) * grp] = o.reshape(n, grp, -1)
            lse[lo:hi, h * grp:(h + 1) * grp] = z.reshape(n, grp)
    return out, lse
