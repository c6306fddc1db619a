"""Rotary positions (aladdin_worker_rotate) and appending to a cache of 16 bits (aladdin_worker_append) against their
definitions in 64 bits.

Tolerances, fixed before the first run: the result is rounded once, u |x| (u: 2^-8 for bf16, 2^-11 for f16; half a step
of 2^-24 below 2^-14 in f16); cosine and sine are off by 2^-23, products and the factor round in 32 bits: 2^-21 of the
pair's size. What is copied, lengths, positions and weights are equal."""
import math

import numpy as np
import pytest

import worker8_ref as ref8
from test_gpu_worker import A, Dev, f64, make, rounded  # noqa: F401

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def pair_size(x, n, layout):
    """Size of the pair that every channel belongs to; 0 where none."""
    out = np.zeros_like(x)
    for c in range(n):
        a, b = (2 * c, 2 * c + 1) if layout == "interleaved" else (c, c + n)
        out[..., a] = out[..., b] = np.hypot(x[..., a], x[..., b])
    return out


def check_rotated(got, x, pos, freq, layout, scale, kind):
    want = ref8.rotate(x, pos, freq, layout, scale)
    size = pair_size(x, len(freq), layout)
    fin = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fin)
    tol = U[kind] * np.abs(want) + 2.0 ** -21 * scale * size + (2.0 ** -25 if kind == "f16" else 0.0)
    d = np.abs(np.where(fin, got, 0.0) - np.where(fin, want, 0.0))
    tol = np.where(fin & (size > 0), tol, 0.0)  # channels that are not rotated stay as they are
    assert np.all(d[fin] <= tol[fin]), (d - tol)[fin].max()


def rope_of(A, freq, layout, scale=1.0):  # noqa: F811
    return A.make_rope(2 * len(freq), layout=layout, freq=freq, scale=scale)


SHAPES = [("bf16", 8, 2, 128, 128), ("f16", 8, 2, 128, 128), ("bf16", 4, 4, 64, 64), ("f16", 7, 1, 96, 64),
          ("bf16", 4, 2, 256, 256), ("f16", 6, 3, 128, 2), ("bf16", 5, 5, 96, 96), ("f16", 12, 4, 256, 74),
          ("bf16", 64, 8, 64, 34), ("f16", 40, 8, 128, 112), ("bf16", 3, 1, 96, 90)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,q_heads,kv_heads,dim,turn", SHAPES)
@pytest.mark.parametrize("where", ["fresh", "place", "wide"])
def test_rotate(A, kind, q_heads, kv_heads, dim, turn, layout, where):  # noqa: F811
    """Trees, chains of one and of many tokens, no tokens; into new tensors, in place, into another one's columns."""
    import torch
    toks = [1, 0, 5, 64, 2]
    case = make(kind, q_heads, kv_heads, dim, 16, [3, 0, 40, 100000 % 977, 16], toks, seed=turn)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    scale = 1.25 if turn % 3 == 0 else 1.0
    rope = rope_of(A, freq, layout, scale)
    start = [7, 0, 131071, 5000, 1 << 20]
    nxt = torch.tensor(start, dtype=torch.int32, device="cuda")
    pos = np.repeat(start, toks) + ref8.depths(case["off"], case["parent"])
    outs = {}
    if where == "place":
        outs = dict(q_out=d.q, k_out=d.k_new)
    if where == "wide":
        w = torch.full((72, q_heads + kv_heads + 1, dim), 7.0, dtype=d.kind, device="cuda")
        outs = dict(q_out=w[:, :q_heads], k_out=w[:, q_heads:q_heads + kv_heads])
    q, k = d.worker.rotate(rope, d.tok, nxt, **outs)
    assert d.worker.status() == 0
    check_rotated(f64(q), case["q"], pos, freq, layout, scale, kind)
    check_rotated(f64(k), case["k_new"], pos, freq, layout, scale, kind)
    if where == "wide":
        assert (w[:, -1] == 7.0).all()
    assert np.array_equal(f64(d.v_new), case["v_new"])


@pytest.mark.parametrize("n", [1, 3, 33, 700, 5000])
def test_rotate_chains(A, n):  # noqa: F811
    """Pieces of prompts of any length, by next positions and by given ones, queries alone and keys alone."""
    import torch
    toks = [n, 0, 1, max(1, n // 3)]
    case = make("bf16", 4, 2, 128, 16, [0] * 4, toks, trees=False)
    d = Dev(A, case)
    freq, _ = A.aladdin_rope_frequencies(128, 500000.0, A.ROPE_PARTS, 8.0, 8192.0)
    rope = A.make_rope(128, 500000.0, scaling="parts", factor=8.0, original=8192)
    start = np.array([100, 5, 2 ** 31 - 2, 0])
    pos = (np.repeat(start, toks) + ref8.depths(case["off"], None)).astype(np.int64)
    q, k = d.worker.rotate(rope, d.tok, torch.from_numpy(start.astype(np.int32)).cuda(), k_out=False)
    assert k is None
    check_rotated(f64(q), case["q"], pos, freq, "half", rope.scale, "bf16")
    given = np.random.default_rng(0).integers(-(2 ** 31), 2 ** 31, len(pos))
    q, k = d.worker.rotate(rope, d.tok, None, torch.from_numpy(given.astype(np.int32)).cuda(), q_out=False)
    assert q is None
    check_rotated(f64(k), case["k_new"], given, freq, "half", rope.scale, "bf16")
    q, k = d.worker.rotate(rope, d.tok)
    check_rotated(f64(q), case["q"], ref8.depths(case["off"], None), freq, "half", rope.scale, "bf16")


def test_rotate_turns_back(A):  # noqa: F811
    """Scores depend on the distance of positions alone, and the opposite frequencies take a rotation back."""
    import torch
    case = make("f16", 4, 2, 64, 16, [0], [40], trees=False)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(32) / 32)
    rope, back = rope_of(A, freq, "half"), rope_of(A, -freq, "half")
    at = lambda p: torch.full((40,), p, dtype=torch.int32, device="cuda")
    q0, k0 = (f64(x) for x in d.worker.rotate(rope, d.tok, pos=at(1000)))
    q1, k1 = (f64(x) for x in d.worker.rotate(rope, d.tok, pos=at(1000000)))
    s0, s1, s = ((q[:, :2] * k).sum(2) for q, k in ((q0, k0), (q1, k1), (case["q"], case["k_new"])))
    size = np.sqrt((case["q"][:, :2] ** 2).sum(2) * (case["k_new"] ** 2).sum(2))
    assert np.all(np.abs(s0 - s) <= 2.1 * 2.0 ** -11 * size) and np.all(np.abs(s1 - s) <= 2.1 * 2.0 ** -11 * size)
    d.worker.rotate(rope, d.tok, pos=at(777), q_out=d.q, k_out=d.k_new)
    d.worker.rotate(back, d.tok, pos=at(777), q_out=d.q, k_out=d.k_new)
    assert np.all(np.abs(f64(d.k_new) - case["k_new"]) <= 2.0 ** -10 * pair_size(case["k_new"], 32, "half"))


def test_rotate_what_is_not_finite_stays_in_its_pair(A):  # noqa: F811
    import torch
    case = make("bf16", 4, 2, 64, 16, [0], [3], trees=False)
    d = Dev(A, case)
    d.q[1, 2, 5] = math.inf
    d.q[1, 2, 60] = math.nan
    q, _ = d.worker.rotate(rope_of(A, [1.0] * 16, "half"), d.tok)  # channels 0 .. 31
    bad = np.argwhere(~np.isfinite(f64(q)))
    assert bad.tolist() == [[1, 2, 5], [1, 2, 21], [1, 2, 60]]


def test_rotate_refuses(A):  # noqa: F811
    import torch
    case = make("bf16", 4, 2, 64, 16, [0, 0, 0], [2, 3, 65])
    d = Dev(A, case)
    rope = rope_of(A, [1.0] * 32, "half")
    fill = lambda: dict(q_out=torch.full_like(d.q, 9.0), k_out=torch.full_like(d.k_new, 9.0))
    # a tree of 65 tokens takes no part; a parent that is no earlier token counts as none
    out = fill()
    d.parent[3] = 2
    q, k = d.worker.rotate(rope, d.tok, **out)
    assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
    assert (q[5:] == 9.0).all() and (k[5:] == 9.0).all()
    parent = case["parent"].copy()
    parent[3] = -1
    depth = ref8.depths(case["off"][:3], parent)
    check_rotated(f64(q[:5]), case["q"][:5], depth, [1.0] * 32, "half", 1.0, "bf16")
    # offsets that make no sense
    for off in ([0, -1, 5, 70], [0, 2, 71, 71], [3, 2, 5, 5]):
        d.off.copy_(torch.tensor(off, dtype=torch.int32))
        d.worker.rotate(rope, d.tok, **fill())
        assert d.worker.status() == A.ERR_STATE, off
    with pytest.raises(A.AladdinError):  # an output in place with another stride
        d.worker.rotate(rope, d.tok, q_out=d.q.as_strided(d.q.shape, (4 * 64, 64, 1)))
    for bad in (A.aladdin_rope(66, 0, 1.0, rope.turn), A.aladdin_rope(0, 0, 1.0, rope.turn), A.aladdin_rope(7, 0, 1.0, rope.turn),
                A.aladdin_rope(64, 2, 1.0, rope.turn), A.aladdin_rope(64, 0, 0.0, rope.turn), A.aladdin_rope(64, 0, math.nan, rope.turn),
                A.aladdin_rope(64, 0, 1.0, None), A.aladdin_rope(64, 0, 1.0, rope.turn + 4)):
        with pytest.raises(A.AladdinError):
            d.worker.rotate(bad, d.tok)
    host = torch.zeros(32, dtype=torch.int64)
    with pytest.raises(A.AladdinError):
        d.worker.rotate(A.aladdin_rope(64, 0, 1.0, host.data_ptr()), d.tok)
    assert d.worker.status() == 0


# ---------------------------------------------------------------------------------------------------------
# append

def check_append(case, d, rotated, tol, acc_off=None, acc=None, skip=()):
    """The cache of d after the tokens entered it; rotated: the keys at their positions, and how far off they may be."""
    k, v = case["k"].copy(), case["v"].copy()
    weight, pos = case["weight"].copy(), case["pos"].copy()
    length, nxt = list(case["len"]), list(case["next"])
    err = np.zeros_like(k)
    for r, held in enumerate(case["len"]):
        if r in skip:
            continue
        toks = ref8.kept(case, r, acc_off, acc)
        for i, t in enumerate(toks):
            p, s = case["table"][r][(held + i) // case["page"]], (held + i) % case["page"]
            if 0 <= p < len(k):
                k[p, :, s], v[p, :, s], err[p, :, s] = rotated[t], case["v_new"][t], tol[t]
                weight[p, :, s], pos[p, :, s] = 0.0, nxt[r] + i
        length[r] += len(toks)
        nxt[r] += len(toks)
    got = f64(d.k)
    same = np.isnan(k)
    assert np.array_equal(np.isnan(got), same)
    assert np.all(np.abs(got - k)[~same] <= err[~same])
    np.testing.assert_array_equal(f64(d.v), v)
    np.testing.assert_array_equal(f64(d.weight), weight)
    np.testing.assert_array_equal(d.pos.cpu().numpy(), pos)
    assert d.len.tolist() == length and d.next.tolist() == nxt


def keys_at(case, freq, layout, kind, scale=1.0, acc_off=None, acc=None):
    """The keys at their positions, and how far off they may be."""
    pos = np.zeros(len(case["k_new"]), int)
    for r, n in enumerate(case["next"]):
        for i, t in enumerate(ref8.kept(case, r, acc_off, acc)):
            pos[t] = n + i
    want = ref8.rotate(case["k_new"], pos, freq, layout, scale)
    size = pair_size(case["k_new"], len(freq), layout)
    tol = U[kind] * np.abs(want) + 2.0 ** -21 * scale * size + (2.0 ** -25 if kind == "f16" else 0.0)
    return want, np.where(size > 0, tol, 0.0)


@pytest.mark.parametrize("rows", ["hnd", "nhd"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,heads,dim,turn,page,lens,toks", [
    ("bf16", 2, 128, 128, 64, [0, 1, 63, 64, 65, 300], [1] * 6),
    ("f16", 8, 128, 128, 16, [0, 15, 16, 100, 5], [17, 1, 40, 0, 333]),
    ("bf16", 1, 96, 64, 32, [31, 0], [2, 900]),
    ("f16", 3, 64, 20, 256, [255, 256, 0], [1, 2, 600]),
    ("bf16", 2, 256, 256, 128, [100, 3], [129, 64])])
def test_append(A, kind, heads, dim, turn, page, lens, toks, layout, rows):  # noqa: F811
    case = make(kind, 2 * heads, heads, dim, page, lens, toks, trees=False)
    case["next"] = [l + 100000 + r for r, l in enumerate(lens)]
    d = Dev(A, case, rows)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    d.worker.append(d.kv, d.tok, rope_of(A, freq, layout))
    assert d.worker.status() == 0
    check_append(case, d, *keys_at(case, freq, layout, kind))


def test_append_choice_and_copies(A):  # noqa: F811
    """Paths of trees, keys that are not rotated; without weights, positions and next positions too."""
    import torch
    case = make("f16", 4, 2, 64, 16, [0, 15, 33], [6, 9, 2])
    acc_off, acc = [0, 3, 3, 4], [0, 2, 5, 1]
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    d = Dev(A, case)
    d.worker.append(d.kv, d.tok, None, ints(acc_off), ints(acc))
    check_append(case, d, case["k_new"], np.zeros_like(case["k_new"]), acc_off, acc)
    d = Dev(A, case)
    d.worker.append(A.make_kv(d.k, d.v, d.table, d.len), d.tok)
    assert d.len.tolist() == [6, 24, 35] and d.next.tolist() == [0, 15, 33]
    np.testing.assert_array_equal(f64(d.weight), case["weight"])
    d2 = Dev(A, case)
    d2.worker.append(d2.kv, d2.tok)
    assert np.array_equal(f64(d.k), f64(d2.k), equal_nan=True)
    # positions behind the cached tokens where there are no next ones
    d = Dev(A, case)
    freq = [1.0, 0.1]
    d.worker.append(A.make_kv(d.k, d.v, d.table, d.len, d.weight, d.pos), d.tok, rope_of(A, freq, "half"))
    d.next.copy_(d.len)
    case["next"] = list(case["len"])
    check_append(case, d, *keys_at(case, freq, "half", "f16"))


def test_append_many_requests(A):  # noqa: F811
    n = 1024
    rng = np.random.default_rng(1)
    case = make("bf16", 2, 1, 64, 16, rng.integers(0, 40, n).tolist(), rng.integers(0, 4, n).tolist(), trees=False)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(32) / 32)
    for _ in range(2):  # the counters come back to where they were
        d = Dev(A, case)
        d.worker.append(d.kv, d.tok, rope_of(A, freq, "half"))
        check_append(case, d, *keys_at(case, freq, "half", "bf16"))


def test_append_refuses(A):  # noqa: F811
    """Requests without room, of lengths, offsets or choices that make no sense keep none; pages outside the pool are
    not written; each is recorded, and the others are served."""
    import torch
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    base = make("bf16", 2, 1, 64, 16, [5, 20, 0], [3, 2, 4], trees=False)
    zero = np.zeros_like(base["k_new"])

    def run(change, skip, acc_off=None, acc=None, **new):
        case = dict(base, **new)
        d = Dev(A, case)
        change(d)
        d.worker.append(d.kv, d.tok, None, None if acc is None else ints(acc_off), None if acc is None else ints(acc))
        assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
        return case, d

    full = base["table"].shape[1] * 16
    case, d = run(lambda d: None, [1], len=[5, full - 1, 0])
    assert d.len.tolist() == [8, full - 1, 4]
    case, d = run(lambda d: None, [1], len=[5, -1, 0])
    assert d.len.tolist() == [8, -1, 4]
    case, d = run(lambda d: d.off.copy_(ints([0, 3, 2, 9])), [1])
    assert d.len.tolist()[:2] == [8, 20]
    for acc in ([0, 3, 0, 1], [0, -1, 0, 1]):
        case, d = run(lambda d: None, [0], [0, 2, 3, 4], acc)
        check_append(case, d, case["k_new"], zero, [0, 2, 3, 4], acc, skip=[0])
    # the page of request 1's new slots: nothing is written there
    for bad in (-1, len(base["k"]), 2 ** 31 - 1, -2 ** 31):
        table = base["table"].copy()
        table[1, 1] = bad
        case, d = run(lambda d: None, [], table=table)
        check_append(case, d, case["k_new"], zero)
    # more chosen tokens than a tree has
    d = Dev(A, base)
    d.worker.append(d.kv, d.tok, None, ints([0, 65, 65, 65]), ints([0] * 65))
    assert d.worker.status() == A.ERR_STATE and d.len.tolist() == [5, 20, 0]


def test_streams_and_graphs(A):  # noqa: F811
    """Calls in the order of another stream, and captured: the replayed step goes on from where the cache is."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [3, 16], [1, 1], room=12)
    freq = 10000.0 ** (-np.arange(32) / 32)
    rope = rope_of(A, freq, "half")
    plain = Dev(A, case)
    for _ in range(5):
        plain.worker.rotate(rope, plain.tok, plain.next)
        plain.worker.append(plain.kv, plain.tok, rope)
    side = torch.cuda.Stream()
    d = Dev(A, case)
    with torch.cuda.stream(side):
        d.worker.append(d.kv, d.tok, rope)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        g = torch.cuda.CUDAGraph()
        worker = A.Worker("bf16", 4, 2, 64, 16)
        with torch.cuda.graph(g, stream=side):
            q, k = worker.rotate(rope, d.tok, d.next)
            worker.append(d.kv, d.tok, rope)
        for _ in range(4):
            g.replay()
    torch.cuda.synchronize()
    assert d.len.tolist() == plain.len.tolist() == [8, 21] and worker.status() == 0
    assert torch.equal(d.k.nan_to_num(), plain.k.nan_to_num()) and torch.equal(d.pos, plain.pos)
    pos = np.array([7, 20])  # of the last replay
    check_rotated(f64(q), case["q"], pos, freq, "half", 1.0, "bf16")
