"""The worker step's operators (aladdin_worker_*) against their definitions in 64 bits.

Tolerances, fixed before the first run. u is half a unit in the last place of 1 (2^-8 for bf16, 2^-11 for f16):
* out: one rounding of the result and one of every softmax weight, u |out| + u sum_j p_j |v_j|; the scores, sums of
  head_dim exact products in 32 bits, are off by less than 1e-4 at these sizes, which moves out by at most twice that
  times sum_j p_j |v_j|; weights of f16 below 2^-14 are rounded at a step of 2^-24, half of it for every key.
* lse: the error of the scores and of a sum and a logarithm in 32 bits, 1e-4 + 2^-21 |lse|.
* weights: e^(error of the scores) - 1 times what was added, plus the 32-bit sums: 2e-4 of the growth + 2^-22 of the weight.
* logprob, top_logprob: 32-bit sums of at most 64 terms a thread and an exponential good to 2^-21: 1e-5 + 2^-21 of the
  logits' and results' size; entropy: the same relative error on a mean distance to the maximum that is at most the
  entropy itself, 1e-5 (1 + entropy).
Whole numbers and moved values are equal."""
import numpy as np
import pytest

import worker_ref as ref

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def A():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()
    from paper_2405_06856_gb300 import build
    build.build()
    from paper_2405_06856_gb300 import aladdin
    return aladdin


def rounded(x, kind):
    """x as kind holds it, in float64."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16 if kind == "bf16" else torch.float16)
    return t.double().numpy()


def make(kind, q_heads, kv_heads, dim, page, lens, toks, seed=0, trees=True, spare=2, room=0):
    """A step's inputs in float64; slots that hold no token are NaN."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    width = max(1, max(-(-(l + max(t, room)) // page) for l, t in zip(lens, toks))) + 1
    need = [-(-(l + max(t, room)) // page) for l, t in zip(lens, toks)]
    pages = sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((n, width), -7, np.int32)
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = order[at:at + m]
        at += m
    shape = (pages, kv_heads, page, dim)
    k, v = np.full(shape, np.nan), np.full(shape, np.nan)
    weight, pos = np.full(shape[:3], np.nan), np.full(shape[:3], -1, np.int32)
    case = dict(kind=kind, page=page, table=table, len=list(lens), scale=dim ** -0.5)
    for r, l in enumerate(lens):
        pg, sl = ref.slots(case, r, l)
        k[pg, :, sl] = rounded(rng.normal(size=(l, kv_heads, dim)), kind)
        v[pg, :, sl] = rounded(rng.normal(size=(l, kv_heads, dim)), kind)
        weight[pg, :, sl] = rng.exponential(size=(l, kv_heads)).astype(np.float32)
        pos[pg, :, sl] = np.arange(l)[:, None]
    off = np.concatenate([[0], np.cumsum(toks)]).astype(np.int32)
    m = int(off[-1])
    parent = np.concatenate([rng.integers(-1, np.arange(t)) for t in toks if t] + [np.empty(0, int)])
    case.update(k=k, v=v, weight=weight, pos=pos, next=list(lens), off=off,
                parent=parent.astype(np.int32) if trees else None,
                q=rounded(1.5 * rng.normal(size=(m, q_heads, dim)), kind),
                k_new=rounded(rng.normal(size=(m, kv_heads, dim)), kind),
                v_new=rounded(rng.normal(size=(m, kv_heads, dim)), kind))
    return case


class Dev:
    """A case's tensors on the GPU, and the call's structs over them."""

    def __init__(self, A, case, rows="hnd", fused=True):
        import torch
        self.A, self.kind = A, torch.bfloat16 if case["kind"] == "bf16" else torch.float16
        put = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()
        self.k, self.v = put(case["k"], self.kind), put(case["v"], self.kind)
        if rows == "nhd":
            self.k, self.v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (self.k, self.v))
        self.table, self.len = put(case["table"], torch.int32), put(case["len"], torch.int32)
        self.weight, self.pos = put(case["weight"], torch.float32), put(case["pos"], torch.int32)
        self.next = put(case["next"], torch.int32)
        self.off = put(case["off"], torch.int32)
        self.parent = None if case["parent"] is None else put(case["parent"], torch.int32)
        q, kn, vn = (put(case[x], self.kind) for x in ("q", "k_new", "v_new"))
        if fused:
            hq, hk = q.shape[1], kn.shape[1]
            x = torch.cat([q, kn, vn], 1)
            q, kn, vn = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        self.q, self.k_new, self.v_new = q, kn, vn
        self.kv = A.make_kv(self.k, self.v, self.table, self.len, self.weight, self.pos, self.next)
        self.tok = A.make_tokens(self.off, q, kn, vn, self.parent)
        hk, page, dim = case["k"].shape[1:]
        self.worker = A.Worker(case["kind"], case["q"].shape[1], hk, dim, page)


def f64(x):
    return x.double().cpu().numpy()


def check_attend(case, out, lse, skip=()):
    want, want_lse = ref.attend(case)
    mag = ref.attend(dict(case, v=np.abs(case["v"]), v_new=np.abs(case["v_new"])))[0]
    got, got_lse = f64(out), f64(lse)
    u = U[case["kind"]]
    tol = u * np.abs(want) + (u + 2e-4) * mag
    if case["kind"] == "f16":
        big = max(np.nanmax(np.abs(x[np.isfinite(x)]), initial=0.0) for x in (case["v"], case["v_new"]))
        tol = tol + (max(case["len"]) + 64) * 2.0 ** -25 * big
    rows = np.ones(len(want), bool)
    for r in skip:
        rows[case["off"][r]:case["off"][r + 1]] = False
    fin = np.isfinite(want[rows])
    assert np.array_equal(np.isnan(got[rows]), np.isnan(want[rows]))
    assert np.array_equal(got[rows][~fin & ~np.isnan(want[rows])], want[rows][~fin & ~np.isnan(want[rows])])
    d = np.abs(got[rows] - want[rows])[fin]
    assert np.all(d <= tol[rows][fin]), (d - tol[rows][fin]).max()
    inf, nan = np.isinf(want_lse[rows]), np.isnan(want_lse[rows])
    assert np.array_equal(got_lse[rows][inf], want_lse[rows][inf])
    assert np.array_equal(np.isnan(got_lse[rows]), nan)
    d = np.abs(got_lse[rows] - want_lse[rows])[~inf & ~nan]
    assert np.all(d <= 1e-4 + 2.0 ** -21 * np.abs(want_lse[rows][~inf & ~nan])), d.max()


EDGES = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300]

ATTEND = [  # kind, query heads, key heads, dim, page, lengths, new tokens
    ("bf16", 8, 2, 128, 64, EDGES, [1] * 12),                      # decoding, every edge of page and tile
    ("f16", 8, 2, 128, 16, EDGES, [1] * 12),
    ("bf16", 4, 4, 64, 32, EDGES, [1] * 12),                       # no shared heads
    ("f16", 7, 1, 96, 128, EDGES, [1] * 12),                       # an odd group, an odd dim
    ("bf16", 4, 2, 256, 256, EDGES, [1] * 12),
    ("f16", 8, 2, 128, 32, [5, 0, 70, 129], [4, 7, 0, 1]),         # ragged trees, none
    ("bf16", 14, 2, 64, 16, [40, 0, 200], [5, 4, 3]),              # two row tiles
    ("f16", 16, 2, 128, 64, [100, 0, 64, 1], [64, 64, 1, 33]),     # the largest trees
    ("bf16", 6, 3, 96, 32, [33, 190], [64, 17]),
    ("f16", 4, 2, 256, 64, [33, 70], [20, 9]),
    ("bf16", 40, 1, 64, 16, [90, 3], [3, 2]),                      # a group of more than a tile's rows
    ("bf16", 2, 1, 64, 16, [20000], [1]),                          # one long axis, split and joined
    ("f16", 4, 1, 128, 128, [9001, 3, 7000], [2, 1, 5]),
]


@pytest.mark.parametrize("kind,hq,hk,dim,page,lens,toks", ATTEND)
@pytest.mark.parametrize("rows,fused,trees", [("hnd", True, True), ("nhd", False, False)])
def test_attend(A, kind, hq, hk, dim, page, lens, toks, rows, fused, trees):
    case = make(kind, hq, hk, dim, page, lens, toks, seed=hq + dim, trees=trees)
    d = Dev(A, case, rows, fused)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend(case, out, lse)
    again, lse2 = d.worker.attend(d.kv, d.tok)
    assert np.array_equal(f64(out), f64(again)) and np.array_equal(f64(lse), f64(lse2))
    assert d.worker.status() == A.OK


def test_attend_many_requests(A):
    """As many requests as a call takes, most of them empty or short."""
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, 1024)
    lens[::3] = 0
    case = make("bf16", 2, 1, 64, 16, lens.tolist(), rng.integers(0, 3, 1024).tolist(), seed=1)
    d = Dev(A, case)
    check_attend(case, *d.worker.attend(d.kv, d.tok))


def test_attend_values_out_of_sight(A):
    """Infinite and NaN keys and values of tokens that a row does not see (siblings, later tokens, slots
    behind the length) leave it alone; rows that see them have what the formula gives."""
    for dim, hq, toks in ((128, 4, [6, 3]), (64, 8, [20, 9]), (96, 2, [64, 2])):
        case = make("bf16", hq, 1, dim, 16, [30, 0], toks, seed=9)
        case["parent"][:toks[0]] = [-1, 0, -1, 2, 1, 0][:toks[0]] + [2] * (toks[0] - 6)
        case["parent"][toks[0]:] = [-1, -1, 0][:toks[1]] + [0] * (toks[1] - 3)
        case["k_new"][1] = np.nan
        case["v_new"][1] = np.nan
        case["v_new"][3, 0, ::2] = np.inf
        case["v_new"][toks[0] + 1] = -np.inf
        d = Dev(A, case)
        check_attend(case, *d.worker.attend(d.kv, d.tok))


def test_attend_scores_of_minus_infinity(A):
    """A row whose scores are all -inf gives zeros and lse -inf, a row with some ignores those keys."""
    case = make("f16", 4, 2, 64, 16, [0, 20, 40], [1, 1, 2], seed=3, trees=False)
    case["q"] = np.abs(case["q"]) + 0.25
    case["q"] = rounded(case["q"], "f16")
    case["k_new"][0] = -np.inf
    pg, sl = ref.slots(case, 1, 20)
    case["k"][pg[:13], :, sl[:13]] = -np.inf
    pg, sl = ref.slots(case, 2, 40)
    case["k"][pg, 0, sl] = -np.inf
    case["k_new"][2, 0] = -np.inf
    d = Dev(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend(case, out, lse)
    assert np.isneginf(f64(lse)[0]).all() and (f64(out)[0] == 0).all()


def test_attend_large_scores(A):
    """Scores of hundreds: only the running maximum keeps the exponentials in range."""
    case = make("bf16", 4, 1, 128, 32, [200, 0], [3, 2], seed=4)
    case["scale"] = 3.0
    d = Dev(A, case)
    out, lse = d.worker.attend(d.kv, d.tok, 3.0)
    got, want = f64(lse), ref.attend(case)[1]
    # the scores' error grows with the scale: 1e-4 at 128^-0.5
    assert np.all(np.abs(got - want) <= 1e-4 * 3.0 * 128 ** 0.5 + 2.0 ** -21 * np.abs(want))
    assert np.isfinite(f64(out)).all()


def test_attend_strided_outputs_and_other_stream(A):
    import torch
    case = make("bf16", 4, 2, 64, 16, [50, 0, 33], [2, 1, 4], seed=6)
    d = Dev(A, case)
    wide = torch.full((7, 6, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    out, lse = d.worker.attend(d.kv, d.tok, out=wide[:, :4])
    check_attend(case, out, lse)
    assert bool((wide[:, 4:] == 5).all())
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        q = d.q * 1  # made on the side stream, read by the call after it
        out2, lse2 = d.worker.attend(d.kv, A.make_tokens(d.off, q, d.k_new, d.v_new, d.parent))
        out2, lse2 = out2 * 1, lse2 * 1
    side.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


def test_offsets_past_32_bits(A):
    """Pages more than 2^31 elements apart."""
    import torch
    case = make("bf16", 2, 1, 64, 16, [40], [2], seed=8, spare=0, room=8)
    d = Dev(A, case)
    far = (1 << 31) + 64
    n = case["k"].shape[0]
    big = []
    for x in (d.k, d.v):
        y = torch.empty((n - 1) * far + 16 * 64, dtype=torch.bfloat16, device="cuda")
        y = y.as_strided((n, 1, 16, 64), (far, 16 * 64, 64, 1))
        y.copy_(x)
        big.append(y)
    kv = A.make_kv(big[0], big[1], d.table, d.len, d.weight, d.pos, d.next)
    out, lse = d.worker.attend(kv, d.tok)
    check_attend(case, out, lse)
    d.worker.accept(kv, d.tok, None, lse)
    got = ref.accept(case, [0, 2], [0, 1], f64(lse))
    pg, sl = ref.slots(case, 0, 42)
    assert np.array_equal(f64(big[0])[pg, :, sl], got[0][pg, :, sl])
    d.worker.evict(kv, torch.tensor([20], dtype=torch.int32, device="cuda"), 4)
    assert int(d.len[0]) == 20 and d.worker.status() == A.OK


def test_attend_refuses_requests_on_the_gpu(A):
    """Lengths, offsets, pages and parents that make no sense: their request alone is touched."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [50, 20, 33, 40], [2, 1, 4, 3], seed=6)
    fresh = lambda: Dev(A, case)
    d = fresh()
    good, good_lse = d.worker.attend(d.kv, d.tok)
    for r, bad in ((0, -1), (1, 10 ** 6), (2, 2 ** 31 - 1)):
        d = fresh()
        d.len[r] = bad
        out, lse = torch.full_like(good, 7.0), torch.full_like(good_lse, 7.0)
        d.worker.attend(d.kv, d.tok, out=out, lse=lse)
        assert d.worker.status() == A.ERR_STATE and d.worker.status() == A.OK
        lo, hi = case["off"][r], case["off"][r + 1]
        rest = [i for i in range(10) if not lo <= i < hi]
        assert torch.equal(out[rest], good[rest]) and bool((out[lo:hi] == 7).all()) and bool((lse[lo:hi] == 7).all())
    for off in ([0, 2, 3, 7, 99], [0, 2, 1, 7, 10], [-3, 2, 3, 7, 10]):
        d = fresh()
        d.off.copy_(torch.tensor(off, dtype=torch.int32))
        out = torch.full_like(good, 7.0)
        d.worker.attend(d.kv, d.tok, out=out)
        assert d.worker.status() == A.ERR_STATE
    # a page outside the pool hides its tokens
    for bad in (-1, case["k"].shape[0], 2 ** 31 - 1):
        d = fresh()
        d.table[0, 1] = bad
        out, lse = d.worker.attend(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE
        hidden = make("bf16", 4, 2, 64, 16, [50, 20, 33, 40], [2, 1, 4, 3], seed=6)
        hidden["table"][0, 1:3] = hidden["table"][0, 2:4]
        hidden["len"][0] = 34
        check_attend(hidden, out, lse)
    d = fresh()
    d.parent[1], d.parent[9] = 1, -5
    out, lse = d.worker.attend(d.kv, d.tok)
    assert d.worker.status() == A.ERR_STATE
    case["parent"][1], case["parent"][9] = -1, -1
    check_attend(case, out, lse)


# ----------------------------------------------------------------------------------------------- accept

def check_cache(case, d, want, grown=None):
    k, v, weight, pos, length, nxt = want
    for r, n in enumerate(length):
        pg, sl = ref.slots(case, r, n)
        assert np.array_equal(f64(d.k)[pg, :, sl], k[pg, :, sl])
        assert np.array_equal(f64(d.v)[pg, :, sl], v[pg, :, sl])
        assert np.array_equal(d.pos.cpu().numpy()[pg, :, sl], pos[pg, :, sl])
        got, w = f64(d.weight)[pg, :, sl], weight[pg, :, sl]
        if grown is None:
            assert np.array_equal(got, w)
        else:
            tol = 2e-4 * grown[pg, :, sl] + 2.0 ** -22 * np.abs(w)
            assert np.all(np.abs(got - w) <= tol), (np.abs(got - w) - tol).max()
    assert d.len.cpu().tolist() == length and d.next.cpu().tolist() == nxt


ACCEPT = [  # kind, query heads, key heads, dim, page, lengths, new tokens, kept
    ("bf16", 8, 2, 128, 64, EDGES, [1] * 12, None),
    ("f16", 7, 1, 96, 16, EDGES, [2] * 12, [[0, 1]] * 5 + [[1]] * 4 + [[]] * 3),
    ("bf16", 4, 2, 256, 32, [10, 0, 130], [5, 4, 3], [[0, 2, 4], [], [2]]),
    ("f16", 40, 2, 64, 16, [100, 70], [6, 3], [[0, 1, 2, 5], [0, 2]]),      # more rows than are staged at once
    ("bf16", 2, 1, 64, 16, [200, 0], [64, 64], [list(range(64)), list(range(64))]),
    ("f16", 4, 1, 128, 128, [9001, 3, 7000], [2, 1, 5], [[1], [0], [0, 3, 4]]),
]


@pytest.mark.parametrize("kind,hq,hk,dim,page,lens,toks,kept", ACCEPT)
@pytest.mark.parametrize("weigh", [True, False])
def test_accept(A, kind, hq, hk, dim, page, lens, toks, kept, weigh):
    import torch
    case = make(kind, hq, hk, dim, page, lens, toks, seed=hq)
    case["next"] = [l + 11 for l in lens]  # requests that were reduced before
    if kept is None:
        acc_off, acc = case["off"], np.concatenate([np.arange(t) for t in toks]).astype(np.int32)
    else:
        acc_off = np.concatenate([[0], np.cumsum([len(x) for x in kept])]).astype(np.int32)
        acc = np.concatenate([np.array(x, np.int32) for x in kept])
        for r, path in enumerate(kept):  # a path from the root
            for i, t in enumerate(path):
                case["parent"][case["off"][r] + t] = path[i - 1] if i else -1
    d = Dev(A, case, "nhd" if dim == 96 else "hnd")
    lse = d.worker.attend(d.kv, d.tok)[1] if weigh else None
    want = ref.accept(case, acc_off, acc, f64(lse) if weigh else None)
    grown = ref.accept(dict(case, weight=np.zeros_like(case["weight"])), acc_off, acc, f64(lse))[2] if weigh else None
    args = (None, None) if kept is None else (torch.from_numpy(acc_off).cuda(), torch.from_numpy(acc).cuda())
    d.worker.accept(d.kv, d.tok, None, lse, *args)
    check_cache(case, d, want, grown)
    assert d.worker.status() == A.OK
    if weigh:  # every kept row's weights sum to one in every head
        total = np.nansum(grown)
        assert abs(total - len(acc) * hq) <= 2e-4 * len(acc) * hq + 1e-9


def test_accept_without_positions(A):
    import torch
    case = make("bf16", 4, 2, 64, 16, [5, 31], [1, 2], seed=2, trees=False)
    d = Dev(A, case)
    kv = A.make_kv(d.k, d.v, d.table, d.len)
    d.worker.accept(kv, A.make_tokens(d.off, None, d.k_new, d.v_new))
    want = ref.accept(case, case["off"], [0, 0, 1])
    for r, n in enumerate(want[4]):
        pg, sl = ref.slots(case, r, n)
        assert np.array_equal(f64(d.k)[pg, :, sl], want[0][pg, :, sl])
    assert d.len.cpu().tolist() == want[4] and d.next.cpu().tolist() == case["next"]
    kv = A.make_kv(d.k, d.v, d.table, d.len, None, d.pos)
    d.worker.accept(kv, A.make_tokens(d.off, None, d.k_new, d.v_new))
    pg, sl = ref.slots(case, 1, 35)
    assert d.pos.cpu().numpy()[pg[33:], 0, sl[33:]].tolist() == [33, 34]
    assert torch.equal(d.len.cpu(), torch.tensor([7, 35], dtype=torch.int32))


def test_accept_refuses_requests_on_the_gpu(A):
    """No room, no page, no such token, more than a tree: the request keeps nothing, the others do."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [47, 20, 16], [2, 1, 4], seed=6)
    acc_off, acc = np.array([0, 2, 3, 4], np.int32), np.array([0, 1, 0, 3], np.int32)
    case["parent"][:2], case["parent"][6] = [-1, 0], -1

    def none_for(r, spoil):
        d = Dev(A, case)
        lse = d.worker.attend(d.kv, d.tok)[1]
        ao, ac = torch.from_numpy(acc_off).cuda(), torch.from_numpy(acc).cuda()
        n0, w0, k0 = d.len.clone(), d.weight.clone(), d.k.clone()
        kv = spoil(d, ac) or d.kv
        d.worker.accept(kv, d.tok, None, lse, ao, ac)
        assert d.worker.status() == A.ERR_STATE
        want = case["len"][:]
        for q, a in enumerate((2, 1, 1)):
            want[q] += 0 if q == r else a
        assert d.len.cpu().tolist() == want
        pg, sl = ref.slots(case, r, case["len"][r])
        assert np.array_equal(w0.cpu().numpy()[pg, :, sl], d.weight.cpu().numpy()[pg, :, sl])
        return d

    def set_table(r, i, p):
        def f(d, ac):
            d.table[r, i] = p
        return f

    none_for(0, set_table(0, 3, -1))
    none_for(0, set_table(0, 3, case["k"].shape[0]))
    none_for(1, lambda d, ac: ac[2:3].fill_(1) and None)
    none_for(1, lambda d, ac: ac[2:3].fill_(-1) and None)
    none_for(0, lambda d, ac: A.make_kv(d.k, d.v, d.table[:, :3], d.len, d.weight, d.pos, d.next))


# ----------------------------------------------------------------------------------------------- evict

EVICT = [  # kind, key heads, dim, page, lengths, budgets, recent
    ("bf16", 2, 64, 16, [0, 1, 17, 64, 65, 300], [0, 0, 5, 64, 64, 100], 3),
    ("f16", 1, 128, 64, [1025, 1024, 1030], [1024, 1024, 1024], 128),
    ("bf16", 3, 96, 32, [500, 700], [499, 1], 0),
    ("f16", 2, 256, 128, [300, 200], [100, 150], 1000),         # everything is recent
    ("bf16", 1, 64, 16, [5000, 9000], [0, 2999], 64),
    ("f16", 2, 64, 256, [40000], [10001], 500),
]


@pytest.mark.parametrize("kind,hk,dim,page,lens,budget,recent", EVICT)
@pytest.mark.parametrize("weights", ["spread", "ties", "odd"])
def test_evict(A, kind, hk, dim, page, lens, budget, recent, weights):
    import torch
    case = make(kind, hk, hk, dim, page, lens, [1] * len(lens), seed=dim)
    rng = np.random.default_rng(1)
    case["next"] = [l + 40 for l in lens]
    for r, l in enumerate(lens):  # positions in any order, with gaps
        pg, sl = ref.slots(case, r, l)
        for h in range(hk):
            case["pos"][pg, h, sl] = rng.permutation(l + 40)[:l]
            w = case["weight"][pg, h, sl]
            if weights == "ties":
                w = rng.integers(0, 3, l).astype(np.float32)
            elif weights == "odd":
                w = (w * 1e-38).astype(np.float32)
                pick = rng.integers(0, 8, l)
                for i, x in enumerate((np.nan, np.inf, -np.inf, -0.0, 0.0, -1.0)):
                    w[pick == i] = x
            case["weight"][pg, h, sl] = w
    d = Dev(A, case, "nhd" if dim == 96 else "hnd")
    d.worker.evict(d.kv, torch.tensor(budget, dtype=torch.int32, device="cuda"), recent)
    k, v, weight, pos, length = ref.evict(case, budget, recent)
    for r, n in enumerate(length):
        pg, sl = ref.slots(case, r, n)
        for got, want in ((f64(d.k), k), (f64(d.v), v), (f64(d.weight), weight), (d.pos.cpu().numpy(), pos)):
            assert np.array_equal(got[pg, :, sl], want[pg, :, sl], equal_nan=True)
    assert d.len.cpu().tolist() == length and d.next.cpu().tolist() == case["next"]
    assert d.worker.status() == A.OK
    before = f64(d.weight)
    d.worker.evict(d.kv, torch.tensor(budget, dtype=torch.int32, device="cuda"), recent)  # all within budget now
    assert np.array_equal(before, f64(d.weight), equal_nan=True) and d.len.cpu().tolist() == length


def test_evict_more_keys_than_shared_memory(A):
    """A request of more slots than a cluster's shared memory holds keys of."""
    import torch
    n, b = 420000, 100003
    pages = -(-n // 256)
    w = torch.rand((pages, 1, 256), device="cuda")
    w[w < 0.05] = 0.5  # equal keys
    pos = torch.arange(pages * 256, device="cuda", dtype=torch.int32).view(pages, 1, 256)
    k = torch.randn((pages, 1, 256, 64), device="cuda").to(torch.bfloat16)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, -1)
    i32 = lambda x: torch.tensor([x], dtype=torch.int32, device="cuda")
    length, nxt = i32(n), i32(n)
    w0, k0 = w.flatten()[:n].cpu().numpy().copy(), k.clone().view(-1, 64)
    with A.Worker("bf16", 1, 1, 64, 256) as worker:
        worker.evict(A.make_kv(k, k.clone(), table, length, w, pos, nxt), i32(b), 1000)
        assert worker.status() == A.OK
    key = w0.astype(np.float64)
    key[n - 1000:] = np.inf
    stay = np.zeros(n, bool)
    stay[np.lexsort((np.arange(n), -key))[:b]] = True
    src = np.arange(b)
    src[~stay[:b]] = b + np.flatnonzero(stay[b:])
    src = torch.from_numpy(src).cuda()
    assert torch.equal(k.view(-1, 64)[:b], k0[src]) and int(length) == b
    assert torch.equal(pos.flatten()[:b].long(), src)


def test_evict_refuses_requests_on_the_gpu(A):
    import torch
    case = make("bf16", 2, 2, 64, 16, [50, 60, 40], [1] * 3, seed=3)
    d = Dev(A, case)
    d.worker.evict(d.kv, torch.tensor([-1, 30, 30], dtype=torch.int32, device="cuda"), 4)
    assert d.worker.status() == A.ERR_STATE and d.len.cpu().tolist() == [50, 30, 30]
    d = Dev(A, case)
    d.len[1] = 10 ** 6
    d.worker.evict(d.kv, torch.tensor([20, 30, 30], dtype=torch.int32, device="cuda"), 4)
    assert d.worker.status() == A.ERR_STATE and d.len.cpu().tolist() == [20, 10 ** 6, 30]
    d = Dev(A, case)
    d.table[2, 1] = 9999  # its slots count as the least
    d.worker.evict(d.kv, torch.tensor([50, 60, 20], dtype=torch.int32, device="cuda"), 0)
    assert d.worker.status() == A.ERR_STATE and d.len.cpu().tolist() == [50, 60, 20]


# ----------------------------------------------------------------------------------------------- logprobs

def check_logprobs(x, token, top, got):
    lp, ent, rank, ids, tlp = ref.logprobs(x, token, top)
    assert np.array_equal(got[2].cpu().numpy(), rank)
    assert np.array_equal(got[3].cpu().numpy(), ids)
    big = np.max(np.abs(np.where(np.isfinite(x), x, 0)))
    for g, w, tol in ((f64(got[0]), lp, None), (f64(got[4]), tlp, None), (f64(got[1]), ent, 1e-5 * (1 + np.abs(ent)))):
        fin = np.isfinite(w)
        assert np.array_equal(np.isnan(g), np.isnan(w))
        assert np.array_equal(g[~fin & ~np.isnan(w)], w[~fin & ~np.isnan(w)])
        if tol is None:
            tol = 1e-5 + 2.0 ** -21 * (big + np.abs(w))
        assert np.all(np.abs(g - w)[fin] <= tol[fin]), np.abs(g - w)[fin].max()


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,vocab,top", [(1, 1, 1), (3, 2, 2), (2, 7, 5), (5, 8, 8), (4, 64, 64), (3, 257, 20),
                                         (2, 4099, 64), (300, 1000, 3), (2, 16000, 20), (1, 33333, 64)])
def test_logprobs(A, kind, n, vocab, top):
    import torch
    rng = np.random.default_rng(vocab)
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[kind]
    x = torch.from_numpy(4.0 * rng.normal(size=(n, vocab))).to(t)
    token = rng.integers(0, vocab, n).astype(np.int32)
    with A.Worker("bf16", 1, 1, 64, 16) as w:
        got = w.logprobs(x.cuda(), torch.from_numpy(token).cuda(), top)
        check_logprobs(x.double().numpy(), token, top, got)
        assert w.status() == A.OK
        part = w.logprobs(x.cuda())
        assert part[0] is None and part[2] is None and torch.equal(part[1], got[1])


@pytest.mark.parametrize("kind", ["bf16", "f32"])
def test_logprobs_rows_at_any_address(A, kind):
    """Rows that start at every offset from 16 bytes, in a wider matrix whose rest is NaN."""
    import torch
    t = torch.bfloat16 if kind == "bf16" else torch.float32
    rng = np.random.default_rng(2)
    with A.Worker("bf16", 1, 1, 64, 16) as w:
        for start in range(9):
            for vocab in (3, 61, 2051):
                wide = torch.full((4, vocab + 21), float("nan"), dtype=t)
                wide[:, start:start + vocab] = torch.from_numpy(3.0 * rng.normal(size=(4, vocab))).to(t)
                token = rng.integers(0, vocab, 4).astype(np.int32)
                x = wide.cuda()[:, start:start + vocab]
                got = w.logprobs(x, torch.from_numpy(token).cuda(), 3)
                check_logprobs(wide[:, start:start + vocab].double().numpy(), token, 3, got)


@pytest.mark.parametrize("vocab", [40, 3000, 20000])
def test_logprobs_odd_rows(A, vocab):
    """Equal values, masked values, infinities, NaN, -0, tokens outside the vocabulary; nearly all large
    entries in one thread's share of the row."""
    import torch
    rng = np.random.default_rng(3)
    x = (2.0 * rng.normal(size=(14, vocab))).astype(np.float32)
    x[0] = 1.5
    x[1] = -np.inf
    x[2, ::2] = -np.inf
    x[3, vocab // 2] = np.nan
    x[4, vocab // 3] = np.inf
    x[5] = np.finfo(np.float32).min
    x[6] = np.where(np.arange(vocab) % 3 == 0, 0.0, -0.0)
    x[7] = np.round(x[7])
    x[8] = np.arange(vocab) * 1e-3
    x[9] = -np.arange(vocab) * 1e-3
    x[10, ::1024] = 30.0
    x[10, 1::1024] = 31.0
    x[10, 2::1024] = 32.0
    x[11] = 5.0e4
    x[12, :] = np.nan
    x[13] = np.where(np.arange(vocab) // 4 % 256 == 3, 40.0 + x[13], x[13])
    token = rng.integers(0, vocab, 14).astype(np.int32)
    token[3], token[6] = vocab // 2, vocab - 1
    with A.Worker("bf16", 1, 1, 64, 16) as w:
        for top in (1, 20, 40):
            got = w.logprobs(torch.from_numpy(x).cuda(), torch.from_numpy(token).cuda(), top)
            check_logprobs(x.astype(np.float64), token, top, got)
        assert w.status() == A.OK
        token[:4] = [-1, vocab, 2 ** 31 - 1, -2 ** 31]
        got = w.logprobs(torch.from_numpy(x).cuda(), torch.from_numpy(token).cuda(), 2)
        check_logprobs(x.astype(np.float64), token, 2, got)
        assert w.status() == A.ERR_STATE


def test_logprobs_list_overflow(A):
    """More large entries than the kernel's list holds, held by too few threads for a tight bound."""
    import torch
    vocab = 400000
    x = np.random.default_rng(4).normal(size=(1, vocab)).astype(np.float32)
    own = np.arange(vocab) // 4 % 256 < 8  # the vectors of eight threads of every slice
    x[0, own] += 100.0
    with A.Worker("bf16", 1, 1, 64, 16) as w:
        got = w.logprobs(torch.from_numpy(x).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda"), 20)
    want = np.lexsort((np.arange(vocab), -x[0].astype(np.float64)))[:20]
    assert np.array_equal(got[3].cpu().numpy()[0], want)


# ----------------------------------------------------------------------------------------------- refusals

def test_worker_refuses_arguments(A):
    import torch
    case = make("bf16", 4, 2, 64, 16, [5, 31], [1, 2], seed=2)
    d = Dev(A, case)
    w = d.worker
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(A.AladdinError) as e:
            w.attend(d.kv, d.tok, scale)
        assert e.value.code == A.ERR_ARG
    with pytest.raises(TypeError):
        A.make_kv(d.k.cpu(), d.v.cpu(), d.table, d.len)
    with pytest.raises(TypeError):
        A.make_kv(d.k, d.v, d.table.long(), d.len)
    with pytest.raises(ValueError):
        A.make_kv(d.k, d.v, d.table, d.len[:1])
    with pytest.raises(ValueError):
        A.make_kv(d.k, d.v[:, :1], d.table, d.len)
    with pytest.raises(ValueError):
        w.attend(A.make_kv(d.k, d.v, d.table[:1], d.len[:1]), d.tok)
    with pytest.raises(ValueError):
        w.attend(A.make_kv(d.k.half(), d.v.half(), d.table, d.len), d.tok)
    with pytest.raises(ValueError):
        w.evict(A.make_kv(d.k, d.v, d.table, d.len), d.len)
    with pytest.raises(ValueError):
        w.accept(A.make_kv(d.k, d.v, d.table, d.len), d.tok, None, torch.zeros(3, 4, device="cuda"))
    # the C ABI's own checks
    kv, tok = A.make_kv(d.k, d.v, d.table, d.len, d.weight, d.pos, d.next), d.tok
    out = torch.empty(3, 4, 64, dtype=torch.bfloat16, device="cuda")

    def refused(code=A.ERR_ARG, **change):
        bad = A.aladdin_kv.from_buffer_copy(kv)
        bad_tok = A.aladdin_tokens.from_buffer_copy(tok)
        for name, value in change.items():
            setattr(bad if hasattr(bad, name) and not name.startswith("t_") else bad_tok,
                    name.removeprefix("t_"), value)
        with pytest.raises(A.AladdinError) as e:
            A.aladdin_worker_attend(w.handle, bad, bad_tok, 0.1, out.data_ptr(), 256, None)
        assert e.value.code == code

    host = np.zeros(4096, np.int32)
    refused(k=None)
    refused(len=None)
    refused(table=host.ctypes.data)
    refused(pages=0)
    refused(table_width=0)
    refused(table_width=1 << 30)
    refused(token_stride=63)
    refused(token_stride=60)
    refused(page_stride=0)
    refused(k=d.k.data_ptr() + 2)
    refused(t_n_req=-1)
    refused(t_n_req=1025)
    refused(t_n_tok=-1)
    refused(t_off=None)
    refused(t_q=None)
    refused(t_q=host.ctypes.data)
    refused(t_q_stride=100)
    refused(t_k_stride=64)
    for args in ((0, 256), (out.data_ptr() + 2, 256), (out.data_ptr(), 248), (host.ctypes.data, 256)):
        with pytest.raises(A.AladdinError):
            A.aladdin_worker_attend(w.handle, kv, tok, 0.1, args[0] or None, args[1], None)
    x = torch.zeros(2, 100, device="cuda")
    t = torch.zeros(2, dtype=torch.int32, device="cuda")
    f = torch.zeros(2, device="cuda")
    for dtype, n, vocab, logits, stride, tk, top in ((3, 2, 100, x.data_ptr(), 100, t, 0), (2, -1, 100, x.data_ptr(), 100, t, 0),
                                                     (2, 2, 0, x.data_ptr(), 100, t, 0), (2, 2, 100, None, 100, t, 0),
                                                     (2, 2, 100, x.data_ptr(), 99, t, 0), (2, 2, 100, x.data_ptr(), 100, None, 0),
                                                     (2, 2, 100, x.data_ptr(), 100, t, 65), (2, 2, 30, x.data_ptr(), 100, t, 31),
                                                     (2, 2, 100, x.data_ptr() + 2, 100, t, 0), (2, 2, 100, host.ctypes.data, 100, t, 0)):
        with pytest.raises(A.AladdinError) as e:
            A.aladdin_worker_logprobs(w.handle, dtype, n, vocab, logits, stride, tk, top, f, None, None, None, None)
        assert e.value.code == A.ERR_ARG
    with pytest.raises(A.AladdinError):
        A.aladdin_worker_evict(w.handle, kv, 2, t, -1)
    with pytest.raises(A.AladdinError):
        A.aladdin_worker_evict(w.handle, kv, 2, None, 0)
    assert w.status() == A.OK


def test_nothing_to_do(A):
    """No requests, no tokens: calls succeed and leave everything alone."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [5, 31], [0, 0], seed=2)
    d = Dev(A, case, fused=False)
    out, lse = d.worker.attend(d.kv, d.tok)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    d.worker.accept(d.kv, d.tok)
    got = d.worker.logprobs(torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), 3)
    assert got[3].shape == (0, 3)
    assert d.len.cpu().tolist() == [5, 31] and d.worker.status() == A.OK
