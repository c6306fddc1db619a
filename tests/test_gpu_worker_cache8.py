"""The cache of 8 bits: appending to it (aladdin_worker_append8) and attention over it (aladdin_worker_attend8) against their
definitions in 64 bits.

Tolerances, fixed before the first run.
* codes: those of the definition, but for values that 32-bit arithmetic puts on the other side of a border: their rotation is
  off by 2^-21 of the pair's size (see test_gpu_worker_rope.py), so codes are compared as the values that they stand for,
  which differ by a step (2^-3 of the larger, 2^-9 scales at least) where the exact value lies that near to a border, and
  are equal otherwise. Values are not rotated: their codes are equal. Scales likewise, where the largest value lies that
  near to 448 scales.
* out: as for 16 bits (u |out|; scores, sums of exact products in 32 bits, off by less than 1e-4, which moves out by twice
  that times sum_j p_j |v_j|), with weights rounded to half precision: 2^-11 of each, and below 2^-14 of the largest a step
  of 2^-24, half of it for every key, in units of 448 times the largest scale, 2^8 times that where the maximum that
  weights refer to may lag behind.
* lse: 1e-4 + 2^-21 |lse|."""
import math

import numpy as np
import pytest

import worker8_ref as ref8
import worker_ref as ref
from test_gpu_worker import A, f64, rounded  # noqa: F401
from test_gpu_worker_rope import keys_at, rope_of

pytestmark = pytest.mark.gpu

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def make8(kind, q_heads, kv_heads, dim, page, lens, toks, block=16, seed=0, trees=True, spare=2, room=0, scales="power"):
    """A step's inputs; slots that hold no token have NaN codes, and blocks without tokens NaN scales. scales: powers of two
    near 1 / 448, any numbers, or ones of very different size, some of them 0."""
    rng = np.random.default_rng(seed)
    n = len(lens)
    need = [-(-(l + max(t, room)) // page) for l, t in zip(lens, toks)]
    width, pages = max(1, max(need)) + 1, sum(need) + spare
    order = rng.permutation(pages)
    table = np.full((n, width), -7, np.int32)
    at = 0
    for r, m in enumerate(need):
        table[r, :m] = order[at:at + m]
        at += m
    case = dict(kind=kind, page=page, table=table, len=list(lens), next=list(lens), scale=dim ** -0.5)
    for name in ("k", "v"):
        codes = np.full((pages, kv_heads, page, dim), 127, np.uint8)
        s = np.full((pages, kv_heads, page // block), np.nan, np.float32)
        for r, l in enumerate(lens):
            pg, sl = ref.slots(case, r, l)
            x = rng.normal(size=(l, kv_heads, dim))
            if scales == "power":
                sc = 2.0 ** rng.integers(-8, -5, (pages, kv_heads, page // block))
            elif scales == "any":
                sc = rng.uniform(0.005, 0.02, (pages, kv_heads, page // block))
            else:
                sc = 2.0 ** rng.integers(-45, 3, (pages, kv_heads, page // block)) * (rng.random((pages, kv_heads, page // block)) < 0.8)
                x = 200.0 * x.clip(-2, 2)
            sc = sc.astype(np.float32)
            blocks = sc[pg, :, sl // block]
            if scales in ("power", "any"):
                x = (x / blocks[..., None].astype(np.float64)).clip(-448, 448)
            codes[pg, :, sl] = ref8.code(x)
            s[pg, :, sl // block] = blocks
        case[name], case[name + "_scale"] = codes, s
    off = np.concatenate([[0], np.cumsum(toks)]).astype(np.int32)
    m = int(off[-1])
    parent = np.concatenate([rng.integers(-1, np.arange(t)) for t in toks if t] + [np.empty(0, int)])
    case.update(off=off, parent=parent.astype(np.int32) if trees else None,
                q=rounded(1.5 * rng.normal(size=(m, q_heads, dim)), kind),
                k_new=rounded(rng.normal(size=(m, kv_heads, dim)), kind),
                v_new=rounded(rng.normal(size=(m, kv_heads, dim)), kind))
    return case


class Dev8:
    """A case's tensors on the GPU, and the call's structs over them."""

    def __init__(self, A, case, rows="hnd", worker=None):  # noqa: F811
        import torch
        self.kind = torch.bfloat16 if case["kind"] == "bf16" else torch.float16
        put = lambda x, t: torch.from_numpy(np.ascontiguousarray(x)).to(t).cuda()
        self.codes = {}
        for name in ("k", "v"):
            x = put(case[name], torch.uint8)
            if rows == "nhd":
                x = x.transpose(1, 2).contiguous().transpose(1, 2)
            self.codes[name] = x
        self.k, self.v = (self.codes[x].view(torch.float8_e4m3fn) for x in ("k", "v"))
        self.k_scale, self.v_scale = put(case["k_scale"], torch.float32), put(case["v_scale"], torch.float32)
        self.table, self.len, self.next = (put(case[x], torch.int32) for x in ("table", "len", "next"))
        self.off = put(case["off"], torch.int32)
        self.parent = None if case["parent"] is None else put(case["parent"], torch.int32)
        x = torch.cat([put(case[x], self.kind) for x in ("q", "k_new", "v_new")], 1)
        hq, hk = case["q"].shape[1], case["k_new"].shape[1]
        self.q, self.k_new, self.v_new = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        self.kv = A.make_kv8(self.k, self.v, self.k_scale, self.v_scale, self.table, self.len, self.next)
        self.tok = A.make_tokens(self.off, self.q, self.k_new, self.v_new, self.parent)
        self.worker = worker or A.Worker(case["kind"], hq, hk, case["q"].shape[2], case["page"])


def check_attend8(case, out, lse, skip=()):
    want, want_lse = ref8.attend8(case)
    mag = ref8.attend8(dict(case, v=case["v"] & 127, v_new=np.abs(case["v_new"])))[0]
    got, got_lse = f64(out), f64(lse)
    u = U[case["kind"]]
    tol = u * np.abs(want) + (2.0 ** -11 + 2e-4) * mag
    s = case["v_scale"][np.isfinite(case["v_scale"])]
    tol = tol + (max(case["len"]) + 64) * 2.0 ** -17 * 448 * s.max(initial=0.0) * 2.0 ** -8
    if case["kind"] == "f16":
        tol = tol + 2.0 ** -25
    rows = np.ones(len(want), bool)
    for r in skip:
        rows[case["off"][r]:case["off"][r + 1]] = False
    got, want, tol, got_lse, want_lse = got[rows], want[rows], tol[rows], got_lse[rows], want_lse[rows]
    nan, inf = np.isnan(want), np.isinf(want)
    assert np.array_equal(np.isnan(got), nan)
    assert np.array_equal(got[inf], want[inf])
    fin = ~nan & ~inf
    d = np.abs(got[fin] - want[fin])
    assert np.all(d <= tol[fin]), (d - tol[fin]).max()
    nan, inf = np.isnan(want_lse), np.isinf(want_lse)
    assert np.array_equal(np.isnan(got_lse), nan) and np.array_equal(got_lse[inf], want_lse[inf])
    fin = ~nan & ~inf
    d = np.abs(got_lse[fin] - want_lse[fin])
    assert np.all(d <= 1e-4 + 2.0 ** -21 * np.abs(want_lse[fin])), d.max()


EDGES = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300]

ATTEND = [  # kind, query heads, key heads, dim, page, block, lengths, new tokens
    ("bf16", 8, 2, 128, 64, 16, EDGES, [1] * 12),                      # decoding, every edge of page and tile
    ("f16", 8, 2, 128, 16, 16, EDGES, [1] * 12),
    ("bf16", 4, 4, 64, 32, 32, EDGES, [1] * 12),                       # no shared heads
    ("f16", 7, 1, 96, 128, 64, EDGES, [1] * 12),                       # an odd group, an odd dim
    ("bf16", 4, 2, 256, 256, 256, EDGES, [1] * 12),
    ("f16", 3, 1, 64, 256, 128, EDGES, [1] * 12),
    ("f16", 8, 2, 128, 32, 16, [5, 0, 70, 129], [4, 7, 0, 1]),         # ragged trees, none
    ("bf16", 14, 2, 64, 16, 16, [40, 0, 200], [5, 4, 3]),              # two row tiles
    ("bf16", 16, 2, 96, 32, 16, [40, 0, 200, 31], [9, 8, 17, 2]),
    ("bf16", 8, 1, 256, 32, 32, [77, 0, 32], [3, 1, 20]),
    ("f16", 64, 8, 128, 32, 16, [130, 3], [64, 33]),                   # trees of many tokens
    ("bf16", 64, 8, 128, 64, 64, [130, 0, 517], [40, 64, 1]),
    ("bf16", 28, 4, 96, 16, 16, [300, 129, 128], [21, 64, 40]),
    ("f16", 8, 1, 64, 128, 32, [1000, 17], [64, 50]),
    ("bf16", 16, 1, 256, 64, 16, [65, 300], [64, 30]),
    ("bf16", 20, 2, 128, 16, 16, [1, 127, 128, 129, 256, 383], [13, 14, 13, 12, 13, 13])]


@pytest.mark.parametrize("scales", ["power", "any", "wide"])
@pytest.mark.parametrize("kind,q_heads,kv_heads,dim,page,block,lens,toks", ATTEND)
def test_attend8(A, kind, q_heads, kv_heads, dim, page, block, lens, toks, scales):  # noqa: F811
    case = make8(kind, q_heads, kv_heads, dim, page, lens, toks, block, scales=scales)
    d = Dev8(A, case, "nhd" if dim == 96 else "hnd")
    out, lse = d.worker.attend(d.kv, d.tok)
    assert d.worker.status() == 0
    check_attend8(case, out, lse)
    again, lse2 = d.worker.attend(d.kv, d.tok)
    assert (out.nan_to_num() == again.nan_to_num()).all() and (lse == lse2).all()


@pytest.mark.parametrize("kind,q_heads,kv_heads,dim,new", [("bf16", 8, 2, 128, 1), ("f16", 4, 4, 64, 1), ("bf16", 16, 2, 96, 3),
                                                           ("bf16", 4, 1, 256, 1), ("bf16", 32, 2, 128, 16), ("f16", 8, 1, 64, 40)])
def test_attend8_long(A, kind, q_heads, kv_heads, dim, new):  # noqa: F811
    """Few long requests: units that many warps or CTAs share."""
    case = make8(kind, q_heads, kv_heads, dim, 64, [9001, 0, 2500], [new, 1, new])
    d = Dev8(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend8(case, out, lse)


@pytest.mark.parametrize("kind,q_heads,kv_heads,dim,new", [("bf16", 64, 8, 128, 40), ("f16", 16, 8, 64, 40), ("bf16", 24, 8, 96, 60),
                                                           ("f16", 8, 8, 256, 30), ("bf16", 40, 8, 128, 30), ("f16", 16, 8, 128, 3),
                                                           ("bf16", 8, 8, 64, 2), ("f16", 8, 8, 256, 1)])
def test_attend8_many_units(A, kind, q_heads, kv_heads, dim, new):  # noqa: F811
    """Warps and CTAs with several units each, of one and of two row tiles in turn, and more tiles than their rings hold."""
    rng = np.random.default_rng(new)
    n = 70
    case = make8(kind, q_heads, kv_heads, dim, 32, rng.integers(0, 900, n).tolist(), rng.integers(0, new + 1, n).tolist(), 32)
    d = Dev8(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    assert d.worker.status() == 0
    check_attend8(case, out, lse)


def test_attend8_chains(A):  # noqa: F811
    case = make8("bf16", 8, 2, 128, 16, [33, 0, 200], [5, 1, 64], trees=False)
    d = Dev8(A, case)
    check_attend8(case, *d.worker.attend(d.kv, d.tok))


def test_attend8_queries_of_any_size(A):  # noqa: F811
    """Rows of queries from 2^-100 to 2^100 (bf16), channels of very different size in one."""
    case = make8("bf16", 8, 2, 64, 16, [100, 40], [3, 5])
    rng = np.random.default_rng(3)
    case["q"] = rounded(case["q"] * 2.0 ** rng.integers(-20, 1, case["q"].shape), "bf16")
    case["q"][1] *= 2.0 ** -100
    case["k_new"] *= 0.5
    d = Dev8(A, case)
    check_attend8(case, *d.worker.attend(d.kv, d.tok))
    # sizes that make one key win, far beyond half precision's range: scores to 2^-21 of their terms' size
    case["q"] = rounded(rng.normal(size=case["q"].shape), "bf16") * 2.0 ** 100
    d = Dev8(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    want, want_lse = ref8.attend8(case)
    assert np.all(np.abs(f64(lse) - want_lse) <= 2.0 ** -20 * 64 * 2.0 ** 102 * case["scale"] * 3)
    assert np.isfinite(f64(out)).all()


@pytest.mark.parametrize("q_heads,toks", [(4, [4, 3]), (32, [40, 9])])
def test_attend8_values_out_of_sight(A, q_heads, toks):  # noqa: F811
    """New tokens that are not finite reach only the rows that see them."""
    case = make8("bf16", q_heads, 2, 64, 16, [20, 0], toks)
    case["parent"][:4] = [-1, 0, 0, 1]
    case["v_new"][2, 0, 3] = math.inf     # seen by token 2 alone
    case["v_new"][3, 1, 5] = math.nan     # by token 3 alone
    case["parent"][4:toks[0]] = 0
    d = Dev8(A, case)
    check_attend8(case, *d.worker.attend(d.kv, d.tok))


@pytest.mark.parametrize("q_heads,toks", [(4, [2, 1]), (32, [30, 2])])
def test_attend8_scores_of_minus_infinity(A, q_heads, toks):  # noqa: F811
    """A row whose scores are all -inf has no result; one with cached tokens does without the new one."""
    case = make8("f16", q_heads, 2, 64, 16, [0, 20], toks)
    case["q"] = np.abs(case["q"]) + 0.1
    case["q"] = rounded(case["q"], "f16")
    case["k_new"][0] = -math.inf
    case["k_new"][toks[0]] = -math.inf
    case["parent"][:toks[0]] = -1
    d = Dev8(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend8(case, out, lse)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()


@pytest.mark.parametrize("q_heads,toks", [(4, [2, 1, 1]), (32, [30, 2, 20])])
def test_attend8_codes_and_scales_that_are_not_finite(A, q_heads, toks):  # noqa: F811
    """NaN codes of cached tokens: keys make their head's rows NaN, values their channel; a scale that is not finite the
    rows of its head and request; others are as they were."""
    import torch
    case = make8("bf16", q_heads, 2, 64, 16, [40, 40, 40], toks)
    good = Dev8(A, case)
    want, want_lse = good.worker.attend(good.kv, good.tok)
    hq = q_heads // 2
    rows = [slice(0, toks[0]), slice(toks[0], toks[0] + toks[1]), slice(toks[0] + toks[1], None)]
    for name, at in (("k", None), ("v", 7)):
        d = Dev8(A, case)
        d.codes[name][int(case["table"][1, 2]), 1, 3, 7] = 255
        out, lse = d.worker.attend(d.kv, d.tok)
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[rows[1], hq:, slice(None) if at is None else at] = True
        assert torch.equal(out.isnan(), bad), name
        assert torch.equal(out[~bad], want[~bad])
        assert torch.equal(lse.isnan(), bad.all(2))
    for name in ("k_scale", "v_scale"):
        for x in (math.nan, math.inf):
            d = Dev8(A, case)
            getattr(d, name)[int(case["table"][1, 1]), 1, 0] = x
            out, lse = d.worker.attend(d.kv, d.tok)
            bad = torch.zeros_like(out, dtype=torch.bool)
            bad[rows[1], hq:] = True
            assert (~out[rows[1], hq:].isfinite()).all(), (name, x)
            assert torch.equal(out[~bad], want[~bad])


@pytest.mark.parametrize("q_heads,toks", [(4, [1, 2, 1]), (32, [30, 2, 20])])
def test_attend8_hidden_pages(A, q_heads, toks):  # noqa: F811
    """A page index outside the pool hides its tokens, and is recorded."""
    for bad in (-1, 1 << 30, -2 ** 31):
        case = make8("bf16", q_heads, 2, 128, 16, [40, 100, 16], toks)
        table = case["table"].copy()
        table[1, 2] = bad if bad != 1 << 30 else len(case["k"])
        table[2, 0] = bad
        d = Dev8(A, dict(case, table=table))
        out, lse = d.worker.attend(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
        # as if the page were not there: request 1 without its third page, request 2 without tokens
        t2 = np.full_like(case["table"], -7)
        t2[0] = case["table"][0]
        t2[1, :-1] = np.delete(case["table"][1], 2)
        check_attend8(dict(case, table=t2, len=[40, 84, 0]), out, lse)


def test_attend8_refuses(A):  # noqa: F811
    import torch
    case = make8("bf16", 8, 2, 64, 16, [40, 20, 16], [1, 2, 1])
    full = case["table"].shape[1] * 16
    for change in (dict(len=[40, -1, 16]), dict(len=[40, full + 1, 16]), dict(off=[0, 1, 0, 4])):
        d = Dev8(A, dict(case, **change))
        out = torch.full((4, 8, 64), 9.0, dtype=torch.bfloat16, device="cuda")
        out, lse = d.worker.attend(d.kv, d.tok, out=out)
        assert d.worker.status() == A.ERR_STATE
        if "len" in change:
            assert (out[1:3] == 9.0).all()
            check_attend8(dict(case, len=[40, 0, 16]), out, lse, skip=[1])
    d = Dev8(A, case)
    kv = d.kv
    for name, bad in (("block", 8), ("block", 32), ("block", 0), ("block", 24), ("page_stride", 8), ("token_stride", 56), ("token_stride", 72),
                      ("head_stride", 0), ("head_stride", -16), ("pages", 0), ("table_width", 0), ("k_scale", None), ("v_scale", None), ("k", None),
                      ("k", d.k.data_ptr() + 8), ("len", None), ("k_scale", d.k_scale.data_ptr() + 2)):
        keep = getattr(kv, name)
        setattr(kv, name, bad)
        for call in (lambda: d.worker.attend(kv, d.tok), lambda: d.worker.append(kv, d.tok)):
            with pytest.raises(A.AladdinError):
                call()
        setattr(kv, name, keep)
    host = torch.ones(d.k_scale.shape)
    kv.k_scale = host.data_ptr()
    with pytest.raises(A.AladdinError):
        d.worker.attend(kv, d.tok)
    assert d.len.tolist() == [40, 20, 16]


@pytest.mark.parametrize("q_heads,most", [(2, 1), (8, 6)])
def test_attend8_thousand_requests(A, q_heads, most):  # noqa: F811
    """As many requests as a call may have, some of them without tokens or cache, in a table with spare columns, into an
    output with spare columns."""
    import torch
    n = 1024
    rng = np.random.default_rng(4)
    case = make8("bf16", q_heads, 1, 64, 16, rng.integers(0, 60, n).tolist(), rng.integers(0, most + 1, n).tolist())
    d = Dev8(A, case)
    m = len(case["q"])
    wide = torch.full((m, q_heads + 1, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    table = torch.cat([d.table, torch.full_like(d.table, -5)], 1)[:, :d.table.shape[1]]
    kv = A.make_kv8(d.k, d.v, d.k_scale, d.v_scale, table, d.len)
    out, lse = d.worker.attend(kv, d.tok, out=wide[:, :q_heads])
    assert d.worker.status() == 0 and (wide[:, q_heads] == 9.0).all()
    check_attend8(case, out, lse)


def test_nothing_to_do(A):  # noqa: F811
    """No requests, no tokens: nothing is read or written."""
    import torch
    case = make8("bf16", 4, 2, 64, 16, [40, 3], [1, 1])
    d = Dev8(A, case)
    rope = rope_of(A, [1.0], "half")
    for off in ([0], [0, 0, 0]):
        n = len(off) - 1
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        kv = A.make_kv8(d.k, d.v, d.k_scale, d.v_scale, d.table[:n], d.len[:n], d.next[:n])
        tok = A.make_tokens(ints(off), d.q[:0], d.k_new[:0], d.v_new[:0])
        out, lse = d.worker.attend(kv, tok)
        assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
        d.worker.append(kv, tok, rope)
        assert d.worker.rotate(rope, tok, d.next[:n])[0].shape == (0, 4, 64)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    d.worker.append(d.kv, d.tok, rope, torch.zeros(3, dtype=torch.int32, device="cuda"), none)
    assert d.len.tolist() == [40, 3] and d.worker.status() == 0
    assert np.array_equal(d.codes["k"].cpu().numpy(), case["k"])


def test_attend8_far_pages(A):  # noqa: F811
    """Pages whose offsets pass 32 bits."""
    import torch
    case = make8("bf16", 8, 2, 128, 64, [150, 64], [1, 2], spare=0)
    big = torch.empty(len(case["k"]) * (3 << 29), dtype=torch.uint8, device="cuda")
    shape, st = case["k"].shape, (3 << 29, 64 * 128, 128, 1)
    d = Dev8(A, case)
    far = []
    for i, name in enumerate(("k", "v")):
        x = big[i * (1 << 28):].as_strided(shape, st)
        x.copy_(d.codes[name])
        far.append(x.view(torch.float8_e4m3fn))
    kv = A.make_kv8(*far, d.k_scale, d.v_scale, d.table, d.len, d.next)
    want = d.worker.attend(d.kv, d.tok)
    got = d.worker.attend(kv, d.tok)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    d.worker.append(kv, d.tok)
    d2 = Dev8(A, case)
    d2.worker.append(d2.kv, d2.tok)
    for x, name in zip(far, ("k", "v")):
        assert torch.equal(x.view(torch.uint8), d2.codes[name])


def test_attend8_in_graphs_and_streams(A):  # noqa: F811
    import torch
    case = make8("f16", 8, 2, 64, 16, [40, 3000, 0], [1, 1, 1])
    d = Dev8(A, case)
    want = d.worker.attend(d.kv, d.tok)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = d.worker.attend(d.kv, d.tok)
        worker = A.Worker("f16", 8, 2, 64, 16)
        graphs, outs = [], []
        for _ in range(2):  # two graphs that share the worker's workspaces
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                outs.append(worker.attend(d.kv, d.tok))
            graphs.append(g)
        for g in graphs + graphs[::-1]:
            g.replay()
    torch.cuda.synchronize()
    for out, lse in [got] + outs:
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])


# ---------------------------------------------------------------------------------------------------------
# append8

def check_append8(case, d, rotated, tol, acc_off=None, acc=None, skip=()):
    after = lambda x: ref8.append8(case, x, acc_off, acc, skip)
    nan = lambda c: np.where(c & 127 == 127, 127, c)  # one NaN is as good as the other
    want = after(rotated)
    block = case["page"] // case["k_scale"].shape[2]
    for name in ("k", "v"):
        got, got_s = nan(d.codes[name].cpu().numpy()), getattr(d, name + "_scale").cpu().numpy()
        want[name] = nan(want[name])
        same = (got_s == want[name + "_scale"]) | (np.isnan(got_s) & np.isnan(want[name + "_scale"]))
        if name == "v":
            assert same.all()
            np.testing.assert_array_equal(got, want[name])
            continue
        # a block's scale is the other power of two only where its largest value is that near to the border
        for p, h, b in np.argwhere(~same):
            s = min(got_s[p, h, b], want["k_scale"][p, h, b])
            assert max(got_s[p, h, b], want["k_scale"][p, h, b]) == 2 * s
            assert {after(rotated + x * tol)["k_scale"][p, h, b] for x in (-1.0, 1.0)} == {s, 2 * s}
        # codes differ only where a value is that near to a border
        lo, hi = (nan(after(rotated + x * tol)["k"]) for x in (-1.0, 1.0))
        ok = (got == want["k"]) | (got == lo) | (got == hi) | ~np.repeat(same, block, 2)[..., None]
        assert ok.all()
        assert (got == want["k"]).mean() > 0.999
    length = [l + (0 if r in skip else len(ref8.kept(case, r, acc_off, acc))) for r, l in enumerate(case["len"])]
    assert d.len.tolist() == length
    assert (np.array(d.next.tolist()) - case["next"]).tolist() == (np.array(length) - case["len"]).tolist()


def keys8(case, freq, layout, scale=1.0, acc_off=None, acc=None):
    want, tol = keys_at(case, freq, layout, case["kind"], scale, acc_off, acc)
    u = U[case["kind"]]
    # without the rounding to 16 bits
    return want, np.where(tol > 0, np.maximum(tol - u * np.abs(want) - (2.0 ** -25 if case["kind"] == "f16" else 0.0), 0.0), 0.0)


@pytest.mark.parametrize("rows", ["hnd", "nhd"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,heads,dim,turn,page,block,lens,toks", [
    ("bf16", 2, 128, 128, 64, 16, [0, 1, 15, 16, 63, 64, 65, 300], [1] * 8),
    ("f16", 8, 128, 128, 16, 16, [0, 15, 16, 100, 5], [17, 1, 40, 0, 133]),
    ("bf16", 1, 96, 64, 32, 32, [31, 0, 33], [2, 200, 70]),
    ("f16", 3, 64, 20, 256, 64, [255, 256, 0, 70], [1, 2, 300, 5]),
    ("f16", 2, 64, 64, 256, 256, [255, 100, 0], [2, 30, 300]),
    ("bf16", 2, 256, 256, 128, 128, [100, 3], [129, 64]),
    ("bf16", 1, 128, 128, 128, 128, [100, 0, 127], [1, 1, 1])])
def test_append8(A, kind, heads, dim, turn, page, block, lens, toks, layout, rows):  # noqa: F811
    case = make8(kind, 2 * heads, heads, dim, page, lens, toks, block, trees=False)
    case["k_new"][::3] *= 8  # scales grow
    case["v_new"][::2] *= 4
    case["next"] = [l + 100000 + r for r, l in enumerate(lens)]
    d = Dev8(A, case, rows)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    d.worker.append(d.kv, d.tok, rope_of(A, freq, layout))
    assert d.worker.status() == 0
    check_append8(case, d, *keys8(case, freq, layout))


def test_append8_token_by_token(A):  # noqa: F811
    """Blocks do not depend on how their tokens came in, but for values below 2^-6 of a scale, which may be rounded
    twice: off by two half steps of 2^-9 scales at most."""
    import torch
    rng = np.random.default_rng(5)
    case = make8("bf16", 4, 2, 64, 32, [0, 0], [40, 23], 16, trees=False)
    case["k_new"] = rounded(case["k_new"] * np.exp(rng.normal(size=case["k_new"].shape[:2]))[..., None], "bf16")
    d = Dev8(A, case)
    rope = rope_of(A, [1.0, 0.25, 0.01], "interleaved")
    d.worker.append(d.kv, d.tok, rope)
    e = Dev8(A, case)
    e.worker = d.worker
    for i in range(40):
        toks = [t for t in (i, 40 + i) if t < 40 or (t < 63 and i < 23)]
        off = torch.tensor([0, 1, len(toks)], dtype=torch.int32, device="cuda")
        e.worker.append(e.kv, A.make_tokens(off, None, e.k_new[toks], e.v_new[toks]), rope)
    assert d.len.tolist() == e.len.tolist() == [40, 23] and d.worker.status() == 0
    for name in ("k", "v"):
        s = getattr(d, name + "_scale")
        assert torch.equal(s.nan_to_num(), getattr(e, name + "_scale").nan_to_num())
        x, y = (z.codes[name].view(torch.float8_e4m3fn).float().nan_to_num() for z in (d, e))
        assert torch.equal(x[x.abs() >= 2.0 ** -6], y[x.abs() >= 2.0 ** -6]) and (x - y).abs().max() <= 2.0 ** -9


def test_append8_choice_and_copies(A):  # noqa: F811
    import torch
    case = make8("f16", 4, 2, 64, 32, [0, 15, 33], [6, 9, 2])
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    acc_off, acc = [0, 3, 3, 4], [0, 2, 5, 1]
    d = Dev8(A, case)
    d.worker.append(d.kv, d.tok, None, ints(acc_off), ints(acc))
    check_append8(case, d, case["k_new"], np.zeros_like(case["k_new"]), acc_off, acc)
    d = Dev8(A, case)
    d.worker.append(d.kv, d.tok)
    check_append8(case, d, case["k_new"], np.zeros_like(case["k_new"]))


def test_append8_sizes_and_what_is_not_finite(A):  # noqa: F811
    """From the smallest to the largest values of the type, zeros, infinities and NaN: stored as NaN, without influence on
    the scale; old codes of NaN stay."""
    import torch
    case = make8("bf16", 2, 1, 64, 16, [0, 0, 0, 5, 0], [16, 4, 2, 3, 3])
    case["parent"] = None
    k = case["k_new"]
    k[:16] *= 2.0 ** -126
    k[16:20] *= 2.0 ** 120
    k[20:22] = 0.0
    k[22, 0, 3], k[22, 0, 4], k[23, 0, 5] = math.inf, -math.inf, math.nan
    case["v_new"][22:] = 448.0 * 2.0 ** -3
    case["v_new"][25:] = math.nan
    k[:] = rounded(k, "bf16")
    p = case["table"][3][0]
    case["k"][p, 0, 2, 2] = 255
    case["k_scale"][p] = 2.0 ** -12
    d = Dev8(A, case)
    d.worker.append(d.kv, d.tok)
    check_append8(case, d, k, np.zeros_like(k))
    got = d.codes["k"][int(p), 0].cpu().numpy()
    assert got[5, 3] & 127 == 127 and got[5, 4] & 127 == 127 and got[6, 5] & 127 == 127 and got[2, 2] & 127 == 127
    assert d.v_scale[int(case["table"][4][0]), 0, 0] == 2.0 ** -126


def test_append8_refuses(A):  # noqa: F811
    import torch
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    base = make8("bf16", 2, 1, 64, 16, [5, 20, 0], [3, 2, 4], trees=False)
    zero = np.zeros_like(base["k_new"])
    full = base["table"].shape[1] * 16
    for change, skip in ((dict(len=[5, full - 1, 0]), [1]), (dict(len=[5, -1, 0]), [1])):
        case = dict(base, **change)
        d = Dev8(A, case)
        d.worker.append(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE
        check_append8(case, d, case["k_new"], zero, skip=skip)
    for acc in ([0, 3, 0, 1], [0, -1, 0, 1]):
        d = Dev8(A, base)
        d.worker.append(d.kv, d.tok, None, ints([0, 2, 3, 4]), ints(acc))
        assert d.worker.status() == A.ERR_STATE
        check_append8(base, d, base["k_new"], zero, [0, 2, 3, 4], acc, skip=[0])
    for bad in (-1, len(base["k"]), 2 ** 31 - 1, -2 ** 31):
        table = base["table"].copy()
        table[1, 1] = bad
        case = dict(base, table=table)
        d = Dev8(A, case)
        d.worker.append(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
        check_append8(case, d, case["k_new"], zero)


def test_append8_many_requests(A):  # noqa: F811
    n = 1024
    rng = np.random.default_rng(1)
    case = make8("bf16", 2, 1, 64, 16, rng.integers(0, 40, n).tolist(), rng.integers(0, 4, n).tolist(), trees=False)
    freq = 10000.0 ** (-np.arange(32) / 32)
    d = Dev8(A, case)
    d.worker.append(d.kv, d.tok, rope_of(A, freq, "half"))
    check_append8(case, d, *keys8(case, freq, "half"))


# ---------------------------------------------------------------------------------------------------------
# the operators together

@pytest.mark.parametrize("drafted", [1, 5])
def test_a_step_of_all(A, drafted):  # noqa: F811
    """Prompts enter the cache, then steps of rotate, attend and append, eager and from a captured graph: each agrees
    with the definitions on what the cache held before it, and the two with each other."""
    import torch
    kind, hq, hk, dim, page, block = "bf16", 8, 2, 64, 32, 16
    rng = np.random.default_rng(2)
    freq, scale = A.aladdin_rope_frequencies(dim, 10000.0, A.ROPE_PARTS, 4.0, 2048.0)
    rope = A.make_rope(dim, scaling="parts", factor=4.0, original=2048)
    prompt = make8(kind, hq, hk, dim, page, [0, 0, 0], [70, 1, 200], block, trees=False, room=260)
    states = [Dev8(A, prompt) for _ in range(2)]
    for d in states:
        d.worker.append(d.kv, d.tok, rope)
    n = 3 * drafted
    parent = np.concatenate([[-1] + rng.integers(0, np.arange(1, drafted)).tolist() for _ in range(3)]).astype(np.int32)
    off = torch.arange(4, dtype=torch.int32, device="cuda") * drafted
    paths = []
    for r in range(3):
        t, path = drafted - 1, []
        while t >= 0:
            path.insert(0, t)
            t = parent[r * drafted + t]
        paths.append(path)
    acc_off = torch.tensor(np.concatenate([[0], np.cumsum([len(p) for p in paths])]), dtype=torch.int32, device="cuda")
    acc = torch.tensor(np.concatenate(paths), dtype=torch.int32, device="cuda")
    new = torch.randn(n, hq + 2 * hk, dim, device="cuda").to(torch.bfloat16)

    def step(d, x, worker):
        tok = A.make_tokens(off, x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:], torch.from_numpy(parent).cuda() if d.p is None else d.p)
        q, k = worker.rotate(rope, tok, d.next)
        tok = A.make_tokens(off, q, k, x[:, hq + hk:], d.p)
        out = worker.attend(d.kv, tok)
        worker.append(d.kv, tok, None, acc_off, acc)
        return q, k, out

    for d in states:
        d.p = torch.from_numpy(parent).cuda()
    x = new.clone()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        worker = A.Worker(kind, hq, hk, dim, page)
        with torch.cuda.graph(g, stream=side):
            captured = step(states[1], x, worker)
    torch.cuda.synchronize()
    for i in range(4):
        x.copy_(torch.randn(n, hq + 2 * hk, dim, generator=torch.Generator("cuda").manual_seed(i), device="cuda"))
        d = states[0]
        case = dict(prompt, len=d.len.tolist(), next=d.next.tolist(), off=np.arange(4) * drafted, parent=parent,
                    k=d.codes["k"].cpu().numpy(), v=d.codes["v"].cpu().numpy(), k_scale=d.k_scale.cpu().numpy(), v_scale=d.v_scale.cpu().numpy())
        q, k, (out, lse) = step(d, x, d.worker)
        case.update(q=f64(q), k_new=f64(k), v_new=f64(x[:, hq + hk:]))
        check_attend8(case, out, lse)
        check_append8(case, d, case["k_new"], np.zeros_like(case["k_new"]), acc_off.tolist(), acc.tolist())
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        torch.cuda.synchronize()
        for a, b in ((captured[0], q), (captured[1], k), (captured[2][0], out), (captured[2][1], lse), (states[1].codes["k"], d.codes["k"]),
                     (states[1].codes["v"], d.codes["v"]), (states[1].len, d.len), (states[1].next, d.next)):
            assert torch.equal(a, b)
    assert states[0].worker.status() == 0 and worker.status() == 0
