"""The cache of 8 bits at the ends of what its calls allow: scales, weights and values of very different size, what is not
finite, and paths of appending that only large calls take. Tolerances: those of test_gpu_worker_cache8.py where a test
does not say otherwise."""
import math

import numpy as np
import pytest

import worker8_ref as ref8
from test_gpu_worker import A, f64, rounded  # noqa: F401
from test_gpu_worker_cache8 import U, Dev8, check_attend8, make8

pytestmark = pytest.mark.gpu

FEW_MANY = [(4, [3, 2]), (32, [30, 20])]  # query heads and new tokens that the kernel of few (many) rows serves


@pytest.mark.parametrize("q_heads,toks", FEW_MANY)
def test_attend8_small_key_scales(A, q_heads, toks):  # noqa: F811
    """Keys of 2^-101 under scales of 2^-110 and queries of 2^100: scores of order one. A scale of 0: scores of 0."""
    case = make8("bf16", q_heads, 2, 64, 16, [100, 40], toks)
    case["q"] = case["q"] * 2.0 ** 100
    case["k_new"] = case["k_new"] * 2.0 ** -100
    case["k_scale"] = case["k_scale"] * np.float32(2.0 ** -100)
    d = Dev8(A, case)
    check_attend8(case, *d.worker.attend(d.kv, d.tok))
    case["k_scale"][case["table"][0, 1]] = 0.0
    d = Dev8(A, case)
    check_attend8(case, *d.worker.attend(d.kv, d.tok))


@pytest.mark.parametrize("q_heads,toks", FEW_MANY)
@pytest.mark.parametrize("held", [1, 16, 100])
def test_attend8_infinite_key_scales(A, q_heads, toks, held):  # noqa: F811
    """A key scale that is not finite makes the rows of its head and request not finite, also where all of its block's
    products with the queries are negative."""
    import torch
    case = make8("bf16", q_heads, 2, 64, 16, [held, 40], toks)
    case["q"] = -np.abs(case["q"])
    case["k"] = np.where(case["k"] & 127 == 127, case["k"], case["k"] & 127)  # keys > 0
    good = Dev8(A, case)
    want, want_lse = good.worker.attend(good.kv, good.tok)
    for x in (math.inf, math.nan):
        d = Dev8(A, case)
        d.k_scale[int(case["table"][0, 0]), 1, 0] = x
        out, lse = d.worker.attend(d.kv, d.tok)
        bad = torch.zeros_like(out, dtype=torch.bool)
        bad[:toks[0], q_heads // 2:] = True
        assert not out[bad].isfinite().any() and not lse[bad[..., 0]].isfinite().any()
        assert torch.equal(out[~bad], want[~bad]) and torch.equal(lse[~bad[..., 0]], want_lse[~bad[..., 0]])


# ---------------------------------------------------------------------------------------------------------
# Scales of values of any size. A weight's rounding counts against the largest product of a weight and its value's scale in
# the row, not against the largest scale of all.

def largest_parts(case):
    """By row and query head, the largest weight times its block's scale (of a new token: times 2^-14 of its largest value),
    and how many keys it has."""
    k, v, q = ref8.dequantised(case, "k"), ref8.dequantised(case, "v"), case["q"]
    hk = k.shape[1]
    grp = q.shape[1] // hk
    block = case["page"] // case["v_scale"].shape[2]
    best, lse = np.zeros(q.shape[:2]), ref8.attend8(case)[1]
    for r, held in enumerate(case["len"]):
        lo, hi = case["off"][r], case["off"][r + 1]
        i = np.arange(held)
        pg, sl = case["table"][r][i // case["page"]], i % case["page"]
        parent = np.arange(hi - lo) - 1 if case["parent"] is None else case["parent"][lo:hi]
        for h in range(q.shape[1]):
            e = case["v_scale"][pg, h // grp, sl // block].astype(np.float64)
            s = q[lo:hi, h] @ k[pg, h // grp, sl].T * case["scale"]
            new = q[lo:hi, h] @ case["k_new"][lo:hi, h // grp].T * case["scale"]
            en = np.abs(case["v_new"][lo:hi, h // grp]).max(1, initial=0.0) * 2.0 ** -14
            for t in range(hi - lo):
                x = np.exp(s[t] - lse[lo + t, h]) * e
                sees = [t]
                while parent[sees[-1]] >= 0:
                    sees.append(parent[sees[-1]])
                y = np.exp(new[t, sees] - lse[lo + t, h]) * en[sees]
                best[lo + t, h] = max(x.max(initial=0.0), y.max())
    return best


def expected(case):
    """(out, its tolerance, lse). As check_attend8, but below 2^-21 of the largest part weights have a step of 2^-31 of it (2^-14 and 2^-24 with a room of
    2^7 above the reference, which may be 2^4 ahead of or 2^8 behind it), half of it for every key, whose value is below 2^9
    scales (a new token's 2^15)."""
    want, want_lse = ref8.attend8(case)
    mag = ref8.attend8(dict(case, v=case["v"] & 127, v_new=np.abs(case["v_new"])))[0]
    tol = U[case["kind"]] * np.abs(want) + (2.0 ** -11 + 2e-4) * mag
    tol = tol + (2.0 ** -32 * (max(case["len"]) * 2.0 ** 9 + 64 * 2.0 ** 15) * largest_parts(case))[..., None]
    tol = tol + (2.0 ** -25 if case["kind"] == "f16" else 2.0 ** -126)
    return want, tol, want_lse


def check_ranges(case, out, lse, want=None):
    want, tol, want_lse = want or expected(case)
    got, got_lse = f64(out), f64(lse)
    assert np.isfinite(got).all()
    d = np.abs(got - want)
    assert np.all(d <= tol), (d / tol).max()
    d = np.abs(got_lse - want_lse)
    assert np.all(d <= 1e-4 + 2.0 ** -21 * np.abs(want_lse)), d.max()


def steered(kind, q_heads, toks, lens, block=16, seed=0):
    """A case whose keys score by their first channel alone: `score`, in powers of two against 0; new tokens score `score_new`
    in the same way."""
    case = make8(kind, q_heads, 2, 64, 64, lens, toks, block, seed=seed)
    case["scale"] = math.log(2.0)
    case["q"][:] = 0.0
    case["q"][:, :, 0] = 1.0
    case["k_new"][:] = 0.0
    for name in ("k", "v"):
        case[name + "_scale"][:] = 1.0
    case["k"][:] = 0
    case["v"][:] = 127
    return case


def put(case, r, i, name, value):
    """Cached tokens i of request r: codes of `value`, all heads."""
    i = np.asarray(i)
    case[name][case["table"][r][i // case["page"]], :, i % case["page"]] = ref8.code(value)


def set_scale(case, r, i, name, value):
    """The scale of the blocks that tokens i of request r lie in, all heads."""
    i = np.asarray(i)
    block = case["page"] // case["v_scale"].shape[2]
    case[name + "_scale"][case["table"][r][i // case["page"]], :, i % case["page"] // block] = value


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,toks", FEW_MANY)
@pytest.mark.parametrize("apart", [12, 24, 40, 100])
@pytest.mark.parametrize("where", ["first", "last", "between"])
def test_attend8_large_scale_without_weight(A, kind, q_heads, toks, apart, where):  # noqa: F811
    """A block whose values' scale is 2^apart times the others', and whose weights are next to nothing, costs the others no
    bits: weights e^-0.35 and e^-0.7 of the largest and ones below 2^-14 of it, in front of it and behind."""
    case = steered(kind, q_heads, toks, [200, 70])
    rng = np.random.default_rng(apart)
    for r, held in enumerate(case["len"]):
        i = np.arange(held)
        put(case, r, i, "v", rng.uniform(-100, 300, (held, 2, 64)))
        k = np.zeros((held, 2, 64))
        k[:, :, 0] = rng.choice([0.0, -0.5, -1.0, -3.0, -16.0], (held, 1))
        big = {"first": np.arange(16), "last": np.arange(held // 16 * 16, held), "between": np.arange(32, 48)}[where]
        k[big, :, 0] = -448.0
        put(case, r, i, "k", k)
        set_scale(case, r, i, "v", np.float32(2.0 ** (-10 - apart)))
        set_scale(case, r, big, "v", np.float32(2.0 ** -10))
    case["v_new"] = rounded(case["v_new"] * 2.0 ** -max(apart - 8, 0), kind)
    case["k_new"][:, :, 0] = -1.0
    d = Dev8(A, case)
    check_ranges(case, *d.worker.attend(d.kv, d.tok, case["scale"]))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("group,new,requests", [(1, 1, 200), (16, 3, 30)])
@pytest.mark.parametrize("gap,scale", [(26, 1.0), (14, 4096.0), (28, 1.0), (30, 0.125)])
def test_attend8_long_flat_tail(A, kind, group, new, requests, gap, scale):  # noqa: F811
    """Thousands of keys far below a peak whose own value is next to nothing, in units that a worker has whole (requests that
    read the same pages): what the keys hold of the sum reaches the output. The peak's block has `scale` times the others' scale."""
    import torch
    held, heads = 3000, 16
    case = make8(kind, heads * group, heads, 64, 64, [held], [new], 16, trees=False)
    case["q"][:] = 0.0
    case["q"][:, :, 0] = 0.25
    case["k_new"][:] = 0.0
    case["k_new"][:, :, 0] = -400.0
    case["scale"] = math.log(2.0)
    k, v = np.zeros((held, heads, 64)), np.full((held, heads, 64), 300.0)
    k[:, :, 0] = -4.0 * gap
    k[777, :, 0], v[777], v[777, :, 0] = 0.0, 0.0, 2.0 ** -6
    for name, x in (("k", k), ("v", v)):
        put(case, 0, np.arange(held), name, x)
        case[name + "_scale"][:] = 1.0
    set_scale(case, 0, [777], "v", np.float32(scale))
    d = Dev8(A, case)
    off = torch.arange(requests + 1, dtype=torch.int32, device="cuda") * new
    kv = A.make_kv8(d.k, d.v, d.k_scale, d.v_scale, d.table.repeat(requests, 1), d.len.repeat(requests))
    tok = A.make_tokens(off, *(x.repeat(requests, 1, 1) for x in (d.q, d.k_new, d.v_new)))
    out, lse = d.worker.attend(kv, tok, case["scale"])
    want = expected(case)
    for r in range(requests):
        check_ranges(case, out[r * new:(r + 1) * new], lse[r * new:(r + 1) * new], want)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,dim,toks", [(4, 64, [3, 1, 2]), (2, 96, [1, 1, 1]), (2, 128, [4, 2, 1]), (4, 256, [1, 2, 1]),
                                              (32, 64, [30, 9, 20]), (8, 96, [40, 30, 2]), (16, 128, [30, 64, 20]), (32, 256, [20, 7, 9])])
@pytest.mark.parametrize("most", [20, 100])
def test_attend8_scales_of_any_size(A, kind, q_heads, dim, toks, most):  # noqa: F811
    """Blocks whose values' scales lie anywhere from 2^-most to 2^most, some of them 0 under codes that are not, new values
    likewise; scores of up to 100 apart."""
    lens = [300, 33, 0]
    case = make8(kind, q_heads, 2, dim, 64, lens, toks, 16, seed=most)
    rng = np.random.default_rng(most)
    shape = case["v_scale"].shape
    far = 2.0 ** rng.integers(-most, most + 1, shape) * (rng.random(shape) < 0.8)
    case["v_scale"] = np.where(np.isnan(case["v_scale"]), np.nan, far).astype(np.float32)
    case["q"] = rounded(case["q"] * 4.0, kind)
    reach = 15 if kind == "f16" else most
    case["v_new"] = rounded(case["v_new"] * (2.0 ** rng.integers(-reach, reach - 3, case["v_new"].shape[:2]))[..., None], kind)
    if kind == "f16":  # (results within the type's range)
        case["v_scale"] = case["v_scale"] * np.float32(2.0 ** -(most + 6))
    d = Dev8(A, case)
    check_ranges(case, *d.worker.attend(d.kv, d.tok, case["scale"]))


@pytest.mark.parametrize("q_heads,toks", FEW_MANY)
def test_attend8_smallest_scales(A, q_heads, toks):  # noqa: F811
    """Values under the smallest scale of all, and scales of 0 alone; new values of any size next to them."""
    case = make8("bf16", q_heads, 2, 64, 16, [100, 40], toks)
    case["v_scale"] = np.where(np.isnan(case["v_scale"]), np.nan, 2.0 ** -126).astype(np.float32)
    for size in (1.0, 2.0 ** -100, 2.0 ** -118, 0.0):
        c = dict(case, v_new=rounded(case["v_new"] * size, "bf16"))
        d = Dev8(A, c)
        check_ranges(c, *d.worker.attend(d.kv, d.tok))
    case["v_scale"] = case["v_scale"] * 0
    for size in (1.0, 2.0 ** -118, 0.0):
        c = dict(case, v_new=rounded(case["v_new"] * size, "bf16"))
        d = Dev8(A, c)
        check_ranges(c, *d.worker.attend(d.kv, d.tok))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,toks", FEW_MANY)
def test_attend8_large_values_out_of_sight(A, kind, q_heads, toks):  # noqa: F811
    """A new token whose values are 2^24 times the others' costs the rows that do not see it, and those for which it has no
    weight, no bits."""
    case = make8(kind, q_heads, 2, 64, 16, [100, 40], toks)
    case["parent"][:toks[0]] = -1
    case["parent"][2] = 1
    case["v_scale"] = (case["v_scale"] * 2.0 ** -12).astype(np.float32)
    case["v_new"] = rounded(case["v_new"] * 2.0 ** -10, kind)
    case["v_new"][1] = rounded(np.sign(case["v_new"][1]) * 2.0 ** 15, kind)  # seen by tokens 1 and 2
    case["q"][2] = rounded(np.abs(case["q"][2]), kind)
    case["k_new"][1] = -64.0                                                 # which token 2 gives no weight
    case["q"][1] = 0.0
    d = Dev8(A, case)
    check_ranges(case, *d.worker.attend(d.kv, d.tok, case["scale"]))


# ---------------------------------------------------------------------------------------------------------
# Values of new tokens that are not finite.

@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("q_heads,dim,toks,held", [(4, 64, [3, 2], 20), (2, 128, [20, 3], 3), (2, 256, [14, 1], 0), (4, 96, [2, 3], 2000),
                                                   (32, 64, [30, 20], 20), (16, 128, [40, 9], 0), (32, 96, [30, 9], 2000), (16, 256, [30, 4], 40)])
@pytest.mark.parametrize("below", [0, 200])
def test_attend8_values_that_are_not_finite(A, kind, q_heads, dim, toks, held, below):  # noqa: F811
    """They make their channel what they are in the rows that see them, also where their weight is e^-200, and nothing in
    other rows and channels."""
    case = make8(kind, q_heads, 2, dim, 64, [held, 17], toks)
    case["parent"][:] = np.concatenate([np.arange(t) - 1 for t in toks])  # chains: what comes later sees it
    case["q"] = rounded(np.abs(case["q"]) + 0.5, kind)
    at = toks[0] + 1 if len(toks) < 2 else 1
    finite = case["v_new"].copy()
    finite[at, 0, [3, 40]] = finite[at, 1, 7] = 0.0
    case["v_new"] = finite
    if below:
        # a score at least 200 below any other: those of the rest are within 40
        case["k_new"][at] = rounded(np.full(dim, -1600.0 / dim ** 0.5), kind)
    d = Dev8(A, case)
    want, want_lse = (f64(x) for x in d.worker.attend(d.kv, d.tok))
    scores = np.einsum("thgd,hd->thg", case["q"].reshape(len(want), 2, -1, dim), case["k_new"][at]) * case["scale"]
    assert not below or (scores[at:toks[0]].reshape(toks[0] - at, -1) - want_lse[at:toks[0]]).max() < -150
    bad = case["v_new"].copy()
    bad[at, 0, 3], bad[at, 0, 40], bad[at, 1, 7] = math.inf, math.nan, -math.inf
    d = Dev8(A, dict(case, v_new=bad))
    got, lse = (f64(x) for x in d.worker.attend(d.kv, d.tok))
    g = q_heads // 2
    seen = slice(at, toks[0])
    want[seen, :g, 3], want[seen, :g, 40], want[seen, g:, 7] = math.inf, math.nan, -math.inf
    np.testing.assert_array_equal(got, want)
    np.testing.assert_array_equal(lse, want_lse)


@pytest.mark.parametrize("q_heads,toks", [(4, [2, 1]), (32, [30, 2])])
def test_attend8_no_score_and_no_value(A, q_heads, toks):  # noqa: F811
    """A row whose scores are all -inf has no result, whatever the values."""
    case = make8("f16", q_heads, 2, 64, 16, [0, 20], toks)
    case["q"] = rounded(np.abs(case["q"]) + 0.1, "f16")
    case["k_new"][0] = -math.inf
    case["v_new"][0, :, 3] = math.inf
    case["parent"][:toks[0]] = -1
    d = Dev8(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()
    assert out[1:].isfinite().all()
