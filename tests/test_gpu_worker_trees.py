"""The attention of many rows a key head (trees of drafted tokens, large groups) where test_gpu_worker.py does not
take it: maxima that grow, two row tiles in every type and dimension, refusals, masked and infinite values. The
tolerances are that file's; with a larger scale the scores' error, and what it does to out, grows with it."""
import numpy as np
import pytest

import worker_ref as ref
from test_gpu_worker import A, Dev, U, check_attend, f64, make, rounded  # noqa: F401  (A is a fixture)

pytestmark = pytest.mark.gpu


def rows_mean(case, hq, hk):
    return len(case["q"]) * (hq // hk) / len(case["len"])


GROW = [  # kind, query heads, key heads, dim, lengths, new tokens: one row tile, then two
    ("bf16", 8, 2, 64, [700, 0, 300], [20, 9, 12]), ("f16", 8, 2, 96, [700, 0, 300], [20, 9, 12]),
    ("f16", 8, 2, 128, [700, 0, 300], [20, 9, 12]), ("bf16", 8, 2, 256, [700, 0, 300], [20, 9, 12]),
    ("f16", 8, 1, 64, [700, 130], [40, 17]), ("bf16", 8, 1, 96, [700, 130], [40, 17]),
    ("bf16", 8, 1, 128, [700, 130], [40, 17]),
]


@pytest.mark.parametrize("kind,hq,hk,dim,lens,toks", GROW)
def test_maximum_grows_from_tile_to_tile(A, kind, hq, hk, dim, lens, toks):
    """Keys that get longer towards a request's end: a row's maximum rises by more than 2^8 over the one that
    its accumulator refers to, several times."""
    case = make(kind, hq, hk, dim, 32, lens, toks, seed=dim)
    assert rows_mean(case, hq, hk) > 16
    scale = case["scale"] = 3.0 * dim ** -0.5
    for r, n in enumerate(lens):
        pg, sl = ref.slots(case, r, n)
        grow = (0.05 + 0.01 * np.arange(n) / max(n, 1) * 200)[:, None, None]
        case["k"][pg, :, sl] = rounded(case["k"][pg, :, sl] * grow, kind)
    # it does: the maxima of the first request's rows over tiles of 128 keys (64 for 256 channels)
    pg, sl = ref.slots(case, 0, lens[0])
    grp, kt = hq // hk, 64 if dim == 256 else 128
    s = np.einsum("thd,nhd->thn", case["q"][:toks[0], ::grp], case["k"][pg, :, sl]) * scale * np.log2(np.e)
    tops = np.stack([s[..., i:i + kt].max(-1) for i in range(0, lens[0] // kt * kt, kt)])
    grown = (tops[1:] > np.maximum.accumulate(tops, 0)[:-1] + 8).sum(0)
    assert (grown > 0).mean() > 0.5
    d = Dev(A, case)
    out, lse = d.worker.attend(d.kv, d.tok, scale)
    want, want_lse = ref.attend(case)
    mag = ref.attend(dict(case, v=np.abs(case["v"]), v_new=np.abs(case["v_new"])))[0]
    # keys are up to 2.05 times as long as in the other tests, the scale 3 times
    e, u = 1e-4 * 2.05 * 3.0, U[kind]
    tol = u * np.abs(want) + (u + 2 * e) * mag
    if kind == "f16":
        tol = tol + (max(lens) + 64) * 2.0 ** -25 * np.nanmax(np.abs(case["v"]))
    assert np.all(np.abs(f64(out) - want) <= tol), (np.abs(f64(out) - want) - tol).max()
    assert np.all(np.abs(f64(lse) - want_lse) <= e + 2.0 ** -21 * np.abs(want_lse))
    assert d.worker.status() == A.OK


TWO = [  # two row tiles: more than 128 rows a key head on average
    ("bf16", 8, 1, 64, 16, [100, 0, 129], [64, 33, 20]),
    ("f16", 8, 1, 64, 64, [64, 300], [64, 17]),
    ("bf16", 16, 2, 96, 32, [100, 65], [64, 30]),
    ("f16", 7, 1, 96, 128, [200, 1], [64, 25]),
    ("bf16", 16, 2, 128, 16, [100, 0, 64], [64, 64, 1]),
    ("bf16", 64, 1, 128, 256, [257, 31], [3, 2]),       # a group of half a row tile
    ("f16", 300, 1, 64, 16, [50, 3], [1, 2]),           # one of more than a unit's rows
    ("bf16", 300, 1, 256, 16, [50, 3], [1, 2]),
]


@pytest.mark.parametrize("kind,hq,hk,dim,page,lens,toks", TWO)
@pytest.mark.parametrize("rows,fused,trees", [("hnd", True, True), ("nhd", False, False)])
def test_two_row_tiles(A, kind, hq, hk, dim, page, lens, toks, rows, fused, trees):
    case = make(kind, hq, hk, dim, page, lens, toks, seed=hq + dim, trees=trees)
    assert rows_mean(case, hq, hk) > 128
    d = Dev(A, case, rows, fused)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend(case, out, lse)
    again, lse2 = d.worker.attend(d.kv, d.tok)
    assert np.array_equal(f64(out), f64(again)) and np.array_equal(f64(lse), f64(lse2))
    assert d.worker.status() == A.OK


@pytest.mark.parametrize("kind,hq,dim,toks", [("bf16", 8, 64, 64), ("f16", 8, 128, 64), ("bf16", 4, 96, 20)])
def test_long_units_are_split_and_joined(A, kind, hq, dim, toks):
    """One request of many tiles: its units' parts, in both row tiles where there are two, come from many CTAs."""
    case = make(kind, hq, 1, dim, 64, [21003], [toks], seed=11)
    d = Dev(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend(case, out, lse)
    for _ in range(20):
        again, lse2 = d.worker.attend(d.kv, d.tok)
        assert bool((out == again).all()) and bool((lse == lse2).all())
    assert d.worker.status() == A.OK


@pytest.mark.parametrize("kind,hq,dim,toks,lens", [("bf16", 8, 128, [64, 30], [30, 0]), ("f16", 8, 64, [64, 20], [130, 127]),
                                                   ("f16", 8, 96, [40, 33], [100, 0]), ("bf16", 8, 256, [64, 9], [70, 0])])
def test_values_out_of_sight_of_two_row_tiles(A, kind, hq, dim, toks, lens):
    """Infinite and NaN keys and values of new tokens whose rows lie in the first and in the second row tile."""
    case = make(kind, hq, 1, dim, 16, lens, toks, seed=9)
    assert rows_mean(case, hq, 1) > 128
    n = toks[0]
    case["parent"][:n] = [-1, 0, -1, 2, 1, 0] + [2] * (n - 6)
    case["parent"][n - 3:n] = [3, n - 3, 1]  # of the second row tile: below 3, below that, below 1
    case["k_new"][1] = case["v_new"][1] = np.nan
    case["v_new"][3, 0, ::2] = np.inf
    case["v_new"][n - 2, 0, 1::2] = -np.inf
    case["parent"][n:] = [-1, -1, 0] + [0] * (toks[1] - 3)
    case["v_new"][n + 1] = -np.inf
    d = Dev(A, case)
    check_attend(case, *d.worker.attend(d.kv, d.tok))


@pytest.mark.parametrize("hq,hk", [(8, 2), (16, 1)])
def test_scores_of_minus_infinity_in_many_rows(A, hq, hk):
    case = make("f16", hq, hk, 64, 16, [0, 20, 200], [12, 9, 11], seed=3)
    assert rows_mean(case, hq, hk) > (16 if hk == 2 else 128)
    case["q"] = rounded(np.abs(case["q"]) + 0.25, "f16")
    case["k_new"][:12] = -np.inf       # the first request's rows see nothing else
    pg, sl = ref.slots(case, 1, 20)
    case["k"][pg[:13], :, sl[:13]] = -np.inf
    pg, sl = ref.slots(case, 2, 200)   # a whole tile and more of nothing, then something
    case["k"][pg[:150], :, sl[:150]] = -np.inf
    case["k"][pg[150:], 0, sl[150:]] = -np.inf
    case["k_new"][21:, 0] = -np.inf
    d = Dev(A, case)
    out, lse = d.worker.attend(d.kv, d.tok)
    check_attend(case, out, lse)
    assert np.isneginf(f64(lse)[:12]).all() and (f64(out)[:12] == 0).all()


@pytest.mark.parametrize("hq,hk", [(8, 2), (32, 1)])
def test_refused_requests_and_hidden_pages_of_many_rows(A, hq, hk):
    import torch
    lens, toks, dim = [150, 20, 133, 40], [12, 7, 14, 5], 64
    case = make("bf16", hq, hk, dim, 16, lens, toks, seed=6)
    assert rows_mean(case, hq, hk) > (16 if hk == 2 else 128)
    for r, bad in ((0, -1), (1, 10 ** 6), (2, 2 ** 31 - 1)):
        d = Dev(A, case)
        d.len[r] = bad
        out = torch.full((38, hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((38, hq), 7.0, device="cuda")
        d.worker.attend(d.kv, d.tok, out=out, lse=lse)
        assert d.worker.status() == A.ERR_STATE and d.worker.status() == A.OK
        lo, hi = case["off"][r], case["off"][r + 1]
        assert bool((out[lo:hi] == 7).all()) and bool((lse[lo:hi] == 7).all())
        spared = dict(case, len=[0 if i == r else n for i, n in enumerate(lens)])
        check_attend(spared, out, lse, skip=[r])
    for off in ([0, 12, 11, 33, 38], [0, 12, 19, 33, 99], [-3, 12, 19, 33, 38]):
        d = Dev(A, case)
        d.off.copy_(torch.tensor(off, dtype=torch.int32))
        d.worker.attend(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE
    for bad in (-1, case["k"].shape[0], 2 ** 31 - 1, -2 ** 31):
        d = Dev(A, case)
        d.table[0, 1], d.table[0, 8], d.table[2, 0] = bad, bad, bad
        out, lse = d.worker.attend(d.kv, d.tok)
        assert d.worker.status() == A.ERR_STATE
        hidden = dict(case, table=case["table"].copy(), len=[150 - 32, 20, 133 - 16, 40])
        hidden["table"][0, :8] = np.delete(case["table"][0], [1, 8])[:8]
        hidden["table"][2, :8] = case["table"][2, 1:9]
        check_attend(hidden, out, lse)
    d = Dev(A, case)
    d.parent[1], d.parent[37] = 1, -5
    out, lse = d.worker.attend(d.kv, d.tok)
    assert d.worker.status() == A.ERR_STATE
    parent = case["parent"].copy()
    parent[1] = parent[37] = -1
    check_attend(dict(case, parent=parent), out, lse)


def test_pages_more_than_32_bits_apart_with_many_rows(A):
    import torch
    case = make("bf16", 16, 1, 64, 16, [40], [20], seed=8, spare=0)
    far, n = (1 << 31) + 64, case["k"].shape[0]
    d = Dev(A, case)
    big = []
    for x in (d.k, d.v):
        y = torch.empty((n - 1) * far + 16 * 64, dtype=torch.bfloat16, device="cuda")
        y = y.as_strided((n, 1, 16, 64), (far, 16 * 64, 64, 1))
        y.copy_(x)
        big.append(y)
    out, lse = d.worker.attend(A.make_kv(big[0], big[1], d.table, d.len), d.tok)
    check_attend(case, out, lse)
    assert d.worker.status() == A.OK
