"""Rotation and appending: tokens without a request, and the paths that only large calls take. Tolerances: those of
test_gpu_worker_rope.py and test_gpu_worker_cache8.py."""
import math

import numpy as np
import pytest

import worker8_ref as ref8
from test_gpu_worker import A, Dev, f64, make, rounded  # noqa: F401
from test_gpu_worker_cache8 import Dev8, check_append8, keys8, make8
from test_gpu_worker_rope import check_append, check_rotated, keys_at, rope_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("offsets", [[0], [0, 0, 0], [2, 5], None])
def test_rotate_by_positions_alone(A, offsets):  # noqa: F811
    """With given positions the requests are not read: there may be none, they may leave tokens out, and the
    offsets may be missing."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [0], [9], trees=False)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(32) / 32)
    pos = np.arange(9) * 1000 + 7
    where = torch.from_numpy(pos.astype(np.int32)).cuda()
    fill = lambda: dict(q_out=torch.full_like(d.q, 9.0), k_out=torch.full_like(d.k_new, 9.0))
    tok = A.make_tokens(torch.tensor(offsets or [0], dtype=torch.int32, device="cuda"), d.q, d.k_new, d.v_new)
    if offsets is None:
        tok.off = None
    q, k = d.worker.rotate(rope_of(A, freq, "half"), tok, None, where, **fill())
    assert d.worker.status() == 0
    check_rotated(f64(q), case["q"], pos, freq, "half", 1.0, "bf16")
    check_rotated(f64(k), case["k_new"], pos, freq, "half", 1.0, "bf16")


def test_rotate_padding(A):  # noqa: F811
    """Tokens that no request has stay out where positions come from the requests."""
    import torch
    case = make("bf16", 4, 2, 64, 16, [0], [9], trees=False)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(32) / 32)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, k = torch.full_like(d.q, 9.0), torch.full_like(d.k_new, 9.0)
    d.worker.rotate(rope_of(A, freq, "half"), A.make_tokens(ints([2, 5, 7]), d.q, d.k_new, d.v_new), ints([100, 50]), q_out=q, k_out=k)
    assert d.worker.status() == 0
    check_rotated(f64(q[2:7]), case["q"][2:7], np.array([100, 101, 102, 50, 51]), freq, "half", 1.0, "bf16")
    check_rotated(f64(k[2:7]), case["k_new"][2:7], np.array([100, 101, 102, 50, 51]), freq, "half", 1.0, "bf16")
    for x in (q, k):
        assert (x[:2] == 9.0).all() and (x[7:] == 9.0).all()
    with pytest.raises(A.AladdinError):  # without positions the offsets are needed
        tok = A.make_tokens(ints([0, 9]), d.q, d.k_new, d.v_new)
        tok.off = None
        d.worker.rotate(rope_of(A, freq, "half"), tok, q_out=q, k_out=k)
    none = A.make_tokens(ints([0]), d.q, d.k_new, d.v_new)
    q.fill_(9.0)
    d.worker.rotate(rope_of(A, freq, "half"), none, q_out=q, k_out=False)
    assert (q == 9.0).all() and d.worker.status() == 0


# ---------------------------------------------------------------------------------------------------------
# append8, a token at a time

@pytest.mark.parametrize("kind,heads,dim,block", [("bf16", 8, 128, 16), ("f16", 3, 64, 64), ("bf16", 2, 96, 32), ("f16", 2, 256, 16)])
def test_append8_scales_that_grow(A, kind, heads, dim, block):  # noqa: F811
    """A token a call to each of many requests, each twice as large as the one before it: every call rounds what the
    block holds again, under the scale that it had."""
    import torch
    n, steps = 60, 9
    case = make8(kind, heads, heads, dim, 64, [(7 * r) % 50 for r in range(n)], [steps] * n, block, trees=False)
    grow = np.tile(2.0 ** np.arange(steps), n)[:, None, None]
    for name in ("k_new", "v_new"):
        case[name] = rounded(np.sign(case[name]) * np.clip(np.abs(case[name]), 0.1, 1.0) * grow, kind)
    d = Dev8(A, case)
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    for i in range(steps):
        x = torch.arange(n, device="cuda") * steps + i
        d.worker.append(d.kv, A.make_tokens(off, None, d.k_new[x], d.v_new[x]))
    assert d.worker.status() == 0 and d.len.tolist() == [l + steps for l in case["len"]]
    now = dict(case)
    for i in range(steps):  # (one request after the other, a token at a time)
        step = dict(now, len=[l + i for l in case["len"]], off=np.arange(n + 1), k_new=case["k_new"][i::steps], v_new=case["v_new"][i::steps])
        now.update(ref8.append8(step, step["k_new"]))
    nan = lambda c: np.where(c & 127 == 127, 127, c)
    for name in ("k", "v"):
        np.testing.assert_array_equal(getattr(d, name + "_scale").cpu().numpy(), now[name + "_scale"].astype(np.float32))
        np.testing.assert_array_equal(nan(d.codes[name].cpu().numpy()), nan(now[name]))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("grow", [False, True])
def test_append8_under_scales_of_another_origin(A, kind, grow):  # noqa: F811
    """Held scales that are no powers of two: new values, many of them in the middle between two codes, are rounded once, and
    so are the held codes under a scale that grows."""
    odd = [3.0, 5.0, 7.0] + [float(np.float32(t / z)) for t in (9, 11, 13, 15, 17, 19, 21, 23, 25, 27, 29, 31) for z in (9, 10, 11, 13, 14, 15)]
    scales = np.array([s for s in odd if math.frexp(s)[0] != 0.5], np.float32) * np.float32(2.0 ** -9)
    n = len(scales)
    case = make8(kind, 2, 2, 64, 16, [5] * n, [6] * n, 16, trees=False)
    rng = np.random.default_rng(n)
    ties = np.concatenate([(ref8.VALUES[40:120] + ref8.VALUES[41:121]) / 2, ref8.VALUES[30:126]])
    for name in ("k", "v"):
        for r, s in enumerate(scales):
            p = case["table"][r][0]
            case[name + "_scale"][p] = s
            case[name][p, :, :5] = rng.integers(0, 127, (2, 5, 64)) + 128 * rng.integers(0, 2, (2, 5, 64))
            x = rng.choice(ties, (6, 2, 64)) * rng.choice([-1.0, 1.0], (6, 2, 64)) * float(s)
            if grow:
                x[0, :, 0] = 448.0 * 4 * 2.0 ** math.ceil(math.log2(float(s)))
            case[name + "_new"][r * 6:(r + 1) * 6] = rounded(x, kind)
    d = Dev8(A, case)
    d.worker.append(d.kv, d.tok)
    assert d.worker.status() == 0
    want = ref8.append8(case, case["k_new"])
    nan = lambda c: np.where(c & 127 == 127, 127, c)
    for name in ("k", "v"):
        np.testing.assert_array_equal(getattr(d, name + "_scale").cpu().numpy(), want[name + "_scale"].astype(np.float32))
        np.testing.assert_array_equal(nan(d.codes[name].cpu().numpy()), nan(want[name]))


# ---------------------------------------------------------------------------------------------------------
# Prompts: more units than the GPU has warps, several turns of every loop.

@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,q_heads,kv_heads,dim,turn", [("bf16", 40, 8, 64, 64), ("f16", 12, 4, 256, 256), ("bf16", 28, 4, 96, 64), ("f16", 64, 8, 128, 20)])
@pytest.mark.parametrize("place", [False, True])
def test_rotate_prompts(A, kind, q_heads, kv_heads, dim, turn, layout, place):  # noqa: F811
    """A warp has a token's rows in several turns."""
    import torch
    toks = [1250, 0, 1, 77]
    case = make(kind, q_heads, kv_heads, dim, 16, [0] * 4, toks, trees=False)
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    start = np.array([5000, 3, 0, 100000])
    pos = np.repeat(start, toks) + ref8.depths(case["off"], None)
    outs = dict(q_out=d.q, k_out=d.k_new) if place else {}
    q, k = d.worker.rotate(rope_of(A, freq, layout), d.tok, torch.from_numpy(start.astype(np.int32)).cuda(), **outs)
    assert d.worker.status() == 0
    check_rotated(f64(q), case["q"], pos, freq, layout, 1.0, kind)
    check_rotated(f64(k), case["k_new"], pos, freq, layout, 1.0, kind)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,heads,dim,turn,page", [("bf16", 1, 64, 64, 16), ("f16", 8, 256, 256, 64), ("bf16", 12, 128, 96, 32), ("f16", 5, 96, 58, 128)])
@pytest.mark.parametrize("rotated", [True, False])
def test_append_prompts(A, kind, heads, dim, turn, page, layout, rotated):  # noqa: F811
    """A warp has several units, turned on from one to the next across pages and requests, and a unit's heads in several turns;
    a page outside the pool among them."""
    toks = [3001, 0, 1, 2500, 64, 3200]
    case = make(kind, heads, heads, dim, page, [5, 100, 16, 0, 31, 900], toks, trees=False)
    case["next"] = [l + 70000 * r for r, l in enumerate(case["len"])]
    case["table"][3, 700 // page] = -1
    d = Dev(A, case)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    d.worker.append(d.kv, d.tok, rope_of(A, freq, layout) if rotated else None)
    assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
    if rotated:
        check_append(case, d, *keys_at(case, freq, layout, kind))
    else:
        check_append(case, d, case["k_new"], np.zeros_like(case["k_new"]))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,heads,dim,turn,page,block,tokens", [
    ("bf16", 4, 64, 64, 16, 16, 40000),    # a warp a block, several rows of heads a unit
    ("f16", 2, 256, 40, 64, 16, 20500),    # four warps a block
    ("bf16", 3, 128, 128, 128, 64, 27000)])  # eight
def test_append8_prompts(A, kind, heads, dim, turn, page, block, tokens, layout):  # noqa: F811
    """Several rows of heads a unit, several units a group of warps one after the other; infinities and NaN among them, which
    one warp of several meets, and a page outside the pool."""
    toks = [tokens // 2, 1, 0, tokens - tokens // 2]
    case = make8(kind, heads, heads, dim, page, [block + 3, 7, 20, 0], toks, block, trees=False)
    case["next"] = [l + 70000 * r for r, l in enumerate(case["len"])]
    rng = np.random.default_rng(dim)
    for name in ("k_new", "v_new"):
        case[name] *= 2.0 ** rng.integers(-2, 3, (len(case[name]), 1, 1))
        t, h, c = rng.integers(0, tokens, 40), rng.integers(0, heads, 40), rng.integers(0, dim, 40)
        case[name][t, h, c] = rng.choice([math.inf, -math.inf, math.nan], 40)
    case["table"][3, 700 // page] = len(case["k"])
    d = Dev8(A, case)
    freq = 10000.0 ** (-np.arange(turn // 2) / (turn // 2))
    d.worker.append(d.kv, d.tok, rope_of(A, freq, layout))
    assert d.worker.status() == A.ERR_STATE and d.worker.status() == 0
    with np.errstate(invalid="ignore"):
        check_append8(case, d, *keys8(case, freq, layout))
