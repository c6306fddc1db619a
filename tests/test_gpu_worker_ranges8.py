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
