"""Rotation and appending: tokens without a request, and the paths that only large calls take. Tolerances: those of
test_gpu_worker_rope.py and test_gpu_worker_cache8.py."""
import math

import numpy as np
import pytest

import worker8_ref as ref8
from test_gpu_worker import A, Dev, f64, make, rounded  # noqa: F401
from test_gpu_worker_rope import check_rotated, rope_of

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
