"""The example's worker under a budget wider than its window of recent positions: what leaves the cache is decided by
the accumulated weights."""
import os
import sys

import numpy as np
import pytest

import worker_ref as ref

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.init()
    from paper_2405_06856_gb300 import build
    build.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import worker_step
    return worker_step


def test_least_weights_leave_and_recent_positions_stay(example):
    budget, recent, page, heads = 60, 16, 16, 2
    w = example.ServingWorker([100, 5, 64], q_heads=4, kv_heads=heads, dim=64, page=page, vocab=64, seed=2)
    w.limit(budget, recent)
    evict, seen = w.worker.evict, []

    def state():
        f = lambda x: x.double().cpu().numpy()
        return dict(page=page, table=w.table.cpu().numpy(), k=f(w.k), v=f(w.v), weight=w.weight.cpu().numpy(),
                    pos=w.pos.cpu().numpy(), len=w.length.tolist(), next=w.next_pos.tolist())

    def watched(kv, b, r):
        before = state()
        evict(kv, b, r)
        seen.append((before, state(), b.tolist(), r))

    w.worker.evict = watched
    for _ in range(8):
        w.step(4)
    assert len(seen) == 8 and w.worker.status() == 0
    by_weight = 0
    for before, after, b, r in seen:
        assert r == recent
        want = ref.evict(before, b, r)
        assert after["len"] == want[4]
        for q, n in enumerate(want[4]):
            pg, sl = ref.slots(after, q, n)
            for name, x in zip(("k", "v", "weight", "pos"), want):
                assert np.array_equal(after[name][pg, :, sl], x[pg, :, sl])
            for h in range(heads):
                pos = set(after["pos"][pg, h, sl].tolist())
                last = set(range(max(0, after["next"][q] - recent), after["next"][q]))
                assert len(pos) == n and last <= pos
                by_weight += before["len"][q] > budget and pos != set(range(after["next"][q] - n, after["next"][q]))
    assert by_weight >= 2 * heads  # requests that hold something other than their last positions
