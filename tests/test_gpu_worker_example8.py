"""The worker of examples/worker_step.py with rotary positions and a cache of 8 bits."""
import os
import sys

import pytest

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


@pytest.mark.parametrize("rotary,cache", [(True, 16), (False, 8), (True, 8)])
def test_steps_of_trees(example, rotary, cache):
    """Every step the requests grow by the tokens that they gained, in cache and position."""
    lengths = [40, 0, 16, 77]
    w = example.ServingWorker(lengths, q_heads=8, kv_heads=2, dim=64, page=16, vocab=97, seed=5, rotary=rotary, cache=cache)
    assert w.length.tolist() == w.next_pos.tolist() == lengths
    total = list(lengths)
    for drafted in (1, 5, 7):
        for r, (new, probs) in enumerate(w.step(drafted)):
            total[r] += len(new)
            assert len(new) >= 1 and all(p <= 0 for p in probs)
        assert w.length.tolist() == w.next_pos.tolist() == total
    assert w.worker.status() == 0
    if cache == 8:
        with pytest.raises(ValueError, match="weights"):
            w.limit(10)


def test_rotary_positions_matter(example):
    """The same tokens at other positions have other probabilities; without rotary positions they have not."""
    for rotary in (False, True):
        seen = []
        for shift in (0, 1000):
            w = example.ServingWorker([30, 50], q_heads=8, kv_heads=2, dim=64, page=16, vocab=97, seed=5, rotary=rotary, cache=8)
            w.next_pos += shift
            seen.append([probs for _, probs in w.step()])
        assert (seen[0] != seen[1]) == rotary


def test_the_program_runs(example, capsys):
    tokens, (k2, c2, c3), place = example.main(["--requests", "8", "--steps", "3", "--workers", "4", "--rotary", "--cache", "8"])
    assert tokens >= 24 and k2 + c2 + c3 > 0
    assert len(place) == 64 and "placed" in capsys.readouterr().out
