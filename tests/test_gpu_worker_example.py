"""The worker of examples/worker_step.py: its operators together, as a worker uses them."""
import os
import sys

import numpy as np
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


def test_drafted_trees_give_the_tokens_of_plain_decoding(example):
    """Greedy decoding with trees that hold the right tokens among others gives the tokens of one-by-one
    decoding, in fewer iterations, and the same cache."""
    shape = dict(q_heads=8, kv_heads=2, dim=64, page=16, vocab=97, seed=5)
    lengths = [40, 0, 16, 77]
    plain = example.ServingWorker(lengths, **shape)
    want = [[] for _ in lengths]
    for _ in range(12):
        for r, (new, _) in enumerate(plain.step()):
            want[r] += new
    drafted = example.ServingWorker(lengths, **shape)
    rng = np.random.default_rng(0)
    got = [[] for _ in lengths]

    def drafts(r, n):  # a chain of the next right tokens, one wrong sibling in front of each
        token, parent, at = [], [], 0
        for right in want[r][len(got[r]):]:
            token += [(right + 1 + int(rng.integers(0, 90))) % 97, right]
            parent += [at, at]
            at = len(token)
        token, parent = token[:n], parent[:n]
        while len(token) < n:
            token.append(int(rng.integers(0, 97)))
            parent.append(0)
        return token, parent

    steps = 0
    while min(len(g) for g in got) < 12:
        steps += 1
        assert steps <= 12
        for r, (new, _) in enumerate(drafted.step(7, drafts)):
            got[r] += new
    for r in range(len(lengths)):
        assert got[r][:12] == want[r], r
    assert steps <= 4
    assert drafted.worker.status() == 0 and plain.worker.status() == 0
    # the caches agree over the tokens that both hold
    for r, n in enumerate(plain.length.tolist()):
        m = min(n, int(drafted.length[r]))
        for a, b in ((plain.k, drafted.k), (plain.v, drafted.v), (plain.pos, drafted.pos)):
            i = np.arange(lengths[r], m)
            pa, pb = plain.table[r].cpu().numpy()[i // 16], drafted.table[r].cpu().numpy()[i // 16]
            assert (a[pa, :, i % 16] == b[pb, :, i % 16]).all()


def test_budget_bounds_the_cache(example):
    w = example.ServingWorker([100, 5, 64], q_heads=4, kv_heads=2, dim=64, page=16, vocab=64, seed=2)
    w.limit(60)
    total = w.next_pos.clone()
    for _ in range(6):
        for r, (new, probs) in enumerate(w.step(4)):
            total[r] += len(new)
            assert all(p <= 0 for p in probs)
    assert w.length.tolist()[0] == 60 and w.length.tolist()[2] == 60 and w.length.tolist()[1] < 60
    assert w.next_pos.tolist() == total.tolist()
    # the most recent positions are all there, in every head
    for r in (0, 2):
        i = np.arange(60)
        pos = w.pos[w.table[r].cpu().numpy()[i // 16], :, i % 16].cpu().numpy()
        for h in range(2):
            assert set(range(int(w.next_pos[r]) - 60, int(w.next_pos[r]))) >= set(pos[:, h][pos[:, h] >= int(w.next_pos[r]) - 60])
            assert (pos[:, h] >= int(w.next_pos[r]) - 64).sum() >= 1 and len(set(pos[:, h])) == 60


def test_the_program_runs(example, capsys):
    tokens, (k2, c2, c3), place = example.main(["--requests", "8", "--steps", "3", "--workers", "4"])
    assert tokens >= 24 and k2 >= 0 and c2 >= 0 and c3 >= 0 and k2 + c2 + c3 > 0
    assert len(place) == 64 and "placed" in capsys.readouterr().out
