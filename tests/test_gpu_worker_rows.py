"""Log probabilities of rows with many equal, masked or very large logits, against their definitions in 64 bits.

Tolerances as in test_gpu_worker.py, fixed before the first run: 1e-5 + 2^-21 of the logits' and results' size for
log probabilities, 1e-5 (1 + entropy) for entropies; ranks and the alternatives' indices are equal."""
import numpy as np
import pytest

from test_gpu_worker import A, check_logprobs  # noqa: F401  (A is a fixture)

pytestmark = pytest.mark.gpu

KINDS = ["bf16", "f16", "f32"]


def tensor(x, kind):
    """x as kind holds it, on the CPU."""
    import torch
    t = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[kind]
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(t)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab,holders", [(1500, 128), (20000, 96), (20000, 128)])
def test_logprobs_many_equal_maxima(A, kind, vocab, holders):
    """More threads than alternatives and 32 hold the same largest entry: all threads of a row, or those of three
    of its four warps, the first one not among them. Many rows at once, so that warps run apart."""
    n = 400
    rng = np.random.default_rng(vocab + holders)
    x = rng.integers(-3, 1, (n, vocab)).astype(np.float32)
    per = 4 if kind == "f32" else 8  # logits of a 16-byte vector; a thread takes every 128th
    quiet = np.arange(vocab) // per % 128 < 128 - holders
    x[:, quiet] -= 4.0
    token = rng.integers(0, vocab, n)
    for top in (1, 20, 64):
        few = slice(0, 8) if top == 64 else slice(0, 40)  # (the definition in Python is slow)
        t = tensor(x, kind)
        import torch
        with A.Worker("bf16", 1, 1, 64, 16) as w:
            got = w.logprobs(t.cuda(), torch.from_numpy(token.astype(np.int32)).cuda(), top)
            again = w.logprobs(t.cuda(), torch.from_numpy(token.astype(np.int32)).cuda(), top)
            assert w.status() == A.OK
        assert all(torch.equal(a, b) for a, b in zip(got, again))
        check_logprobs(t.double().numpy()[few], token[few], top, [g[few] for g in got])
        # every row's alternatives: the first of the equal ones
        order = np.argsort(-t.double().numpy(), axis=1, kind="stable")[:, :top]
        assert np.array_equal(got[3].cpu().numpy(), order)
