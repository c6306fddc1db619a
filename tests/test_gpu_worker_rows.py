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


def check_rows(A, x, token, top):
    """Every row by itself: x and the maximum are exact, so that errors are those of the difference, 2^-21 of the
    result, and of the sums."""
    import torch
    import worker_ref as ref
    with A.Worker("bf16", 1, 1, 64, 16) as w:
        got = w.logprobs(x.cuda(), torch.from_numpy(np.asarray(token, np.int32)).cuda(), top)
        assert w.status() == A.OK
    got = [g.double().cpu().numpy() for g in got]
    rows = x.double().numpy()
    lp, ent, rank, ids, tlp = ref.logprobs(rows, token, top)
    for r, row in enumerate(rows):  # with the maximum taken off first: next to 1e30 a logarithm vanishes in 64 bits, too
        if np.isfinite(row.max()):
            d = row - row.max()
            d -= np.log(np.exp(d).sum())
            lp[r], tlp[r] = d[token[r]], d[ids[r]]
    assert np.array_equal(got[2], rank) and np.array_equal(got[3], ids)
    for name, g, w, tol in (("logprob", got[0], lp, None), ("top_logprob", got[4], tlp, None),
                            ("entropy", got[1], ent, 1e-5 * (1 + np.abs(ent)))):
        fin = np.isfinite(w)
        assert np.array_equal(np.isnan(g), np.isnan(w)), (name, g, w)
        assert np.array_equal(g[~fin & ~np.isnan(w)], w[~fin & ~np.isnan(w)]), (name, g, w)
        if tol is None:
            tol = 1e-5 + 2.0 ** -21 * np.abs(w)
        off = np.abs(np.where(fin, g, 0.0) - np.where(fin, w, 0.0))
        assert np.all(off <= np.where(fin, tol, 0.0)), (name, off.max(), g, w)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [40, 3000, 20000])
def test_logprobs_masks_of_the_lowest_value(A, kind, vocab):
    """Rows masked by the type's lowest value, by -inf, and by both, alone and beside ordinary logits."""
    import torch
    rng = np.random.default_rng(7)
    low = float(torch.finfo(tensor(np.zeros(1), kind).dtype).min)
    place = np.arange(vocab)
    both = np.where(place % 2 == 0, low, -np.inf)
    some = 3.0 * rng.normal(size=vocab)
    x = np.stack([np.full(vocab, low), both, np.where(place == vocab // 2, low, -np.inf),
                  np.where(place < vocab // 2, both, some), np.where(place < vocab - 3, both, some),
                  np.where(place >= vocab // 4, both, some), np.where(place % 97 == 5, some, both),
                  np.where(place % 97 == 5, some, low), np.where(place % 97 == 5, some, -np.inf)])
    token = rng.integers(0, vocab, len(x))
    for top in (1, 20):
        check_rows(A, tensor(x, kind), token, top)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [40, 3000, 20000])
def test_logprobs_large_logits(A, kind, vocab):
    """Rows of large logits of either sign: equal ones, neighbours in the type, with -inf, and as a mask in front of
    ordinary ones (a row masked by -1e9 or -1e30 is one of them)."""
    import torch
    rng = np.random.default_rng(8)
    sizes = [1e3, 5e3, 2e4, 3.3e4, 5e4, 6.5e4] if kind == "f16" else [1e5, 1e7, 1e8, 4e8, 1e9, 1e10, 1e20, 1e30, 1e37, 3e38]
    t = tensor(np.zeros(1), kind).dtype
    place = np.arange(vocab)
    some = 3.0 * rng.normal(size=vocab)
    rows = []
    for size in sizes:
        for v in (size, -size):
            a = torch.tensor(v).to(t)
            b = torch.nextafter(a.float(), torch.tensor(0.0)) if kind == "f32" else (a.view(torch.int16) - 1).view(t)
            a, b = float(a), float(b)  # b: the neighbour nearer to 0
            rows += [np.full(vocab, a), np.where(place % 3 == 1, a, b), np.where(place % 2 == 0, a, -np.inf)]
            if v < 0:
                rows += [np.where(place < vocab // 2, a, some), np.where(place % 97 == 5, some, a)]
    x = np.stack(rows)
    token = rng.integers(0, vocab, len(x))
    check_rows(A, tensor(x, kind), token, 5)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("vocab", [40, 3000, 20000])
def test_logprobs_odd_rows_of_16_bits(A, kind, vocab):
    """Equal and rounded values, infinities, NaN, -0 and denormal ones in rows of 16 bits; every row's token among
    several places."""
    rng = np.random.default_rng(3)
    tiny = 1e-39 if kind == "bf16" else 1e-7  # denormal in the type
    x = (2.0 * rng.normal(size=(14, vocab))).astype(np.float32)
    x[0] = 1.5
    x[1] = -np.inf
    x[2, ::2] = -np.inf
    x[3, vocab // 2] = np.nan
    x[4, vocab // 3] = np.inf
    x[5] = np.nan
    x[6] = np.where(np.arange(vocab) % 3 == 0, 0.0, -0.0)
    x[7] = np.round(x[7])
    x[8] = tiny * rng.integers(-4, 5, vocab)
    x[9, ::1024], x[9, 1::1024], x[9, 2::1024] = 30.0, 31.0, 32.0
    x[10, ::3] = np.nan
    x[10, 1::3] = -np.inf
    x[11] = np.where(np.arange(vocab) // 8 % 128 == 3, 40.0 + x[11], x[11])
    x[12] = -100.0 + x[12]
    x[13, 5:] = -np.inf
    for at in (0, vocab // 3, vocab // 2, vocab - 1):
        check_rows(A, tensor(x, kind), np.full(14, at), 20)
