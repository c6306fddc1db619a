"""A worker that serves requests with the library's decode-step operators, measured for the scheduler.

The scheduler's model of a worker (Eq. iter time) says that a decode iteration over b requests with sum(ctx)
cached tokens takes t_d = k2 sum(ctx) + c2 b + c3. This program is such a worker, with one attention layer of
random weights: it holds the requests of a synthetic workload in a paged cache and decodes them with drafted
trees,

    attend     the drafted tokens of every request, over its cached tokens,
    logprobs   of what the model says after each of them: the most likely next token, and its probability,
    accept     the drafted path that the model agrees with, into the cache, with the attention weights,
    evict      what a request holds over its budget,

times iterations of several sizes, fits k2, c2 and c3, and has the scheduler place waiting requests on a fleet
of such workers. With rotary positions,

    rotate     the drafted tokens' queries and keys to their positions in the trees, before attend;

and with a cache of 8 bits, which holds twice as many tokens,

    append     the prompts, rotated on the way, and then the drafted path, in the place of accept.

    python examples/worker_step.py --requests 64 --steps 20 --budget 1024
    python examples/worker_step.py --requests 64 --steps 20 --rotary --cache 8
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2405_06856_gb300 import aladdin as A  # noqa: E402
from paper_2405_06856_gb300 import synth  # noqa: E402


class ServingWorker:
    """Requests in a paged cache, and a model of one attention layer with tied random embeddings."""

    def __init__(self, lengths, q_heads=32, kv_heads=8, dim=128, page=64, vocab=4096, room=512, kind="bf16", seed=1,
                 rotary=False, cache=16):
        """rotary: rotary positions, scaled for a context four times as long; cache: bits of a cached number, 16 or 8."""
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rng = np.random.default_rng(seed)
        self.worker = A.Worker(kind, q_heads, kv_heads, dim, page)
        dt, dev = self.worker.dtype, self.worker.device
        normal = lambda *s: torch.randn(s, generator=self.gen, device=dev, dtype=torch.float32)
        self.vocab, self.heads = vocab, (q_heads, kv_heads)
        self.embed = normal(vocab, 256).to(dt)
        self.project = (normal(256, (q_heads + 2 * kv_heads) * dim) / 16).to(dt)
        self.head = normal(q_heads * dim, vocab) / dim ** 0.5  # logits in 32 bits: fewer of them are equal
        n = len(lengths)
        self.length = torch.tensor(lengths, dtype=torch.int32, device=dev)
        self.next_pos = self.length.clone()
        width = -(-(max(lengths) + room) // page)
        pages = n * width
        self.table = torch.from_numpy(self.rng.permutation(pages).astype(np.int32)).view(n, width).to(dev)
        if cache != 8:
            self.k, self.v = normal(pages, kv_heads, page, dim).to(dt), normal(pages, kv_heads, page, dim).to(dt)
        self.rope = A.make_rope(dim, scaling="parts", factor=4.0, original=8192) if rotary else None
        self.eight, self.budget = cache == 8, None
        self.root = torch.randint(0, vocab, (n,), generator=self.gen, device=dev)  # each request's last token
        if self.eight:
            self._prompts(lengths, pages, kv_heads, page, dim)
            return
        self.weight = torch.zeros((pages, kv_heads, page), device=dev)
        slot = torch.arange(width * page, device=dev, dtype=torch.int32).view(width, 1, page)
        self.pos = torch.zeros((pages, kv_heads, page), dtype=torch.int32, device=dev)
        self.pos[self.table.flatten().long()] = slot.expand(width, kv_heads, page).repeat(n, 1, 1)
        self.kv = A.make_kv(self.k, self.v, self.table, self.length, self.weight, self.pos, self.next_pos)

    def _prompts(self, lengths, pages, kv_heads, page, dim):
        """A cache of 8 bits, with the requests' prompts in it: random tokens' keys, rotated, and values."""
        dev = self.worker.device
        self.k, self.v = (torch.zeros((pages, kv_heads, page, dim), dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
                          for _ in range(2))
        self.k_scale, self.v_scale = (torch.zeros((pages, kv_heads, page // 16), device=dev) for _ in range(2))
        self.length.zero_()
        self.next_pos.zero_()
        self.kv = A.make_kv8(self.k, self.v, self.k_scale, self.v_scale, self.table, self.length, self.next_pos)
        off = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), dtype=torch.int32, device=dev)
        token = torch.randint(0, self.vocab, (int(sum(lengths)),), generator=self.gen, device=dev)
        hq, hk = self.heads
        x = (self.embed[token] @ self.project).view(len(token), hq + 2 * hk, dim)
        self.worker.append(self.kv, A.make_tokens(off, None, x[:, hq:hq + hk], x[:, hq + hk:]), self.rope)

    def step(self, drafted=1, drafts=None):
        """One iteration. Every request's tree has its last token as root and ``drafted`` - 1 drafted tokens
        (``drafts(request, n)`` gives their tokens and parents; random ones otherwise). Returns the tokens that
        each request gained, and their log probabilities."""
        n, dev = len(self.root), self.worker.device
        parent = np.full((n, drafted), -1, np.int32)
        token = np.zeros((n, drafted), np.int64)
        token[:, 0] = self.root.cpu().numpy()
        for r in range(n):
            if drafted > 1:
                token[r, 1:], parent[r, 1:] = drafts(r, drafted - 1) if drafts else (
                    self.rng.integers(0, self.vocab, drafted - 1), self.rng.integers(0, np.arange(1, drafted)))
        x = self.embed[torch.from_numpy(token).to(dev)].view(n * drafted, -1) @ self.project
        hq, hk = self.heads
        x = x.view(n * drafted, hq + 2 * hk, -1)
        off = torch.arange(n + 1, dtype=torch.int32, device=dev) * drafted
        tok = A.make_tokens(off, x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:],
                            torch.from_numpy(parent.ravel()).to(dev))
        if self.rope is not None:  # in place: the tokens' own queries and keys
            self.worker.rotate(self.rope, tok, self.next_pos, q_out=x[:, :hq], k_out=x[:, hq:hq + hk])
        out, lse = self.worker.attend(self.kv, tok)
        logits = out.view(n * drafted, -1).float() @ self.head
        _, _, _, best, logprob = self.worker.logprobs(logits, top=1)
        best, logprob = best.view(n, drafted).cpu().numpy(), logprob.view(n, drafted).cpu().numpy()
        gained, path, at = [], [], [0]
        for r in range(n):
            t, new, probs = 0, [], []
            while t is not None:  # follow the drafted tokens that the model would have chosen itself
                path.append(t)
                new.append(int(best[r, t]))
                probs.append(float(logprob[r, t]))
                t = next((c for c in range(t + 1, drafted) if parent[r, c] == t and token[r, c] == new[-1]), None)
            at.append(len(path))
            gained.append((new, probs))
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)
        if self.eight:
            self.worker.append(self.kv, tok, None, ints(at), ints(path))
        else:
            self.worker.accept(self.kv, tok, None, lse, ints(at), ints(path))
        if self.budget is not None:
            self.worker.evict(self.kv, self.budget, self.recent)
        self.root = torch.tensor([g[0][-1] for g in gained], device=dev)
        return gained

    def limit(self, budget, recent=64):
        """From the next step on every request keeps ``budget`` tokens a head, the last ``recent`` ones among them."""
        if self.eight:
            raise ValueError("a cache of 8 bits keeps no attention weights to choose by")
        self.budget, self.recent = torch.full_like(self.length, budget), recent


def iteration_ms(requests, context, repeat=5, **shape):
    """Time of the operators of a plain decode iteration: attend, logprobs, accept."""
    w = ServingWorker([context] * requests, **shape)
    hq, hk = w.heads
    x = (w.embed[w.root] @ w.project).view(requests, hq + 2 * hk, -1)
    tok = A.make_tokens(torch.arange(requests + 1, dtype=torch.int32, device="cuda"), x[:, :hq], x[:, hq:hq + hk],
                        x[:, hq + hk:])
    logits = torch.randn(requests, w.vocab, device="cuda")
    out, lse = w.worker.attend(w.kv, tok)
    times = []
    for _ in range(repeat + 2):
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        if w.rope is not None:
            w.worker.rotate(w.rope, tok, w.next_pos, q_out=x[:, :hq], k_out=x[:, hq:hq + hk])
        w.worker.attend(w.kv, tok, out=out, lse=lse)
        w.worker.logprobs(logits, top=1)
        if w.eight:
            w.worker.append(w.kv, tok)
        else:
            w.worker.accept(w.kv, tok, None, lse)
        e[1].record()
        torch.cuda.synchronize()
        times.append(e[0].elapsed_time(e[1]))
    return float(np.median(times[2:]))


def fit(sizes, **shape):
    """(k2, c2, c3) >= 0 of iterations over (requests, context) pairs, least squares of the relative error."""
    rows, times = [], []
    for b, ctx in sizes:
        rows.append([b * ctx, b, 1.0])
        times.append(iteration_ms(b, ctx, **shape))
    rows, times = np.array(rows), np.array(times)
    use, x = [0, 1, 2], np.zeros(3)
    while True:  # a coefficient that comes out negative is 0
        x[:] = 0.0
        x[use] = np.linalg.lstsq(rows[:, use] / times[:, None], np.ones(len(times)), rcond=None)[0]
        if (x >= 0).all() or len(use) == 1:
            break
        use.remove(int(np.argmin(x)))
    return x, times


def main(argv=None):
    p = argparse.ArgumentParser()
    p.add_argument("--requests", type=int, default=64)
    p.add_argument("--steps", type=int, default=20)
    p.add_argument("--drafted", type=int, default=8)
    p.add_argument("--budget", type=int, default=1024)
    p.add_argument("--rotary", action="store_true", help="rotary positions")
    p.add_argument("--cache", type=int, choices=(16, 8), default=16, help="bits of a cached number")
    p.add_argument("--workers", type=int, default=16, help="workers of the fleet that the scheduler fills")
    a = p.parse_args(argv)
    torch.cuda.set_device(0)
    wl = synth.config("tiny", n_cand=64)
    rng = np.random.default_rng(3)
    ctx = synth.lognormal_lengths(rng, 512.0, 0.8, 16, 2048, a.requests)
    model = dict(rotary=a.rotary, cache=a.cache)
    w = ServingWorker([int(c) for c in ctx], **model)
    if a.cache == 16:
        w.limit(a.budget)
    before = w.length.sum().item()
    tokens = sum(len(g[0]) for _ in range(a.steps) for g in w.step(a.drafted))
    assert w.worker.status() == A.OK
    print("%d requests, %d cached tokens: %d iterations of %d drafted tokens gave %d tokens; %d cached tokens after"
          % (a.requests, before, a.steps, a.drafted, tokens, w.length.sum().item()))
    sizes = [(b, c) for b in (8, 32, 128) for c in (256, 1024, 4096)]
    (k2, c2, c3), times = fit(sizes, **model)
    print("t_d = %.3g ms per cached token + %.3g ms per request + %.3g ms (one layer; measured %.3f to %.3f ms)"
          % (k2, c2, c3, times.min(), times.max()))
    # a fleet of such workers, 32 layers each, under the scheduler
    prm = dict(wl.params, k2=max(32 * k2, 1e-9), c2=32 * c2, c3=32 * c3)
    W, slots = a.workers, 128
    roff = np.arange(W + 1, dtype=np.int32) * 24
    n = int(roff[-1])
    held = synth.lognormal_lengths(rng, 512.0, 0.8, 16, 2048, n)
    pred = synth.lognormal_lengths(rng, 256.0, 0.9, 8, 1024, n)
    gen = rng.integers(0, pred).astype(np.int32)
    with A.Cluster(prm, [1] * W, [65536] * W, [1.0] * W, slots, roff, held, gen, pred) as cl:
        place = cl.place_round(wl.cand_in, wl.cand_pred, wl.cand_wait)
    print("the scheduler placed %d of %d waiting requests on %d workers" % ((place >= 0).sum(), len(place), W))
    return tokens, (k2, c2, c3), place


if __name__ == "__main__":
    main()
