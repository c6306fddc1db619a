"""Eviction from a cache whose table names pages outside the pool: their tokens are hidden, the others are treated
as the definition says. Slots of such a page that lie before the budget stay where they are (nothing can be moved
into them); of the other slots, the best that the rest of the budget has room for stay. Moved values are equal."""
import numpy as np
import pytest

from test_gpu_worker import A  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def expected(weight, pos, hidden, next_pos, budget, recent):
    """Where the token of each slot before the budget comes from (a hidden slot: itself), of one request and head."""
    held = len(weight)
    key = np.where(np.isnan(weight), -np.inf, weight.astype(np.float64))
    key[pos >= next_pos - recent] = np.inf
    slot = np.arange(held)
    stay = hidden & (slot < budget)
    rest = slot[~hidden]
    # (NaN behind -inf, hidden ones last of all)
    order = rest[np.lexsort((rest, np.isnan(weight[rest]) & (pos[rest] < next_pos - recent), -key[rest]))]
    room = budget - stay.sum()
    stay[order[:room]] = True
    src = slot[:budget].copy()
    holes, movers = np.flatnonzero(~stay[:budget]), budget + np.flatnonzero(stay[budget:])
    if room > len(rest):  # all others stay, and hidden ones fill up: nothing moves
        holes = movers = holes[:0]
    assert len(holes) == len(movers)
    src[holes] = movers
    return src


CASES = [  # requests' lengths and budgets, key heads, page, table entries, hidden entries of each request
    ([300, 200, 64], [100, 150, 20], 2, 16, 24, [[1, 3, 15], [12], [0]]),        # one CTA, lists in shared memory
    ([9000], [3000], 2, 64, 160, [[0, 7, 40, 46, 47, 100, 140]]),                # a cluster and the second kernel
    ([70000, 500, 41], [20011, 100, 40], 1, 64, 1100, [[5, 312, 313, 900], [3], [2]]),
    ([10000] + [30] * 79, [5000] + [20] * 79, 4, 64, 160, [[2, 30, 78, 79, 150]] + [[0]] + [[]] * 78),  # one CTA, many moves
    ([4000], [3000], 1, 64, 63, [list(range(10, 50))]),                          # fewer tokens in sight than the budget
    ([5000, 5000], [0, 4999], 2, 256, 20, [[1, 19], [0, 19]]),
]


@pytest.mark.parametrize("lens,budget,hk,page,width,bad", CASES)
@pytest.mark.parametrize("weights", ["spread", "ties", "odd"])
def test_evict_with_hidden_pages(A, lens, budget, hk, page, width, bad, weights):
    import torch
    rng = np.random.default_rng(len(lens) + page)
    n, dim, recent = len(lens), 64, 64
    need = [-(-l // page) for l in lens]
    pages = sum(need)
    table = np.full((n, width), -1, np.int32)
    order, at = rng.permutation(pages), 0
    for r, m in enumerate(need):
        table[r, :m] = order[at:at + m]
        at += m
    real = table.copy()
    outside = [-1, pages, 2 ** 31 - 1, -2 ** 31]
    for r, cols in enumerate(bad):
        for i, c in enumerate(cols):
            table[r, c] = outside[i % 4]
    w = rng.exponential(size=(pages, hk, page)).astype(np.float32)
    if weights == "ties":
        w = rng.integers(0, 3, w.shape).astype(np.float32)
    elif weights == "odd":
        pick = rng.integers(0, 6, w.shape)
        for i, x in enumerate((np.nan, -np.inf, -0.0, 0.0, -1.0)):
            w[pick == i] = x
    pos = np.zeros((pages, hk, page), np.int32)
    for r, l in enumerate(lens):
        for h in range(hk):
            i = np.arange(l)
            pos[real[r, i // page], h, i % page] = rng.permutation(l + 40)[:l]
    mark = torch.arange(pages * hk * page, device="cuda").view(pages, hk, page, 1)
    k = (mark.to(torch.int32) + torch.zeros((1, 1, 1, dim // 2), dtype=torch.int32, device="cuda")).view(torch.bfloat16)
    v = k.flip(3).contiguous()
    k0, v0 = k.clone().view(torch.int32).cpu().numpy(), v.clone().view(torch.int32).cpu().numpy()
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    length, nxt = i32(lens), i32([l + 40 for l in lens])
    dw, dp = torch.from_numpy(w).cuda(), torch.from_numpy(pos).cuda()
    with A.Worker("bf16", hk, hk, dim, page) as worker:
        worker.evict(A.make_kv(k, v, i32(table), length, dw, dp, nxt), i32(budget), recent)
        assert worker.status() == A.ERR_STATE
    assert length.tolist() == [min(l, b) for l, b in zip(lens, budget)]
    k, v = k.view(torch.int32).cpu().numpy(), v.view(torch.int32).cpu().numpy()
    dw, dp = dw.cpu().numpy(), dp.cpu().numpy()
    for r, (l, b) in enumerate(zip(lens, budget)):
        i = np.arange(l)
        pg, sl = real[r, i // page], i % page
        hidden = np.isin(i // page, bad[r])
        for h in range(hk):
            src = expected(w[pg, h, sl], pos[pg, h, sl], hidden, l + 40, b, recent) if l > b else i
            to = np.arange(len(src))
            for got, was in ((k, k0), (v, v0), (dw, w), (dp, pos)):
                assert np.array_equal(got[pg[to], h, sl[to]], was[pg[src], h, sl[src]], equal_nan=got is dw), (r, h)
