// aladdin_worker_evict: requests over their budget drop the cached tokens of
// least accumulated weight.
//
// Per (request, key head) with len > budget the `budget` slots of the largest
// key stay: the accumulated weight, infinite for the window of the most recent
// positions, the lowest slot first among equal keys. Slots behind the budget
// that stay (movers) go, in order, to the dropped slots before it (holes): as
// many as the call needs to move, and no slot is both read and written, so
// that the moves are independent of one another. The order of the cached
// tokens means nothing to the attention; `pos` says what is recent. Slots of a page
// outside the pool are neither: before the budget they stay, whatever the others hold, behind
// it only where all others do. So every hole and mover can be read and written.
//
// One CTA, or a cluster where there are few long requests, serves one (request,
// key head); each CTA keeps the keys of its part of the slots in shared memory.
// The budget-th largest key is found digit by digit (11 + 11 + 10 bits of the
// ordered key): each CTA counts its keys that agree with the digits known so far,
// every CTA adds the cluster's counts and picks the same digit, until all keys of
// the digit stay. Two scans then number equal keys, holes and movers in slot order.
// A warp moves 32 at a time: a lane looks one of them up and moves its weight and
// position, then the warp copies their rows, several 16-byte pieces of a lane in
// flight. One CTA moves what it found itself; after clusters, whose requests differ
// in length, a second kernel shares all moves evenly (the clusters' own moves
// left most of the GPU to the longest request: 89 us for three requests of up to
// 65,536 tokens; with the second kernel 69, 33 for the lists and 39 for the moves when each
// runs alone). One token over 1,024 on 64 requests of 8 heads takes 13 us, 15 with the launch.
#include <cooperative_groups.h>

#include "worker_dev.cuh"

namespace cg = cooperative_groups;

namespace aladdin {
namespace wk {
namespace {

constexpr int BINS = 2048;
constexpr int MAX_KEYS = 50 * 1024;  // keys that a CTA holds; it forms the others again where it needs them

// Order of the floats as unsigned numbers: -0 as +0, NaN below everything. 0 and the largest
// number stand for slots of pages outside the pool, behind the budget and before it.
__device__ __forceinline__ uint32_t ordered(float w)
{
    if (w != w) return 1u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Evict {
    const int32_t* row;  // the request's pages
    int h, held, budget, recent_from;
};

__device__ __forceinline__ int page_of(const EvictArgs& a, const Evict& e, int slot)
{
    const int p = e.row[slot >> a.kv.page_shift];
    return (unsigned)p < (unsigned)a.kv.pages ? p : -1;
}
// Index of a slot's weight and position.
__device__ __forceinline__ long long meta_at(const EvictArgs& a, const Evict& e, int page, int slot)
{
    return ((long long)page * a.kv.kv_heads + e.h) * a.kv.page + (slot & (a.kv.page - 1));
}
// Element of a slot's key and value.
__device__ __forceinline__ long long row_at(const EvictArgs& a, const Evict& e, int page, int slot)
{
    return page * a.kv.page_stride + e.h * a.kv.head_stride + (slot & (a.kv.page - 1)) * a.kv.token_stride;
}

// Keys of N slots first, first + step, ... below end, their loads together; pages outside
// the pool are recorded.
template <int N>
__device__ __forceinline__ void keys_of(const EvictArgs& a, const Evict& e, int first, int step, int end,
                                        uint32_t (&key)[N])
{
    int page[N], pos[N];
    float w[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int slot = first + i * step;
        page[i] = slot < end ? page_of(a, e, slot) : -1;
        if (slot < end && page[i] < 0) atomicOr(a.err, WORKER_BAD_INPUT);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const long long m = page[i] < 0 ? 0 : meta_at(a, e, page[i], first + i * step);
        pos[i] = page[i] < 0 ? 0 : a.kv.pos[m];
        w[i] = page[i] < 0 ? 0.0f : a.kv.weight[m];
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        key[i] = page[i] < 0 ? (first + i * step < e.budget ? 0xffffffffu : 0u)
                             : pos[i] >= e.recent_from ? ordered(INFINITY) : ordered(w[i]);
}

// Exclusive sums of two counts over the block's threads, and their totals.
template <int NT>
__device__ __forceinline__ int2 block_scan(int2 v, int2* scratch, int2& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 u = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, u.x, o), y = __shfl_up_sync(0xffffffffu, u.y, o);
        if (lane >= o) {
            u.x += x;
            u.y += y;
        }
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = u;
    __syncthreads();
    int2 before = make_int2(0, 0);
    total = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        const int2 s = scratch[w];
        if (w < warp) {
            before.x += s.x;
            before.y += s.y;
        }
        total.x += s.x;
        total.y += s.y;
    }
    return make_int2(before.x + u.x - v.x, before.y + u.y - v.y);
}

// The i-th of a (request, head)'s moves, whose holes and then movers lie in the workspace from
// `base` on.
__device__ __forceinline__ void listed(const EvictArgs& a, long long base, int moves, int i, int& from, int& to)
{
    to = __ldcg(a.lists + base + i);
    from = __ldcg(a.lists + base + moves + i);
}

// Moves a lane's slot `from` to its slot `to` (the lanes below n; -1: nothing), the warp together.
template <int D, int U>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const Evict& e, int from, int to, int n, int lane)
{
    constexpr int CH = D / 8, PER = 2 * CH;  // 16-byte pieces of a key, of a key and a value; U of a lane in flight
    long long src = -1, dst = -1;
    // (lists of a request whose arrays changed under the call may not be full)
    if (lane < n && from >= 0 && to >= 0 && from < a.kv.cap && to < a.kv.cap) {
        const int pd = page_of(a, e, to), ps = page_of(a, e, from);
        if (pd >= 0 && ps >= 0) {
            src = row_at(a, e, ps, from);
            dst = row_at(a, e, pd, to);
            const long long ms = meta_at(a, e, ps, from), md = meta_at(a, e, pd, to);
            a.kv.weight[md] = a.kv.weight[ms];
            a.kv.pos[md] = a.kv.pos[ms];
        }
    }
    const int pieces = n * PER;
    for (int x0 = 0; x0 < pieces; x0 += 32 * U) {
        uint4 v[U];
        long long at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * 32 + lane, m = x / PER, c = x - m * PER;
            const long long s = __shfl_sync(0xffffffffu, src, m & 31);
            at[u] = __shfl_sync(0xffffffffu, dst, m & 31);
            if (x >= pieces || s < 0) at[u] = -1;
            else {
                const char* const pool = c < CH ? a.kv.k : a.kv.v;
                const int cc = (c < CH ? c : c - CH) * 8;
                v[u] = *reinterpret_cast<const uint4*>(pool + (s + cc) * 2);
                at[u] += cc;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int x = x0 + u * 32 + lane, c = x % PER;
            if (at[u] >= 0) *reinterpret_cast<uint4*>((c < CH ? a.kv.k : a.kv.v) + at[u] * 2) = v[u];
        }
    }
}

// CLUSTER: a cluster serves a (request, head), else one CTA.
template <int D, int NT, bool CLUSTER>
__global__ void __launch_bounds__(NT, CLUSTER ? 2 : 4) k_evict(EvictArgs a, int max_keys)
{
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ __align__(16) int hist[2][BINS];
    __shared__ int2 scratch[NT / 32];
    __shared__ int2 counts;  // what the cluster's other CTAs read of this one
    __shared__ int s_digit, s_above, s_here, s_last;
    __shared__ long long s_base;  // where this (request, head)'s lists start; -1: there is no room
    const int cs = CLUSTER ? (int)cluster.num_blocks() : 1, rank = CLUSTER ? (int)cluster.block_rank() : 0;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int unit = blockIdx.x / cs, H = a.kv.kv_heads, r = unit / H;
    auto meet = [&]() {
        if (CLUSTER) cluster.sync();
        else __syncthreads();
    };

    Evict e;
    e.h = unit - r * H;
    e.row = a.kv.table + (long long)r * a.kv.table_stride;
    e.held = a.kv.len[r];
    const int budget = e.budget = a.budget[r];
    const long long from = (long long)a.kv.next[r] - a.recent;  // recent positions (an int may not hold it)
    e.recent_from = from < -0x7fffffffll ? -0x7fffffff : (int)from;
    const bool ok = e.held >= 0 && e.held <= a.kv.cap && budget >= 0;
    if (!ok && rank == 0 && e.h == 0 && tid == 0) atomicOr(a.err, WORKER_BAD_INPUT);
    if (ok && e.held > budget) {
        const int span = (e.held + cs - 1) / cs, s0 = min(rank * span, e.held), s1 = min(s0 + span, e.held),
                  n = s1 - s0;
        for (int i = tid; i < BINS; i += NT) hist[0][i] = 0;
        __syncthreads();
        // the keys, and the counts of their first digit
        for (int i = tid; i < n; i += 4 * NT) {
            uint32_t k[4];
            keys_of<4>(a, e, s0 + i, NT, s1, k);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                if (i + x * NT < n) {
                    if (i + x * NT < max_keys) keys[i + x * NT] = k[x];
                    atomicAdd(&hist[0][k[x] >> 21], 1);
                }
            }
        }
        auto key = [&](int i) -> uint32_t {
            if (i < max_keys) return keys[i];
            uint32_t k[1];
            keys_of<1>(a, e, s0 + i, 0, s1, k);
            return k[0];
        };

        // the digits of the budget-th largest key, and how many slots that agree with them stay
        uint32_t known = 0, mask = 0;
        int want = budget, here = 0;
        bool found = budget == 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            if (found) break;
            const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            int* const h = hist[pass & 1];
            if (pass) {
                // (cleared since all CTAs read it: there was a barrier of the cluster in between)
                for (int i = tid; i < BINS; i += NT) h[i] = 0;
                __syncthreads();
                for (int i = tid; i < n; i += NT) {
                    const uint32_t k = key(i);
                    if ((k & mask) == known) atomicAdd(h + ((k >> shift) & ((1u << bits) - 1)), 1);
                }
            }
            meet();
            // a thread adds the cluster's counts of a few digits, the highest first
            constexpr int PER = BINS / NT;
            int c[PER], sum = 0;
            const int d0 = BINS - (tid + 1) * PER;  // its lowest digit
#pragma unroll
            for (int x = 0; x < PER; x += 4) {
                int4 q = *reinterpret_cast<const int4*>(h + d0 + x);
                if (CLUSTER) {
                    q = make_int4(0, 0, 0, 0);
#pragma unroll 8
                    for (int b = 0; b < cs; ++b) {
                        const int4 o = *reinterpret_cast<const int4*>(cluster.map_shared_rank(h, b) + d0 + x);
                        q.x += o.x, q.y += o.y, q.z += o.z, q.w += o.w;
                    }
                }
                c[x] = q.x, c[x + 1] = q.y, c[x + 2] = q.z, c[x + 3] = q.w;
                sum += q.x + q.y + q.z + q.w;
            }
            int2 total;
            int above = block_scan<NT>(make_int2(sum, 0), scratch, total).x;
            if (above < want && above + sum >= want) {
                bool got = false;
#pragma unroll
                for (int x = PER - 1; x >= 0; --x) {
                    if (!got) {
                        if (above + c[x] >= want) {
                            s_digit = d0 + x;
                            s_above = above;
                            s_here = c[x];
                            got = true;
                        } else {
                            above += c[x];
                        }
                    }
                }
            }
            __syncthreads();
            known |= (uint32_t)s_digit << shift;
            mask |= ((1u << bits) - 1) << shift;
            want -= s_above;
            here = s_here;
            found = want == here;  // all of them stay
        }
        if (budget == 0) known = mask = 0xffffffffu;  // nothing is above the largest number, and none of it stays

        // a thread looks at a run of slots (odd, so that a warp's reads fall in
        // different banks); counts before it number its equal keys, then its holes and movers
        const int run = ((n + NT - 1) / NT) | 1, i0 = min(tid * run, n), i1 = min(i0 + run, n);
        // counts of the cluster's CTAs before this one; `all` becomes those of all. `take`: room for the
        // lists of as many moves
        auto before_me = [&](int2 total, int2& all, bool take) -> int2 {
            int2 v = make_int2(0, 0);
            all = total;
            if (CLUSTER) {
                if (tid == 0) counts = total;
                cluster.sync();
                all = v;
                for (int b = 0; b < cs; ++b) {
                    const int2 c = *cluster.map_shared_rank(&counts, b);
                    if (b < rank) v.x += c.x, v.y += c.y;
                    all.x += c.x;
                    all.y += c.y;
                }
            }
            if (take && rank == 0 && tid == 0) {
                // (slots that move or are moved into are a slot of the pool each: there is room, unless
                // requests share them)
                const unsigned long long n = 2ull * all.y, at = atomicAdd(a.cursor, n);
                s_base = at + n <= a.lists_n ? (long long)at : -1;
                if (s_base < 0) atomicOr(a.err, WORKER_BAD_INPUT);
            }
            if (CLUSTER) cluster.sync();
            else if (take) __syncthreads();
            return v;
        };
        __syncthreads();
        int2 mine = make_int2(0, 0), total, all, at;
        int equal0 = 0;  // equal keys in front of this thread's run
        if (want != here && budget > 0) {
            for (int i = i0; i < i1; ++i) mine.x += (key(i) & mask) == known;
            at = block_scan<NT>(mine, scratch, total);
            equal0 = at.x + before_me(total, all, false).x;
        }
        int equal = equal0;
        auto stays = [&](uint32_t k) { return (k & mask) > known || ((k & mask) == known && equal++ < want); };
        mine = make_int2(0, 0);
        for (int i = i0; i < i1; ++i) {
            const bool s = stays(key(i));
            if (s0 + i < budget) mine.x += !s;
            else mine.y += s;
        }
        at = block_scan<NT>(mine, scratch, total);
        // the lists of holes and movers: in shared memory (in place of the counts) where one CTA
        // has few of them, else in the workspace
        const bool near = !CLUSTER && total.y <= BINS;
        const int2 moved0 = before_me(total, all, !near);
        at.x += moved0.x;
        at.y += moved0.y;
        int moves = all.y;
        const long long base = near ? 0 : CLUSTER ? *cluster.map_shared_rank(&s_base, 0) : s_base;
        if (base < 0) moves = 0;
        auto note = [&](int list, int i, int slot) {
            if (i >= moves) return;
            if (near) hist[list][i] = slot;
            else a.lists[base + (list ? moves : 0) + i] = slot;
        };
        equal = equal0;
        for (int i = i0; i < i1; ++i) {
            const bool s = stays(key(i));
            if (s0 + i < budget) {
                if (!s) note(0, at.x++, s0 + i);
            } else if (s) {
                note(1, at.y++, s0 + i);
            }
        }
        if (CLUSTER) {
            if (rank == 0 && tid == 0) {
                a.moves[unit] = moves;
                a.bases[unit] = base;
            }
            cluster.sync();  // the others have read this CTA's counts
        } else {
            if (!near) __threadfence();
            __syncthreads();
            // every warp the same number of moves
            const int share = (moves + NT / 32 - 1) / (NT / 32), first = warp * share, last = min(first + share, moves);
            for (int m0 = first; m0 < last; m0 += 32) {
                const int i = m0 + lane;
                int from = -1, to = -1;
                if (i < last) {
                    if (near) {
                        to = hist[0][i];
                        from = hist[1][i];
                    } else {
                        listed(a, base, moves, i, from, to);
                    }
                }
                move_rows<D, 4>(a, e, from, to, min(32, last - m0), lane);
            }
        }
    } else if (CLUSTER && rank == 0 && tid == 0) {
        a.moves[unit] = 0;
    }

    // every CTA has read the lengths: the last one to come here cuts them
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        s_last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (s_last) {
        if (tid == 0) {
            *a.arrived = 0;
            *a.cursor = 0;
        }
        for (int q = tid; q < a.n_req; q += NT) {
            const int len = a.kv.len[q], b = a.budget[q];
            if (len >= 0 && len <= a.kv.cap && b >= 0 && len > b) a.kv.len[q] = b;
        }
    }
}

// The moves that the clusters listed, shared evenly by all warps. units <= MOST_UNITS.
constexpr int MOST_UNITS = 1024, MOVERS = 256, MOVE_CTAS = 3;  // threads of a CTA, CTAs of an SM
template <int D>
__global__ void __launch_bounds__(MOVERS, MOVE_CTAS) k_move(EvictArgs a, int units)
{
    __shared__ int pre[MOST_UNITS + 1];
    __shared__ long long scratch[32];
    const int total = plan_prefix<MOVERS>(units, pre, scratch, [&](int u) -> long long { return a.moves[u]; });
    const int lane = threadIdx.x & 31, warps = gridDim.x * (MOVERS / 32), me = blockIdx.x * (MOVERS / 32) + (threadIdx.x >> 5);
    // (fewer than 2^31: a slot moves once, and a pool's slots are counted in ints)
    const long long share = ((long long)total + warps - 1) / warps, first = me * share, last = min(first + share, (long long)total);
    for (long long m0 = first; m0 < last; m0 += 32) {
        const int n = (int)min(32ll, last - m0);
        Evict e;
        e.row = a.kv.table;
        e.h = e.held = e.budget = e.recent_from = 0;
        int from = -1, to = -1;
        if (lane < n) {
            const int unit = plan_find(pre, units, (int)(m0 + lane)), r = unit / a.kv.kv_heads;
            e.h = unit - r * a.kv.kv_heads;
            e.row = a.kv.table + (long long)r * a.kv.table_stride;
            listed(a, a.bases[unit], pre[unit + 1] - pre[unit], (int)(m0 + lane) - pre[unit], from, to);
        }
        move_rows<D, 8>(a, e, from, to, n, lane);
    }
}

template <int D, int NT, bool CLUSTER>
cudaError_t launch(const EvictArgs& a, long long units, int cs, cudaStream_t st)
{
    cudaError_t e = allow_smem<k_evict<D, NT, CLUSTER>>(MAX_KEYS * 4);
    if (e != cudaSuccess) return e;
    const long long span = (a.kv.cap + cs - 1) / cs;
    const int max_keys = (int)(span < MAX_KEYS ? span : MAX_KEYS);
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)(units * cs));
    c.blockDim = dim3(NT);
    c.dynamicSmemBytes = (size_t)max_keys * 4;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = CLUSTER ? 1 : 0;
    return cudaLaunchKernelEx(&c, k_evict<D, NT, CLUSTER>, a, max_keys);
}

template <int D>
cudaError_t launch_dim(const EvictArgs& a, int sms, cudaStream_t st)
{
    // CTAs for a (request, head): as many as fill the GPU twice, at most the portable
    // cluster, but few slots need no more than one. (Shared memory and clusters follow the slots that
    // the table has room for, as the host does not know the lengths: a wide table over short requests
    // leaves fewer CTAs on an SM.)
    const long long units = (long long)a.n_req * a.kv.kv_heads;
    int cs = 1;
    while (cs < 8 && units * cs < 2ll * sms && a.kv.cap > 2048ll * cs) cs *= 2;
    if (cs == 1 || units > MOST_UNITS) return launch<D, 256, false>(a, units, 1, st);
    const cudaError_t e = launch<D, 512, true>(a, units, cs, st);
    if (e != cudaSuccess) return e;
    k_move<D><<<MOVE_CTAS * sms, MOVERS, 0, st>>>(a, (int)units);
    return cudaGetLastError();
}

}  // namespace
}  // namespace wk

cudaError_t launch_evict(const EvictArgs& a, int sms, cudaStream_t st)
{
    switch (a.dim) {
        case 64: return wk::launch_dim<64>(a, sms, st);
        case 96: return wk::launch_dim<96>(a, sms, st);
        case 128: return wk::launch_dim<128>(a, sms, st);
        case 256: return wk::launch_dim<256>(a, sms, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace aladdin
