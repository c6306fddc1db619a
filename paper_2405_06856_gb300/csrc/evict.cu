// aladdin_worker_evict: requests over their budget drop the cached tokens of
// least accumulated weight.
//
// Per (request, key head) with len > budget the `budget` slots of the largest
// key stay: the accumulated weight, infinite for the window of the most recent
// positions, the lowest slot first among equal keys. Slots behind the budget
// that stay (movers) go, in order, to the dropped slots before it (holes): as
// many as the call needs to move, and no slot is both read and written, so
// that the moves are independent of one another. The order of the cached
// tokens means nothing to the attention; `pos` says what is recent.
//
// A cluster of CTAs serves one (request, key head); each keeps the keys of its
// part of the slots in shared memory. The budget-th largest key is found digit
// by digit (11 + 11 + 10 bits of the ordered key): each CTA counts its keys
// that agree with the digits known so far, every CTA adds the cluster's counts
// and picks the same digit. Two scans then number equal keys, holes and movers
// in slot order, and the cluster's CTAs share the moves.
#include <cooperative_groups.h>

#include "worker_dev.cuh"

namespace cg = cooperative_groups;

namespace aladdin {
namespace wk {
namespace {

constexpr int NT = 512;
constexpr int BINS = 2048;
constexpr int MAX_KEYS = 50 * 1024;  // keys that a CTA holds; it forms the others again where it needs them

// Order of the floats as unsigned numbers: -0 as +0, NaN below everything.
__device__ __forceinline__ uint32_t ordered(float w)
{
    if (w != w) return 0u;
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

struct Evict {
    const int32_t* row;  // the request's pages
    int h, held, recent_from;
};

__device__ __forceinline__ long long meta_at(const EvictArgs& a, const Evict& e, int slot)
{
    const int p = e.row[slot >> a.kv.page_shift];
    if ((unsigned)p >= (unsigned)a.kv.pages) return -1;
    return ((long long)p * a.kv.kv_heads + e.h) * a.kv.page + (slot & (a.kv.page - 1));
}

__device__ __forceinline__ uint32_t key_of(const EvictArgs& a, const Evict& e, int slot)
{
    const long long m = meta_at(a, e, slot);
    if (m < 0) return 0u;
    if (a.kv.pos[m] >= e.recent_from) return ordered(INFINITY);
    return ordered(a.kv.weight[m]);
}

// Exclusive sums of two counts over the block's threads, and their totals.
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

__global__ void __launch_bounds__(NT) k_evict(EvictArgs a, int max_keys)
{
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ int hist[2][BINS];
    __shared__ int2 scratch[NT / 32];
    __shared__ int2 counts;    // what the cluster's other CTAs read of this one
    __shared__ int s_digit, s_above, s_last;
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x;
    const int unit = blockIdx.x / cs, H = a.kv.kv_heads, r = unit / H;

    Evict e;
    e.h = unit - r * H;
    e.row = a.kv.table + (long long)r * a.kv.table_stride;
    e.held = a.kv.len[r];
    const int budget = a.budget[r];
    const bool ok = e.held >= 0 && e.held <= a.kv.cap && budget >= 0;
    if (!ok && rank == 0 && e.h == 0 && tid == 0) atomicOr(a.err, WORKER_BAD_INPUT);
    if (ok && e.held > budget) {
        // positions from next - recent on are recent (an int may not hold the difference)
        const long long from = (long long)a.kv.next[r] - a.recent;
        e.recent_from = from < -0x7fffffffll ? -0x7fffffff : (int)from;
        const int span = (e.held + cs - 1) / cs, s0 = min(rank * span, e.held), s1 = min(s0 + span, e.held),
                  n = s1 - s0;
        for (int i = tid; i < n; i += NT) {
            if (meta_at(a, e, s0 + i) < 0) atomicOr(a.err, WORKER_BAD_INPUT);
            if (i < max_keys) keys[i] = key_of(a, e, s0 + i);
        }
        // (every thread reads the keys that it wrote, up to the next barrier)
        auto key = [&](int i) { return i < max_keys ? keys[i] : key_of(a, e, s0 + i); };

        // the budget-th largest key, and how many slots of that very key stay
        uint32_t known = 0, mask = 0;
        int want = budget;
        if (budget > 0) {
#pragma unroll
            for (int pass = 0; pass < 3; ++pass) {
                const int bits = pass < 2 ? 11 : 10, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
                int* const h = hist[pass & 1];
                for (int i = tid; i < BINS; i += NT) h[i] = 0;
                __syncthreads();
                for (int i = tid; i < n; i += NT) {
                    const uint32_t k = key(i);
                    if ((k & mask) == known) atomicAdd(h + ((k >> shift) & ((1u << bits) - 1)), 1);
                }
                cluster.sync();
                // thread t adds the cluster's counts of four digits, the highest first
                int c[BINS / NT], sum = 0;
#pragma unroll
                for (int x = 0; x < BINS / NT; ++x) {
                    const int d = BINS - 1 - (tid * (BINS / NT) + x);
                    c[x] = 0;
                    for (int b = 0; b < cs; ++b) c[x] += cluster.map_shared_rank(h, b)[d];
                    sum += c[x];
                }
                int2 total;
                int above = block_scan(make_int2(sum, 0), scratch, total).x;
                if (above < want && above + sum >= want) {
                    bool found = false;
#pragma unroll
                    for (int x = 0; x < BINS / NT; ++x) {
                        if (!found) {
                            if (above + c[x] >= want) {
                                s_digit = BINS - 1 - (tid * (BINS / NT) + x);
                                s_above = above;
                                found = true;
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
                // hist[pass & 1] is cleared again two passes on, behind a barrier of the cluster
            }
        }
        // budget 0: no key is above the largest one, and none of it stays
        if (budget == 0) known = 0xffffffffu;

        // a thread looks at a run of slots (odd, so that a warp's reads fall in
        // different banks); counts before it number its equal keys, then its holes and movers
        const int run = ((n + NT - 1) / NT) | 1, i0 = min(tid * run, n), i1 = min(i0 + run, n);
        auto before_me = [&](int2 total) -> int2 {
            if (tid == 0) counts = total;
            cluster.sync();
            int2 v = make_int2(0, 0);
            for (int b = 0; b < rank; ++b) {
                const int2 c = *cluster.map_shared_rank(&counts, b);
                v.x += c.x;
                v.y += c.y;
            }
            cluster.sync();
            return v;
        };
        __syncthreads();
        int2 mine = make_int2(0, 0), total;
        for (int i = i0; i < i1; ++i) mine.x += key(i) == known;
        int2 at = block_scan(mine, scratch, total);
        const int2 eq0 = before_me(total);
        const int equal0 = at.x + eq0.x;  // equal keys in front of this thread's run
        mine = make_int2(0, 0);
        int equal = equal0;
        for (int i = i0; i < i1; ++i) {
            const uint32_t k = key(i);
            const bool stays = k > known || (k == known && equal++ < want);
            if (s0 + i < budget) mine.x += !stays;
            else mine.y += stays;
        }
        at = block_scan(mine, scratch, total);
        const int2 moved0 = before_me(total);
        at.x += moved0.x;
        at.y += moved0.y;
        auto note = [&](int where, int slot) {
            const long long m = meta_at(a, e, where);
            if (m >= 0) a.lists[m] = slot;
        };
        equal = equal0;
        for (int i = i0; i < i1; ++i) {
            const uint32_t k = key(i);
            const bool stays = k > known || (k == known && equal++ < want);
            if (s0 + i < budget) {
                if (!stays) note(at.x++, s0 + i);
            } else if (stays) {
                note(budget + at.y++, s0 + i);
            }
        }
        // the number of moves: the movers of all CTAs
        if (tid == 0) counts = total;
        __threadfence();
        cluster.sync();
        int moves = 0;
        for (int b = 0; b < cs; ++b) moves += cluster.map_shared_rank(&counts, b)->y;

        const int ch = a.dim / 8, per = 2 * ch;  // 16-byte chunks of a key; of a key and a value
        const long long work = (long long)moves * per;
        for (long long x = (long long)rank * NT + tid; x < work; x += (long long)cs * NT) {
            const int i = (int)(x / per), c = (int)(x - (long long)i * per);
            const long long ls = meta_at(a, e, budget + i), ld = meta_at(a, e, i);
            if (ls < 0 || ld < 0) continue;
            const int src = __ldcg(a.lists + ls), dst = __ldcg(a.lists + ld);
            const long long ms = meta_at(a, e, src), md = meta_at(a, e, dst);
            if (ms < 0 || md < 0) continue;
            char* const pool = c < ch ? a.kv.k : a.kv.v;
            const int cc = c < ch ? c : c - ch;
            auto at_slot = [&](int slot) {
                return pool + (e.row[slot >> a.kv.page_shift] * a.kv.page_stride + e.h * a.kv.head_stride +
                               (slot & (a.kv.page - 1)) * a.kv.token_stride + cc * 8) * 2;
            };
            *reinterpret_cast<uint4*>(at_slot(dst)) = *reinterpret_cast<const uint4*>(at_slot(src));
            if (c == 0) a.kv.weight[md] = a.kv.weight[ms];
            if (c == ch) a.kv.pos[md] = a.kv.pos[ms];
        }
        cluster.sync();  // the others have read this CTA's counts
    }

    // every CTA has read the lengths: the last one to come here cuts them
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        s_last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (s_last) {
        if (tid == 0) *a.arrived = 0;
        for (int q = tid; q < a.n_req; q += NT) {
            const int len = a.kv.len[q], b = a.budget[q];
            if (len >= 0 && len <= a.kv.cap && b >= 0 && len > b) a.kv.len[q] = b;
        }
    }
}

}  // namespace
}  // namespace wk

cudaError_t launch_evict(const EvictArgs& a, int sms, cudaStream_t st)
{
    using namespace wk;
    cudaError_t e = allow_smem<k_evict>(MAX_KEYS * 4);
    if (e != cudaSuccess) return e;
    // CTAs for one (request, head): as many as fill the GPU once, at most the
    // portable cluster; few slots need no more than one
    const long long units = (long long)a.n_req * a.kv.kv_heads;
    int cs = 1;
    while (cs < 8 && units * cs * 2 <= 2ll * sms && a.kv.cap > 4096ll * cs) cs *= 2;
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
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_evict, a, max_keys);
}

}  // namespace aladdin
