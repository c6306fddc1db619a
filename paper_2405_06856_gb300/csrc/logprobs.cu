// aladdin_worker_logprobs: log probabilities of given tokens, the entropy of
// their rows, the tokens' ranks and the top alternatives.
//
// For a row x of V logits, with m = max x, S = sum e^(x - m):
//     logprob = x_t - m - log S,   entropy = log S - (sum e^(x - m) (x - m)) / S,
//     rank = #{x > x_t} + #{x = x_t, lower index},
//     the top k in descending order, the lower index first among equals.
// A cluster of CTAs serves one row, each CTA a slice of the vocabulary, in one
// pass with a running maximum and 32-bit sums in every thread. The pass also
// leaves every thread's largest entry: the k-th largest of the maxima of groups
// of threads bounds the k-th best of the slice from below, so only the few
// threads that reach it can hold one of the top k. Their entries are read again
// (from L2), those at or above the bound are kept, and a comparison of all kept
// ones with all others sorts them.
//
// The pass is bound by its instructions: two 16-bit logits are unpacked,
// clamped and compared in a word, the sums take two terms an instruction.
#include <cooperative_groups.h>

#include <type_traits>

#include "worker_dev.cuh"

namespace cg = cooperative_groups;

namespace aladdin {
namespace wk {
namespace {

constexpr int NT = 256;
constexpr int LIST = 1024;   // entries of a slice that the second look may keep
constexpr int MAX_CS = 8;
constexpr int MANY = 32;     // threads over the top k from which equal entries are told apart first

__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// How a vector of 16 bytes of logits is taken apart. low() is what top - 200 or
// less looks like in the type (at least a step below top): entries below it
// count as it, since both exponentials are 0, so that products with differences
// stay finite; a NaN stays one.
template <typename T>
struct Logit;
template <>
struct Logit<float> {
    static constexpr int PER = 4;
    typedef float Low;
    static __device__ __forceinline__ Low low(float v) { return v; }
    static __device__ __forceinline__ float top(const uint4& v)
    {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)),
                     fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4])
    {
        x[0] = __uint_as_float(v.x), x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z), x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ void clamped(const uint4& v, Low low, float (&x)[4])
    {
        unpack(v, x);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = max_nan(x[i], low);
    }
    static __device__ __forceinline__ float one(const char* p) { return *reinterpret_cast<const float*>(p); }
};
__device__ __forceinline__ __nv_bfloat162 both(__nv_bfloat162*, float v)
{
    return __bfloat162bfloat162(__float2bfloat16_rd(v));
}
__device__ __forceinline__ __half2 both(__half2*, float v) { return __half2half2(__float2half_rd(v)); }
template <typename T>
struct Logit {
    static constexpr int PER = 8;
    typedef typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type Low;
    static __device__ __forceinline__ Low low(float v) { return both((Low*)nullptr, v); }
    static __device__ __forceinline__ Low word(uint32_t w) { return *reinterpret_cast<Low*>(&w); }
    static __device__ __forceinline__ uint32_t bits(Low w) { return *reinterpret_cast<uint32_t*>(&w); }
    static __device__ __forceinline__ float top(const uint4& v)
    {
        const Low m = __hmax2(__hmax2(word(v.x), word(v.y)), __hmax2(word(v.z), word(v.w)));
        const float2 f = Num<T>::unpack(bits(m));
        return fmaxf(f.x, f.y);
    }
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8])
    {
        const float2 a = Num<T>::unpack(v.x), b = Num<T>::unpack(v.y), c = Num<T>::unpack(v.z),
                     d = Num<T>::unpack(v.w);
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
    }
    static __device__ __forceinline__ void clamped(const uint4& v, Low low, float (&x)[8])
    {
        const uint4 w = make_uint4(bits(__hmax2_nan(word(v.x), low)), bits(__hmax2_nan(word(v.y), low)),
                                   bits(__hmax2_nan(word(v.z), low)), bits(__hmax2_nan(word(v.w), low)));
        unpack(w, x);
    }
    static __device__ __forceinline__ float one(const char* p)
    {
        return Num<T>::unpack(*reinterpret_cast<const unsigned short*>(p)).x;
    }
};

// The order of values as unsigned numbers (-0 as +0, NaN below everything), the
// value's next lower float, and an entry as a number that orders entries: larger
// values first, the lower index first among equals.
__device__ __forceinline__ uint32_t ordered(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float next_below(float x)  // x not NaN; -inf gives NaN, above which nothing is
{
    const uint32_t o = ordered(x), u = o == 0x80000000u ? 0x7ffffffeu : o - 1;  // below +0: not -0
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ unsigned long long entry(uint32_t order, int i)
{
    return (unsigned long long)order << 32 | (uint32_t)~i;
}

// Maximum m, sum s of e^(x - m) and sum t of e^(x - m) (x - m). A row or part
// without an entry above -inf has m = -inf, s = t = 0.
struct Run {
    float m, s, t;
};

__device__ __forceinline__ void rebase(Run& a, float m)  // m >= a.m
{
    if (a.m == -INFINITY) {
        a.m = m;
        return;
    }
    const float d = a.m - m, f = ex2(d * LOG2E);
    // e^(x - m) (x - m) = f e^(x - a.m) (x - a.m + d)
    a.t = f == 0.0f ? 0.0f : f * fmaf(a.s, d, a.t);
    a.s *= f;
    a.m = m;
}

__device__ __forceinline__ Run join(Run a, Run b)
{
    const float m = fmaxf(a.m, b.m);
    if (m > a.m) rebase(a, m);
    if (m > b.m) rebase(b, m);
    return Run{m, a.s + b.s, a.t + b.t};
}

// x - m - log S; -inf for a logit of -inf unless the row has NaN or +inf.
__device__ __forceinline__ float logprob_of(float x, float m, float ls)
{
    return x == -INFINITY && ls == ls ? -INFINITY : x - m - ls;
}

struct alignas(16) Shared {
    uint32_t group[NT / 2];
    unsigned long long best[NT];
    unsigned long long list[LIST];
    unsigned long long top[ALADDIN_TOP_MAX];  // of this slice, best first
    int owner[NT];                            // threads that may hold one of the top k
    Run run[NT / 32];
    int above[NT / 32];
    Run all;  // this slice's sums
    int all_above;
    int count, owners;
    uint32_t bound;
    unsigned long long bound_entry, prev;
    float m, ls;  // the row's maximum and log S
};

template <typename T>
__global__ void __launch_bounds__(NT, 4) k_logprobs(LogprobArgs a)
{
    using L = Logit<T>;
    constexpr int PER = L::PER, ES = 16 / PER, U = 4;  // logits of a vector, bytes of one, vectors in flight
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ Shared sh;
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / cs, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const char* const x = a.x + (long long)row * a.stride * ES;
    const int k = a.top;

    // the slice: whole vectors of 16 aligned bytes; the row's ends, fewer than PER
    // entries each, go to the last CTA's first threads
    const int head = min(a.vocab, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / ES));
    const int vecs = (a.vocab - head) / PER, tail0 = head + vecs * PER;
    const int per = (vecs + cs - 1) / cs, v0 = min(rank * per, vecs), v1 = min(v0 + per, vecs);
    const uint4* const body = reinterpret_cast<const uint4*>(x + head * ES);
    int ends = -1;
    if (rank == cs - 1) {
        if (tid < head) ends = tid;
        else if (tid >= 32 && tail0 + tid - 32 < a.vocab && tid < 64) ends = tail0 + tid - 32;
    }
    const float end_x = ends >= 0 ? L::one(x + (long long)ends * ES) : -INFINITY;

    const int token = a.token ? a.token[row] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float mine = given ? L::one(x + (long long)token * ES) : 0.0f;
    const bool ranked = given && a.rank;
    const uint32_t mine_o = ordered(mine);
    // entries in front of the token count from its value on, those behind it from above it
    // (a token of NaN stands behind all values: they count from -inf on)
    const float over = mine != mine ? __uint_as_float(0xffffffffu) : mine;
    const float from = mine != mine ? over : next_below(mine);

    float m = -INFINITY, ref = 0.0f;  // the largest entry so far; what differences are taken to
    typename L::Low low = L::low(-200.0f);
    f2 s2 = pair(0.0f, 0.0f), t2 = s2, minus = s2;
    const f2 log2e = pair(LOG2E, LOG2E);
    int above = 0;
    auto raise = [&](float v) {
        if (m != -INFINITY) {
            float sl, sh_, tl, th;
            unpair(s2, sl, sh_);
            unpair(t2, tl, th);
            const float d = ref - v, f = ex2(d * LOG2E);
            s2 = pair(sl * f, sh_ * f);
            t2 = f == 0.0f && sl == sl && sh_ == sh_ ? pair(0.0f, 0.0f)
                                                     : pair(f * fmaf(sl, d, tl), f * fmaf(sh_, d, th));
        }
        m = ref = v;
        minus = pair(-v, -v);
        low = L::low(v - fmaxf(200.0f, fabsf(v) * 0.015625f));
    };
    auto count = [&](float v, int i) {  // one entry against the token
        const uint32_t o = ordered(v);
        above += o > mine_o || (o == mine_o && i < token);
    };
    auto look = [&](const uint4& w, int v) {
        const float top = L::top(w);
        if (top > m) raise(top);
        float f[PER];
        L::clamped(w, low, f);
#pragma unroll
        for (int i = 0; i < PER; i += 2) {
            const f2 d = add2(pair(f[i], f[i + 1]), minus), y = mul2(d, log2e);
            float y0, y1;
            unpair(y, y0, y1);
            const f2 e = pair(ex2(y0), ex2(y1));
            s2 = add2(s2, e);
            t2 = fma2(e, d, t2);
        }
        if (ranked) {
            const int i0 = head + v * PER;
            if (mine != mine || (i0 <= token && token < i0 + PER)) {
                float g[PER];
                L::unpack(w, g);
#pragma unroll
                for (int i = 0; i < PER; ++i) count(g[i], i0 + i);
            } else {
                // clamping keeps the order where the bound is not clamped away; the plain
                // values are compared
                const float thr = i0 < token ? from : over;
                float g[PER];
                L::unpack(w, g);
                if (thr != thr) {  // in front of a token of -inf: everything but NaN
#pragma unroll
                    for (int i = 0; i < PER; ++i) above += g[i] == g[i];
                } else {
#pragma unroll
                    for (int i = 0; i < PER; ++i) above += g[i] > thr;
                }
            }
        }
    };
    int v = v0 + tid;
    for (; v + (U - 1) * NT < v1; v += U * NT) {
        uint4 w[U];
#pragma unroll
        for (int i = 0; i < U; ++i) w[i] = __ldg(body + v + i * NT);
#pragma unroll
        for (int i = 0; i < U; ++i) look(w[i], v + i * NT);
    }
    for (; v < v1; v += NT) look(__ldg(body + v), v);
    if (ends >= 0) {
        if (end_x > m) raise(end_x);
        float d = end_x - ref;
        d = d < -200.0f ? -200.0f : d;  // a NaN stays
        const float e = ex2(d * LOG2E);
        s2 = add2(s2, pair(e, 0.0f));
        t2 = fma2(pair(e, 0.0f), pair(d, 0.0f), t2);
        if (ranked) count(end_x, ends);
    }
    Run run;
    {
        float sl, sh_, tl, th;
        unpair(s2, sl, sh_);
        unpair(t2, tl, th);
        run = Run{m, sl + sh_, tl + th};
    }
    const bool holds = v0 + tid < v1 || ends >= 0;  // this thread has entries

    // the slice's sums
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        Run b;
        b.m = __shfl_xor_sync(0xffffffffu, run.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, run.s, o);
        b.t = __shfl_xor_sync(0xffffffffu, run.t, o);
        // both lanes join in the same order
        run = lane & o ? join(b, run) : join(run, b);
        above += __shfl_xor_sync(0xffffffffu, above, o);
    }
    if (lane == 0) {
        sh.run[warp] = run;
        sh.above[warp] = above;
    }
    const int mine_n = (v1 - v0) * PER + (rank == cs - 1 ? head + a.vocab - tail0 : 0);  // entries of the slice
    const int kk = min(k, mine_n);
    // (of -inf and NaN only: none, which is no more than the truth)
    const uint32_t best = m != -INFINITY ? ordered(m) : 0u;
    // groups of 4 or 2 threads: more of them than k
    const int width = k <= NT / 8 ? 4 : 2, groups = NT / width;
    if (k) {
        uint32_t g = max(best, __shfl_xor_sync(0xffffffffu, best, 1));
        if (width == 4) g = max(g, __shfl_xor_sync(0xffffffffu, g, 2));
        if (tid % width == 0) sh.group[tid / width] = g;
        if (tid == 0) {
            sh.bound = 0;
            sh.count = sh.owners = 0;
        }
    }
    __syncthreads();
    if (warp == NT / 32 - 1) {  // (the other warps go on)
        Run r = lane < NT / 32 ? sh.run[lane] : Run{-INFINITY, 0.0f, 0.0f};
        int c = lane < NT / 32 ? sh.above[lane] : 0;
#pragma unroll
        for (int o = NT / 64; o; o >>= 1) {
            Run b;
            b.m = __shfl_xor_sync(0xffffffffu, r.m, o);
            b.s = __shfl_xor_sync(0xffffffffu, r.s, o);
            b.t = __shfl_xor_sync(0xffffffffu, r.t, o);
            r = lane & o ? join(b, r) : join(r, b);
            c += __shfl_xor_sync(0xffffffffu, c, o);
        }
        if (lane == 0) {
            sh.all = r;
            sh.all_above = c;
        }
    }

    if (k) {
        if (tid < groups) {
            const uint32_t g = sh.group[tid];
            int larger = 0;
            for (int i = 0; i < groups; i += 4) {
                const uint4 q = *reinterpret_cast<const uint4*>(sh.group + i);
                larger += (q.x > g || (q.x == g && i < tid)) + (q.y > g || (q.y == g && i + 1 < tid)) +
                          (q.z > g || (q.z == g && i + 2 < tid)) + (q.w > g || (q.w == g && i + 3 < tid));
            }
            if (larger == k - 1) sh.bound = g;
        }
        __syncthreads();
        const uint32_t bound = sh.bound;
        // the entries of thread `own`, to all lanes of a warp: f(order, index)
        auto entries_of = [&](int own, auto f) {
            const int n = own < v1 - v0 ? (v1 - v0 - own + NT - 1) / NT : 0;
            for (int i = lane; i < n; i += 32) {
                const int w = v0 + own + i * NT;
                float g[PER];
                L::unpack(__ldg(body + w), g);
#pragma unroll
                for (int j = 0; j < PER; ++j) f(ordered(g[j]), head + w * PER + j);
            }
            if (rank == cs - 1 && lane == 0) {
                int e = -1;
                if (own < head) e = own;
                else if (own >= 32 && own < 64 && tail0 + own - 32 < a.vocab) e = tail0 + own - 32;
                if (e >= 0) f(ordered(L::one(x + (long long)e * ES)), e);
            }
        };
        if (holds && best >= bound) sh.owner[atomicAdd(&sh.owners, 1)] = tid;
        if (tid == 0) sh.bound_entry = (unsigned long long)bound << 32;
        __syncthreads();
        int owners = sh.owners;
        if (owners > k + MANY) {
            // many equal maxima (a row of masked or equal logits): the first entry of
            // every thread's maximum tells them apart
            unsigned long long first = 0;
            if (holds && best >= bound) {
                const uint32_t is = ordered(m);
                for (int w = v0 + tid; w < v1 && !first; w += NT) {
                    float g[PER];
                    L::unpack(__ldg(body + w), g);
#pragma unroll
                    for (int j = PER - 1; j >= 0; --j)
                        if (ordered(g[j]) == is) first = entry(is, head + w * PER + j);
                }
                if (ends >= 0 && ordered(end_x) == is) first = max(first, entry(is, ends));
                if (!first) {  // NaN only
                    if (v0 + tid < v1) first = entry(0, head + (v0 + tid) * PER);
                    if (ends >= 0) first = max(first, entry(0, ends));
                }
            }
            sh.best[tid] = first;
            if (tid == 0) sh.owners = 0;
            __syncthreads();
            int larger = 0;
            for (int i = 0; i < NT; ++i) larger += sh.best[i] > first;
            if (first && larger == k - 1) sh.bound_entry = first;
            __syncthreads();
            if (first >= sh.bound_entry && first) sh.owner[atomicAdd(&sh.owners, 1)] = tid;
            __syncthreads();
            owners = sh.owners;
        }
        const unsigned long long bound_entry = sh.bound_entry;
        for (int i = warp; i < owners; i += NT / 32) {
            entries_of(sh.owner[i], [&](uint32_t o, int idx) {
                const unsigned long long e = entry(o, idx);
                if (e >= bound_entry) {
                    const int c = atomicAdd(&sh.count, 1);
                    if (c < LIST) sh.list[c] = e;
                }
            });
        }
        __syncthreads();
        const int count = sh.count;
        if (count <= LIST) {
            for (int c = tid; c < count; c += NT) {
                const unsigned long long e = sh.list[c];
                int larger = 0;
                for (int i = 0; i < count; ++i) larger += sh.list[i] > e;
                if (larger < kk) sh.top[larger] = e;
            }
        } else {
            // a few threads hold nearly everything large: the slice's best below the one
            // before, kk times
            unsigned long long prev = ~0ull;
            for (int c = 0; c < kk; ++c) {
                unsigned long long b = 0;
                for (int w = v0 + tid; w < v1; w += NT) {
                    float g[PER];
                    L::unpack(__ldg(body + w), g);
#pragma unroll
                    for (int j = 0; j < PER; ++j) {
                        const unsigned long long e = entry(ordered(g[j]), head + w * PER + j);
                        if (e < prev && e > b) b = e;
                    }
                }
                if (ends >= 0) {
                    const unsigned long long e = entry(ordered(end_x), ends);
                    if (e < prev && e > b) b = e;
                }
                __syncthreads();
                sh.best[tid] = b;
                __syncthreads();
                if (warp == 0) {
                    for (int i = lane; i < NT; i += 32) b = max(b, sh.best[i]);
#pragma unroll
                    for (int o = 16; o; o >>= 1) b = max(b, __shfl_xor_sync(0xffffffffu, b, o));
                    if (lane == 0) sh.prev = sh.top[c] = b;
                }
                __syncthreads();
                prev = sh.prev;
            }
        }
        for (int c = kk + tid; c < k; c += NT) sh.top[c] = 0;
    }
    if (cs > 1) cluster.sync();
    else __syncthreads();
    if (rank == 0) {
        if (tid == 0) {
            Run r = sh.all;
            int c = sh.all_above;
            for (int b = 1; b < cs; ++b) {
                const Shared* o = cluster.map_shared_rank(&sh, b);
                r = join(r, o->all);
                c += o->all_above;
            }
            const bool empty = r.m == -INFINITY && r.s == 0.0f;  // every logit is -inf
            sh.m = r.m;
            sh.ls = logf(r.s);
            if (a.logprob) a.logprob[row] = given ? logprob_of(mine, r.m, sh.ls) : NAN;
            if (a.entropy) a.entropy[row] = empty ? 0.0f : sh.ls - r.t / r.s;
            if (a.rank) a.rank[row] = given ? c : ALADDIN_INVALID;
            if (a.token && !given) atomicOr(a.err, WORKER_BAD_INPUT);
        }
        if (k) {
            // the slices' bests, at most MAX_CS x ALADDIN_TOP_MAX entries, once more all with all
            const int all = cs * k;
            for (int c = tid; c < all; c += NT) sh.list[c] = cluster.map_shared_rank(&sh, c / k)->top[c % k];
            __syncthreads();
            for (int c = tid; c < all; c += NT) {
                const unsigned long long e = sh.list[c];
                if (!e) continue;
                int larger = 0;
                for (int i = 0; i < all; ++i) larger += sh.list[i] > e;
                if (larger >= k) continue;
                const int id = (int)~(uint32_t)e;
                if (a.top_id) a.top_id[(long long)row * k + larger] = id;
                if (a.top_logprob)
                    a.top_logprob[(long long)row * k + larger] =
                        logprob_of(L::one(x + (long long)id * ES), sh.m, sh.ls);
            }
        }
    }
    if (cs > 1) cluster.sync();  // the first CTA has read the others
}

template <typename T>
cudaError_t launch(const LogprobArgs& a, int sms, cudaStream_t st)
{
    const int vecs = a.vocab / Logit<T>::PER;
    // CTAs for a row: enough that the GPU is filled several times over, so that its last
    // part is short, but with 1,024 vectors at least, four a thread
    int cs = 1;
    while (cs < MAX_CS && (long long)a.n * cs < 16ll * sms && vecs > 1024 * cs) cs *= 2;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)a.n * cs);
    c.blockDim = dim3(NT);
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_logprobs<T>, a);
}

}  // namespace
}  // namespace wk

cudaError_t launch_logprobs(const LogprobArgs& a, int dtype, int sms, cudaStream_t st)
{
    switch (dtype) {
        case ALADDIN_BF16: return wk::launch<__nv_bfloat16>(a, sms, st);
        case ALADDIN_F16: return wk::launch<__half>(a, sms, st);
        case ALADDIN_F32: return wk::launch<float>(a, sms, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace aladdin
