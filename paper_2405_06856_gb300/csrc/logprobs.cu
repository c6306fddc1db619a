// aladdin_worker_logprobs: log probabilities of given tokens, the entropy of
// their rows, the tokens' ranks and the top alternatives.
//
// For a row x of V logits, with m = max x, S = sum e^(x - m):
//     logprob = x_t - m - log S,   entropy = log S - (sum e^(x - m) (x - m)) / S,
//     rank = #{x > x_t} + #{x = x_t, lower index},
//     the top k in descending order, the lower index first among equals.
// A cluster of CTAs serves one row, each CTA a slice of the vocabulary: one
// pass over the logits with a running maximum in 32 bits, which also keeps the
// slice in shared memory where alternatives are asked for. A thread's best
// entry bounds the k-th best of the slice from below (the k-th largest of the
// threads' bests does), so the second look at the slice keeps a few entries,
// which a comparison of all with all sorts.
#include <cooperative_groups.h>

#include "worker_dev.cuh"

namespace cg = cooperative_groups;

namespace aladdin {
namespace wk {
namespace {

constexpr int NT = 256;
constexpr int LIST = 1024;  // entries of a slice that the second look may keep
constexpr int MAX_CS = 8;

template <typename T>
struct Logit;
template <>
struct Logit<float> {
    static constexpr int PER = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[4])
    {
        x[0] = __uint_as_float(v.x);
        x[1] = __uint_as_float(v.y);
        x[2] = __uint_as_float(v.z);
        x[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ float one(const char* p) { return *reinterpret_cast<const float*>(p); }
};
template <typename T>
struct Logit {
    static constexpr int PER = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&x)[8])
    {
        const float2 a = Num<T>::unpack(v.x), b = Num<T>::unpack(v.y), c = Num<T>::unpack(v.z),
                     d = Num<T>::unpack(v.w);
        x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
    }
    static __device__ __forceinline__ float one(const char* p)
    {
        return Num<T>::unpack(*reinterpret_cast<const unsigned short*>(p)).x;
    }
};

// An entry as a number that orders entries: larger values first, the lower
// index first among equals; -0 counts as +0 and NaN lies below everything. No
// entry is 0.
__device__ __forceinline__ uint32_t ordered(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ unsigned long long entry(float x, int i)
{
    return (unsigned long long)ordered(x) << 32 | (uint32_t)~i;
}

// Running maximum m, sum s of e^(x - m) and sum t of e^(x - m) (x - m). A row or
// part without an entry has m = -inf, s = t = 0. The difference is formed before
// it is scaled to base 2: rows of the type's lowest value (a mask) stay finite,
// and a difference that overflows is -inf, whose exponential is 0.
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

__device__ __forceinline__ void add(Run& a, float v)  // v <= a.m, a.m finite
{
    const float d = v - a.m, e = ex2(d * LOG2E);
    a.s += e;
    a.t += e == 0.0f ? 0.0f : e * d;
}

// x - m - log S; -inf for a logit of -inf unless the row has NaN or +inf.
__device__ __forceinline__ float logprob_of(float x, float m, float ls)
{
    return x == -INFINITY && ls == ls ? -INFINITY : x - m - ls;
}

struct Shared {
    unsigned long long best[NT];
    unsigned long long list[LIST];
    unsigned long long top[ALADDIN_TOP_MAX];  // of this slice, best first
    Run run[NT / 32];
    int above[NT / 32];
    Run all;        // this slice's sums
    int all_above;
    int count;
    unsigned long long bound, prev;
    float m, ls;  // the row's maximum and log S
};

template <typename T>
__global__ void __launch_bounds__(NT) k_logprobs(LogprobArgs a, int keeps)
{
    using L = Logit<T>;
    constexpr int PER = L::PER, ES = 16 / PER;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ __align__(16) uint4 slice[];  // this slice's vectors, thread by thread
    __shared__ Shared sh;
    const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int row = blockIdx.x / cs, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const char* const x = a.x + (long long)row * a.stride * ES;
    const int k = a.top;

    // the slice [e0, e1): whole vectors of 16 aligned bytes but at the row's ends
    const int head = min(a.vocab, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / ES));
    const int vecs = (a.vocab - head) / PER, tail0 = head + vecs * PER;
    const int per = (vecs + cs - 1) / cs, v0 = min(rank * per, vecs), v1 = min(v0 + per, vecs);
    const uint4* const body = reinterpret_cast<const uint4*>(x + head * ES);
    const uint4* const again = keeps ? slice : body + v0;  // where the second look reads
    // the ends, fewer than PER each, go to the last CTA's first threads
    int ends = -1;
    if (rank == cs - 1) {
        if (tid < head) ends = tid;
        else if (tid >= 32 && tail0 + tid - 32 < a.vocab && tid < 64) ends = tail0 + tid - 32;
    }
    const float end_x = ends >= 0 ? L::one(x + (long long)ends * ES) : 0.0f;

    const int token = a.token ? a.token[row] : -1;
    const bool given = token >= 0 && token < a.vocab;
    const float mine = given ? L::one(x + (long long)token * ES) : 0.0f;
    const unsigned long long mine_e = entry(mine, token);

    Run run{-INFINITY, 0.0f, 0.0f};
    bool nan = false;
    int above = 0;
    unsigned long long best = 0;
    auto look = [&](float v, int i) {
        if (v > run.m) rebase(run, v);
        if (v != v) nan = true;
        else if (v != -INFINITY) {
            if (run.m == INFINITY) nan = true;  // as the formula's inf - inf
            else add(run, v);
        }
        const unsigned long long e = entry(v, i);
        above += e > mine_e;
        best = e > best ? e : best;
    };
    for (int v = v0 + tid; v < v1; v += NT) {
        const uint4 w = __ldg(body + v);
        if (keeps) slice[v - v0] = w;
        float f[PER];
        L::unpack(w, f);
#pragma unroll
        for (int i = 0; i < PER; ++i) look(f[i], head + v * PER + i);
    }
    if (ends >= 0) look(end_x, ends);
    if (nan) run = Run{run.m, NAN, NAN};

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
    sh.best[tid] = best;
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (tid == 0) {
        Run r = sh.run[0];
        int c = sh.above[0];
        for (int w = 1; w < NT / 32; ++w) {
            r = join(r, sh.run[w]);
            c += sh.above[w];
        }
        sh.all = r;
        sh.all_above = c;
    }

    const int mine_n = (v1 - v0) * PER + (rank == cs - 1 ? head + a.vocab - tail0 : 0);  // entries of the slice
    const int kk = min(k, mine_n);
    if (k) {
        // the k-th largest of the threads' bests; 0 (every entry) where fewer threads have one
        int larger = 0;
        for (int i = 0; i < NT; ++i) larger += sh.best[i] > best;
        if (tid == 0) sh.bound = 0;
        __syncthreads();
        if (best && larger == k - 1) sh.bound = best;
        __syncthreads();
        const unsigned long long bound = sh.bound;
        auto keep = [&](unsigned long long e) {
            if (e >= bound) {
                const int c = atomicAdd(&sh.count, 1);
                if (c < LIST) sh.list[c] = e;
            }
        };
        if (best >= bound) {  // else this thread has nothing to keep
            for (int v = v0 + tid; v < v1; v += NT) {
                float f[PER];
                L::unpack(again[v - v0], f);
#pragma unroll
                for (int i = 0; i < PER; ++i) keep(entry(f[i], head + v * PER + i));
            }
            if (ends >= 0) keep(entry(end_x, ends));
        }
        __syncthreads();
        const int count = sh.count;
        if (count <= LIST) {
            for (int c = tid; c < count; c += NT) {
                const unsigned long long e = sh.list[c];
                int larger2 = 0;
                for (int i = 0; i < count; ++i) larger2 += sh.list[i] > e;
                if (larger2 < kk) sh.top[larger2] = e;
            }
        } else {
            // a few threads hold nearly everything large: the slice's best below the
            // one before, kk times
            unsigned long long prev = ~0ull;
            for (int c = 0; c < kk; ++c) {
                unsigned long long b = 0;
                for (int v = v0 + tid; v < v1; v += NT) {
                    float f[PER];
                    L::unpack(again[v - v0], f);
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const unsigned long long e = entry(f[i], head + v * PER + i);
                        if (e < prev && e > b) b = e;
                    }
                }
                if (ends >= 0) {
                    const unsigned long long e = entry(end_x, ends);
                    if (e < prev && e > b) b = e;
                }
                __syncthreads();
                sh.best[tid] = b;
                __syncthreads();
                if (warp == 0) {
                    for (int i = lane; i < NT; i += 32) b = sh.best[i] > b ? sh.best[i] : b;
#pragma unroll
                    for (int o = 16; o; o >>= 1) {
                        const unsigned long long u = __shfl_xor_sync(0xffffffffu, b, o);
                        b = u > b ? u : b;
                    }
                    if (lane == 0) sh.prev = sh.top[c] = b;
                }
                __syncthreads();
                prev = sh.prev;
            }
        }
        for (int c = kk + tid; c < k; c += NT) sh.top[c] = 0;
    }
    cluster.sync();
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
        __syncthreads();
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
    cluster.sync();
}

template <typename T>
cudaError_t launch(const LogprobArgs& a, int sms, cudaStream_t st)
{
    constexpr int LIMIT = 200 * 1024;
    cudaError_t e = allow_smem<k_logprobs<T>>(LIMIT);
    if (e != cudaSuccess) return e;
    constexpr int PER = Logit<T>::PER;
    const int vecs = a.vocab / PER;
    // CTAs for a row: few rows share the GPU (a CTA with fewer than 1,024 vectors
    // would wait more than it reads); a slice that is kept has to fit
    int cs = 1;
    while (cs < MAX_CS && ((long long)a.n * cs * 2 <= 2ll * sms && vecs > 1024 * cs)) cs *= 2;
    if (a.top)
        while (cs < MAX_CS && (vecs + cs - 1) / cs * 16 > LIMIT / 2) cs *= 2;
    const int bytes = (vecs + cs - 1) / cs * 16;
    const int smem = a.top && bytes <= LIMIT ? bytes : 0;
    cudaLaunchConfig_t c = {};
    c.gridDim = dim3((unsigned)a.n * cs);
    c.blockDim = dim3(NT);
    c.dynamicSmemBytes = (size_t)smem;
    c.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cs;
    at[0].val.clusterDim.y = 1;
    at[0].val.clusterDim.z = 1;
    c.attrs = at;
    c.numAttrs = 1;
    return cudaLaunchKernelEx(&c, k_logprobs<T>, a, (int)(smem > 0));
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
