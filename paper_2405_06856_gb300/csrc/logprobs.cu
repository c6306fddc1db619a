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
// The pass needs many bytes in flight and few instructions a logit: a thread has the
// next four vectors of 16 bytes on their way while it works on four; four vectors
// share one look at the maximum, and 16-bit logits are clamped and compared two in a
// word. (Two terms an instruction in the sums, or a ring in shared memory for the
// vectors, gained nothing.) Of an owner's vectors only the step that holds its best is
// read again, unless another step of it reaches the bound too.
//
// Measured: 777 rows of 128,256 bf16 logits with 20 alternatives 58 to 61 us (3.3 TB/s; 48 without
// alternatives), 2,049 rows of 50,257 f32 logits without alternatives 77 us (5.4 TB/s).
#include <cooperative_groups.h>

#include <type_traits>

#include "worker_dev.cuh"

namespace cg = cooperative_groups;

namespace aladdin {
namespace wk {
namespace {

constexpr int NT = 128;
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
// stay finite; a NaN stays one. A top of more than FAR in size has no such value (in f16, -65504
// less 1,024 is -inf), or the rounding of top log2 e leaves 2^(its rounding) out of range (in 32 bits it is 16
// at most up to 2^28): its row counts the entries equal to it, which leaves out e^-32 at most for each
// other one, as values of the type lie 32 or more apart there.
template <typename T>
struct Logit;
template <>
struct Logit<float> {
    static constexpr int PER = 4;
    static constexpr float FAR = 268435456.0f;
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
    // entries of the vectors above a threshold
    typedef float Thr;
    static __device__ __forceinline__ Thr thr(float v) { return v; }
    template <int U>
    static __device__ __forceinline__ int above(const uint4 (&w)[U], const Thr (&t)[U])
    {
        int n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u)
            n += (__uint_as_float(w[u].x) > t[u]) + (__uint_as_float(w[u].y) > t[u]) +
                 (__uint_as_float(w[u].z) > t[u]) + (__uint_as_float(w[u].w) > t[u]);
        return n;
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
    static constexpr float FAR = std::is_same<T, __half>::value ? 32768.0f : 268435456.0f;
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
    // (a threshold between two values of the type rounds down to the lower one; the counts of
    // 4 U words are whole numbers that the type holds)
    typedef Low Thr;
    static __device__ __forceinline__ Thr thr(float v) { return low(v); }
    template <int U>
    static __device__ __forceinline__ int above(const uint4 (&w)[U], const Thr (&t)[U])
    {
        Low n = low(0.0f);
#pragma unroll
        for (int u = 0; u < U; ++u)
            n = __hadd2(n, __hadd2(__hadd2(__hgt2(word(w[u].x), t[u]), __hgt2(word(w[u].y), t[u])),
                                   __hadd2(__hgt2(word(w[u].z), t[u]), __hgt2(word(w[u].w), t[u]))));
        const float2 f = Num<T>::unpack(bits(n));
        return (int)(f.x + f.y);
    }
    static __device__ __forceinline__ float one(const char* p)
    {
        return Num<T>::unpack(*reinterpret_cast<const unsigned short*>(p)).x;
    }
};

// The order of values as unsigned numbers (-0 as +0, NaN below everything), the next
// lower float of a finite value, and an entry as a number that orders entries: larger
// values first, the lower index first among equals.
__device__ __forceinline__ uint32_t ordered(float x)
{
    if (x != x) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float next_below(float x)
{
    const uint32_t o = ordered(x), u = o == 0x80000000u ? 0x7ffffffeu : o - 1;  // below +0: not -0
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ float value_of(uint32_t order)
{
    return order ? __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order) : NAN;
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
    int owner[NT];                            // threads that may hold one of the top k, and
    int at[NT];                               // the first vector of the only step that may, or -1
    Run run[NT / 32];
    int above[NT / 32];
    Run all;  // this slice's sums
    int all_above;
    int count, owners;
    int apart;  // owners that are left when equal maxima are told apart
    uint32_t bound;
    unsigned long long bound_entry, prev;
};

template <typename T>
__global__ void __launch_bounds__(NT, 8) k_logprobs(LogprobArgs a)
{
    using L = Logit<T>;
    constexpr int PER = L::PER, ES = 16 / PER, U = 4;  // logits of a vector, bytes of one, vectors a step
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
    // vectors in front of the token's count their entries from its value on, those behind it the
    // larger ones, and its own vector goes entry by entry (as all vectors do for a token of NaN
    // or -inf, of which the thresholds do not tell NaN from other entries)
    const bool plain = mine == mine && mine != -INFINITY;
    const int own_vec = plain && token >= head && token < tail0 ? (token - head) / PER : -1;
    const float from_value = next_below(mine);
    const typename L::Thr over = L::thr(mine), from = L::thr(from_value);
    const int split = plain ? token - head : 0;  // vectors v with v PER < split lie in front

    // The largest entry so far, and the sums s of 2^y and t of 2^y y, y = x log2 e - ref with ref =
    // m log2 e rounded: one multiply-add a logit, and the rounding of ref drops out of the results, as
    // every term and the conversion below have the same. Where |m| is more than FAR (a mask of the
    // type's lowest value, +inf), the sum counts the entries that equal m: all others are too far
    // away; `gate` is m, or NaN to have every vector looked at that way.
    float m = -INFINITY, ref = 0.0f, gate = -INFINITY;
    typename L::Low low = L::low(-200.0f);
    int above = 0;
    float s0 = 0.0f, s1 = 0.0f, t0 = 0.0f, t1 = 0.0f;  // (two sums each, by even and odd places)
    // the largest entries of a step and of the other steps, and the step's first vector
    float step1 = -INFINITY, step2 = -INFINITY;
    int step_v = 0;
    auto huge = [](float v) { return fabsf(v) > L::FAR; };
    auto raise = [&](float v) {
        const bool far = gate != gate || huge(v);
        const float next = far ? 0.0f : v * LOG2E, d = ref - next, f = far ? 0.0f : ex2(d);
        if (m != -INFINITY) {
            // (a NaN in a sum stays one)
            t0 = f == 0.0f ? t0 * 0.0f : f * fmaf(s0, d, t0);
            t1 = f == 0.0f ? t1 * 0.0f : f * fmaf(s1, d, t1);
            s0 *= f;
            s1 *= f;
        }
        m = v;
        ref = next;
        if (huge(v)) {
            gate = NAN;
        } else {
            ref = v * LOG2E;
            gate = v;
            low = L::low(v - fmaxf(200.0f, fabsf(v) * 0.015625f));
        }
    };
    auto count = [&](float v, int i) {  // one entry against the token
        const uint32_t o = ordered(v);
        above += o > mine_o || (o == mine_o && i < token);
    };
    auto look = [&](auto& w, int v, int step) {  // vectors v, v + step, ...
        constexpr int N = sizeof(w) / sizeof(uint4);
        float top = L::top(w[0]);
#pragma unroll
        for (int u = 1; u < N; ++u) top = fmaxf(top, L::top(w[u]));
        step2 = fmaxf(step2, fminf(step1, top));
        step_v = top > step1 ? v : step_v;
        step1 = fmaxf(step1, top);
        if (!(top <= gate) && top > m) raise(top);
        if (gate != gate) {
            float s = 0.0f;
#pragma unroll
            for (int u = 0; u < N; ++u) {
                float f[PER];
                L::unpack(w[u], f);
#pragma unroll
                for (int i = 0; i < PER; ++i) s += f[i] == m ? (m == INFINITY ? NAN : 1.0f) : f[i] == f[i] ? 0.0f : NAN;
            }
            s0 += s;
        } else {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                float f[PER];
                L::clamped(w[u], low, f);
#pragma unroll
                for (int i = 0; i < PER; i += 2) {
                    const float y0 = fmaf(f[i], LOG2E, -ref), y1 = fmaf(f[i + 1], LOG2E, -ref), e0 = ex2(y0),
                                e1 = ex2(y1);
                    s0 += e0;
                    s1 += e1;
                    t0 = fmaf(e0, y0, t0);
                    t1 = fmaf(e1, y1, t1);
                }
            }
        }
        if (ranked) {
            if (plain) {
                if (top > from_value) {  // (else nothing here stands in front of the token)
                    typename L::Thr thr[N];
#pragma unroll
                    for (int u = 0; u < N; ++u) thr[u] = (v + u * step) * PER < split ? from : over;
                    above += L::above(w, thr);
                }
            } else {
#pragma unroll
                for (int u = 0; u < N; ++u) {
                    float g[PER];
                    L::unpack(w[u], g);
#pragma unroll
                    for (int i = 0; i < PER; ++i) count(g[i], head + (v + u * step) * PER + i);
                }
            }
        }
    };
    {
        // this thread's vectors v0 + tid, v0 + tid + NT, ...
        const uint4* p = body + v0 + tid;
        int left = v0 + tid < v1 ? (v1 - v0 - tid + NT - 1) / NT : 0, v = v0 + tid;
        uint4 next[U];
        if (left >= U) {
#pragma unroll
            for (int u = 0; u < U; ++u) next[u] = __ldg(p + u * NT);
        }
#pragma unroll 1
        while (left >= U) {
            uint4 w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = next[u];
            left -= U;
            p += U * NT;
            if (left >= U) {
#pragma unroll
                for (int u = 0; u < U; ++u) next[u] = __ldg(p + u * NT);
            }
            look(w, v, NT);
            v += U * NT;
        }
#pragma unroll 1
        for (; left > 0; --left, p += NT, v += NT) {
            uint4 w[1] = {__ldg(p)};
            look(w, v, NT);
        }
    }
    if (ranked && own_vec >= v0 && own_vec < v1 && (own_vec - v0) % NT == tid) {
        // the token's own vector was counted with one threshold: once more, by entries
        uint4 w[1] = {__ldg(body + own_vec)};
        const typename L::Thr thr[1] = {own_vec * PER < split ? from : over};
        above -= L::above(w, thr);
        float g[PER];
        L::unpack(w[0], g);
#pragma unroll
        for (int i = 0; i < PER; ++i) count(g[i], head + own_vec * PER + i);
    }
    Run run{m, s0 + s1, t0 + t1};
    {
        if (m != -INFINITY && gate == gate) {
            const float y = fmaf(m, LOG2E, -ref), f = ex2(-y);  // y of the largest entry: almost 0
            run.t = fmaf(-y, run.s, run.t) * f * LN2;
            run.s *= f;
        }
    }
    if (ends >= 0) {
        if (end_x != -INFINITY) run = join(run, fabsf(end_x) < INFINITY ? Run{end_x, 1.0f, 0.0f} : Run{run.m, NAN, NAN});
        if (end_x > m) m = end_x;
        if (ranked) count(end_x, ends);
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
            sh.count = sh.owners = sh.apart = 0;
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
        if (holds && best >= bound) {
            const int o = atomicAdd(&sh.owners, 1);
            sh.owner[o] = tid;
            // (v1: none of its vectors does, but an end of the row)
            sh.at[o] = !bound || ordered(step2) >= bound ? -1 : ordered(step1) >= bound ? step_v : v1;
        }
        if (tid == 0) sh.bound_entry = (unsigned long long)bound << 32;
        __syncthreads();
        // (nothing writes sh.owners behind this barrier: all threads take the same side here)
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
            __syncthreads();
            int larger = 0;
            for (int i = 0; i < NT; ++i) larger += sh.best[i] > first;
            if (first && larger == k - 1) sh.bound_entry = first;
            __syncthreads();
            if (first >= sh.bound_entry && first) {
                const int o = atomicAdd(&sh.apart, 1);
                sh.owner[o] = tid;
                sh.at[o] = -1;
            }
            __syncthreads();
            owners = sh.apart;
        }
        const unsigned long long bound_entry = sh.bound_entry;
        auto keep = [&](unsigned long long e) {
            if (e >= bound_entry) {
                const int c = atomicAdd(&sh.count, 1);
                if (c < LIST) sh.list[c] = e;
            }
        };
        // the step of an owner that may hold entries that large (a warp would read all its vectors,
        // each in a line of its own, for the few owners that have two)
        const uint32_t least = (uint32_t)(bound_entry >> 32);
        const float least_value = value_of(least);
        auto vector = [&](int w) {
            const uint4 q = __ldg(body + w);
            if (least && !(L::top(q) >= least_value)) return;
            float g[PER];
            L::unpack(q, g);
#pragma unroll
            for (int j = 0; j < PER; ++j) keep(entry(ordered(g[j]), head + w * PER + j));
        };
        for (int i = tid; i < owners * U; i += NT) {
            const int w = sh.at[i / U] + i % U * NT;
            if (sh.at[i / U] >= 0 && w < v1) vector(w);
        }
        for (int i = warp; i < owners; i += NT / 32)
            if (sh.at[i] < 0)
#pragma unroll 2
                for (int w = v0 + sh.owner[i] + lane * NT; w < v1; w += 32 * NT) vector(w);
        if (ends >= 0) keep(entry(ordered(end_x), ends));
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
        // (the sums of the slices, by every thread that writes something: the first one only,
        // or, with alternatives, all)
        if (tid == 0 || k) {
            Run r = sh.all;
            for (int b = 1; b < cs; ++b) r = join(r, cluster.map_shared_rank(&sh, b)->all);
            const float ls = logf(r.s);
            if (tid == 0) {
                int c = sh.all_above;
                for (int b = 1; b < cs; ++b) c += cluster.map_shared_rank(&sh, b)->all_above;
                const bool empty = r.m == -INFINITY && r.s == 0.0f;  // every logit is -inf
                if (a.logprob) a.logprob[row] = given ? logprob_of(mine, r.m, ls) : NAN;
                if (a.entropy) a.entropy[row] = empty ? 0.0f : ls - r.t / r.s;
                if (a.rank) a.rank[row] = given ? c : ALADDIN_INVALID;
                if (a.token && !given) atomicOr(a.err, WORKER_BAD_INPUT);
            }
            auto put = [&](int place, unsigned long long e) {
                if (a.top_id) a.top_id[(long long)row * k + place] = (int)~(uint32_t)e;
                if (a.top_logprob)
                    a.top_logprob[(long long)row * k + place] = logprob_of(value_of((uint32_t)(e >> 32)), r.m, ls);
            };
            if (cs == 1) {
                if (tid < k) put(tid, sh.top[tid]);
            } else if (k) {  // (all threads are here)
                // the slices' bests, at most MAX_CS x ALADDIN_TOP_MAX entries, once more all with all
                const int all = cs * k;
                for (int c = tid; c < all; c += NT) sh.list[c] = cluster.map_shared_rank(&sh, c / k)->top[c % k];
                __syncthreads();
                for (int c = tid; c < all; c += NT) {
                    const unsigned long long e = sh.list[c];
                    if (!e) continue;
                    int larger = 0;
                    for (int i = 0; i < all; ++i) larger += sh.list[i] > e;
                    if (larger < k) put(larger, e);
                }
            }
        }
    }
    if (cs > 1) cluster.sync();  // the first CTA has read the others
}

template <typename T>
cudaError_t launch(const LogprobArgs& a, int sms, cudaStream_t st)
{
    const int vecs = a.vocab / Logit<T>::PER;
    // CTAs for a row: until the GPU has two a SM, with 1,024 vectors each at least. (Measured with
    // 777 rows of 128,256: 61 us with one CTA a row, 72 with two: a CTA's end costs more than
    // the even load gains.)
    int cs = 1;
    while (cs < MAX_CS && (long long)a.n * cs < 2ll * sms && vecs > 1024 * cs) cs *= 2;
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
