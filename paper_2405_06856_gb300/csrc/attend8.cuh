// aladdin_worker_attend8: what its kernels share.
//
// As aladdin_worker_attend (attend.cuh), over cached keys and values of 8 bits: k_j = c_j a_b, v_j = d_j e_b with
// e4m3 codes c, d and scales a, e of the block b that slot j lies in, so that
//     s_j = (scale a_b) q . c_j,      out = sum_j (e^(s_j - lse) e_b) d_j.
// Codes are exact in half precision, and so are queries of it. Queries of bfloat16 are multiplied by a power of two
// for each row that brings its largest channel to 2^14 .. 2^15: half precision then holds every channel above 2^-28
// of the largest without loss. Products and sums are 32-bit, and the scales and the row's power multiply the sums.
//
// The second product's weights e^(s_j - m) e_b are rounded to half precision (2^-12 of each, below 2^-14 of the
// largest 2^-25 of that). For them to fit, results count in units of 2^ref: ref is the logarithm of a block's
// scale, changed (and the results so far with it) where one comes that is more than 2^4 times as large, and the weight's
// exponent takes the difference in, for nothing. Scales below 2^-40 of the reference count as that much, of
// which half precision makes 0 again.
#pragma once

#include "attend.cuh"

namespace aladdin {
namespace wk {

// Two half-precision values of the two e4m3 codes in the lower (upper) half of a word.
__device__ __forceinline__ uint32_t half2_lo(uint32_t u)
{
    uint32_t h;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, lo;\n}" : "=r"(h) : "r"(u));
    return h;
}
__device__ __forceinline__ uint32_t half2_hi(uint32_t u)
{
    uint32_t h;
    asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.rn.f16x2.e4m3x2 %0, hi;\n}" : "=r"(h) : "r"(u));
    return h;
}

// The power of two that bfloat16 values of which `top` is the largest exponent field are multiplied by, and the one
// that takes it back.
__device__ __forceinline__ float half_factor(int top) { return __uint_as_float((uint32_t)(268 - min(max(top, 15), 254)) << 23); }
__device__ __forceinline__ float half_back(int top) { return __uint_as_float((uint32_t)(min(max(top, 15), 254) - 14) << 23); }

// The largest exponent field of two bfloat16 values and `top`.
__device__ __forceinline__ int exponent(uint32_t w, int top) { return max(top, max((int)(w >> 7 & 0xff), (int)(w >> 23 & 0xff))); }
__device__ __forceinline__ uint32_t to_half(uint32_t w, float f)
{
    const float2 v = Num<__nv_bfloat16>::unpack(w);
    return Num<__half>::pack(v.x * f, v.y * f);
}

// A row of queries, 4 lanes together, to half precision; returns what its scores are multiplied by.
template <typename T, int N>
__device__ __forceinline__ float half_row(uint2 (&q)[N])
{
    if constexpr (std::is_same<T, __half>::value) return 1.0f;
    int top = 0;
#pragma unroll
    for (int x = 0; x < N; ++x) top = exponent(q[x].y, exponent(q[x].x, top));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const float f = half_factor(top);
#pragma unroll
    for (int x = 0; x < N; ++x) q[x] = make_uint2(to_half(q[x].x, f), to_half(q[x].y, f));
    return half_back(top);
}

// Logarithm of a block's scale: -inf of 0, NaN of what is none.
__device__ __forceinline__ float log_scale(float v) { return v >= 0.0f && v < INFINITY ? __log2f(v) : NAN; }
// ... relative to the reference
__device__ __forceinline__ float relative(float lv, float ref)
{
    return lv == -INFINITY || lv - ref < -40.0f ? -40.0f : lv - ref;
}

// The tokens that token t of the request under u sees, itself among them; all lanes together, each its own t. A
// parent that is not an earlier token counts as none and is recorded. (A lane holds two tokens; every round joins what a
// token sees with what the one at the end of it sees: the walk up by loads, one after the other, took 10 times as long.)
__device__ __forceinline__ unsigned long long all_ancestors(const AttendArgs& a, const Cursor& u, int t, int lane)
{
    int up[2];
    unsigned long long see[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int i = e * 32 + lane;
        up[e] = i >= u.T ? -1 : a.tok.parent ? a.tok.parent[u.lo + i] : i - 1;
        if (up[e] < -1 || up[e] >= i) {
            atomicOr(a.err, WORKER_BAD_INPUT);
            up[e] = -1;
        }
        see[e] = 1ull << i;
    }
    const auto of = [&](int i) {
        const unsigned long long x = __shfl_sync(0xffffffffu, see[0], i & 31), y = __shfl_sync(0xffffffffu, see[1], i & 31);
        return i < 0 ? 0ull : i < 32 ? x : y;
    };
#pragma unroll 1
    for (int span = 1; span < u.T; span *= 2) {
        const unsigned long long s0 = of(up[0]), s1 = of(up[1]);
        int next[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int x = __shfl_sync(0xffffffffu, up[0], up[e] & 31), y = __shfl_sync(0xffffffffu, up[1], up[e] & 31);
            next[e] = up[e] < 0 ? -1 : up[e] < 32 ? x : y;
        }
        see[0] |= s0, see[1] |= s1;
        up[0] = next[0], up[1] = next[1];
    }
    return of(t);
}

}  // namespace wk
}  // namespace aladdin
