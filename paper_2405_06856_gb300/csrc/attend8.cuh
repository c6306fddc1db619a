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

// Products of e4m3: 16 keys of 32 channels by 8 rows.
__device__ __forceinline__ void mma8(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two e4m3 codes of two 32-bit values, the first in the lower byte.
__device__ __forceinline__ uint32_t codes2(float lo, float hi)
{
    unsigned short u;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u) : "f"(hi), "f"(lo));
    return u;
}

// A row of queries, 4 lanes together, as the sum of N parts of e4m3, each in units of 1 / PART of the one before, times
// the power of two that is returned. The row is scaled so that its largest channel lies in 2^7 .. 2^8; what a part
// leaves over, at most half a step, 2^-4 of it, is exact in 32 bits. Two parts hold 9 bits of every channel
// (bfloat16 has 8), three hold 14 (half precision has 11), where the last part's smallest step, 2^-9, is small
// enough: of channels below 2^-13 (2^-20 with three) of the largest what is lost is less than 2^-22 (2^-27) of it.
constexpr float PART = 32.0f;
template <typename T, int N, int M>
__device__ __forceinline__ float split_row(const uint2 (&q)[M], uint32_t (&p)[N][M])
{
    unsigned most = 0;  // magnitudes as whole numbers: infinity and NaN are the largest
#pragma unroll
    for (int x = 0; x < M; ++x) {
        const float2 u = Num<T>::unpack(q[x].x), v = Num<T>::unpack(q[x].y);
        const auto bits = [](float y) { return __float_as_uint(y) & 0x7fffffffu; };
        most = max(max(most, max(bits(u.x), bits(u.y))), max(bits(v.x), bits(v.y)));
    }
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // exponent fields from 17 (2^-110) on: the factor and its inverse are normal numbers
    const int e = min(max((int)(most >> 23), 17), 254);
    const float f = __uint_as_float((uint32_t)(261 - e) << 23);
#pragma unroll
    for (int x = 0; x < M; ++x) {
        const float2 u = Num<T>::unpack(q[x].x), v = Num<T>::unpack(q[x].y);
        float r[4] = {u.x * f, u.y * f, v.x * f, v.y * f};
#pragma unroll
        for (int z = 0; z < N; ++z) {
            const uint32_t lo = codes2(r[0], r[1]), hi = codes2(r[2], r[3]);
            p[z][x] = lo | hi << 16;
            if (z + 1 < N) {
                const uint32_t a = half2_lo(lo), b = half2_lo(hi);
                const float2 c = Num<__half>::unpack(a), d = Num<__half>::unpack(b);
                r[0] = (r[0] - c.x) * PART, r[1] = (r[1] - c.y) * PART;
                r[2] = (r[2] - d.x) * PART, r[3] = (r[3] - d.y) * PART;
            }
        }
    }
    return most < 0x7f800000u ? __uint_as_float((uint32_t)(e - 7) << 23) : NAN;  // (a query that is not finite has no scores)
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
