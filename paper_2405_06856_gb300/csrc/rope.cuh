// Rotary positions on 8 channels at a time: shared by rotate.cu and append.cu.
//
// Pair c of a token at position p is turned by the angle p freq_c. The frequency comes in
// turns, as a 64-bit fraction of one, so that p times it wraps around exactly and its upper
// 32 bits are the angle to 2^-32 turns, however far the position is, without 64-bit floating point,
// of which this GPU has little. The angle's distance x to the nearest quarter turn, at most pi / 4, goes
// through the Taylor series of sine and cosine: what they leave out is x^11 / 11! < 2^-29 and x^10 / 10! < 2^-25
// (one more term: no fewer codes of 8 bits on the other side of a rounding, and 1 us of 50 in append.cu).
#pragma once

#include "worker_dev.cuh"

namespace aladdin {
namespace wk {

// What turns channels [8 ch, 8 ch + 8) of a head: cosine and sine of each of their pairs at one position, times the
// factor. In the half layout a channel has its pair's sine with the sign of its partner's part: x' = x c + y s.
// Channels that are not turned have 1 and 0.
template <bool INTERLEAVED>
struct Rotor {
    static constexpr int N = INTERLEAVED ? 4 : 8;
    const unsigned long long* turn_of;
    uint32_t hi[4], lo[4];  // frequencies of the pairs whose angles this lane forms
    float c[N], s[N];
    float scale;
    int half, ch;

    __device__ __forceinline__ void load(const RopeDev& rope, int chunk)
    {
        turn_of = rope.turn;
        scale = rope.scale;
        half = rope.half;
        ch = chunk;
        frequencies(hi, lo, upper() ? 4 : 0);
    }
    // Half layout, halves that begin at multiples of 8 channels: the lanes of a pair of chunks form the angles of 4 of their
    // pairs each, the one of the upper half the last 4, and exchange them (all 8 each: 36 us for 34 in append.cu, 16 bits).
    __device__ __forceinline__ bool shared() const { return (half & 7) == 0; }
    __device__ __forceinline__ bool upper() const { return !INTERLEAVED && shared() && ch * 8 >= half; }
    __device__ __forceinline__ int pair(int j) const
    {
        const int at = ch * 8 + j;
        return INTERLEAVED ? ch * 4 + j : at < half ? at : at - half;
    }
    __device__ __forceinline__ void frequencies(uint32_t (&h)[4], uint32_t (&l)[4], int j0) const
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int p = pair(j0 + j);
            const unsigned long long t = p < half ? __ldg(turn_of + p) : 0;
            h[j] = (uint32_t)(t >> 32);
            l[j] = (uint32_t)t;
        }
    }
    // Cosine and sine of 4 pairs at position p.
    static __device__ __forceinline__ void angles(int p, const uint32_t (&h)[4], const uint32_t (&l)[4], float (&cs)[4],
                                                  float (&sn)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // the upper word of p (h, l), p signed
            const uint32_t turn = (uint32_t)p * h[j] + __umulhi((uint32_t)p, l[j]) - (p < 0 ? l[j] : 0u);
            const uint32_t quarter = (turn + 0x20000000u) & 0xc0000000u;
            // the angle is x + y: 2 pi / 2^32 comes in two parts, and the series' leading terms are added last
            const float f = (float)(int)(turn - quarter), x = f * 1.462918119976564e-9f, x2 = x * x;
            const float y = fmaf(f, -4.0709404e-17f, fmaf(f, 1.462918119976564e-9f, -x));
            const float p0 = fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6);
            const float p1 = fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 40320, -1.0f / 720), 1.0f / 24), -0.5f);
            const float a = x + fmaf(x * x2, p0, fmaf(x2 * p1, y, y)), b = 1.0f + fmaf(x2, p1, -x * y);
            // of 0, 1, 2, 3 quarters more: (b, a), (-a, b), (-b, -a), (a, -b)
            const bool odd = quarter & 0x40000000u;
            const float u = odd ? a : b, v = odd ? b : a;
            cs[j] = __uint_as_float(__float_as_uint(u) ^ ((quarter + 0x40000000u) & 0x80000000u));
            sn[j] = __uint_as_float(__float_as_uint(v) ^ (quarter & 0x80000000u));
        }
    }
    // to position p; all lanes of a warp, those of a row with the same p
    __device__ __forceinline__ void at(int p)
    {
        float cs[4], sn[4];
        angles(p, hi, lo, cs, sn);
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool turned = ch * 4 + j < half;
                c[j] = turned ? cs[j] * scale : 1.0f;
                s[j] = turned ? sn[j] * scale : 0.0f;
            }
        } else {
            float co[4], so[4];
            if (shared()) {
                const int mate = (threadIdx.x & 31) + (upper() ? -half / 8 : half / 8);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    co[j] = __shfl_sync(0xffffffffu, cs[j], mate);
                    so[j] = __shfl_sync(0xffffffffu, sn[j], mate);
                }
            } else {
                uint32_t h[4], l[4];
                frequencies(h, l, 4);
                angles(p, h, l, co, so);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = ch * 8 + j;
                const float x = (j < 4) != upper() ? cs[j & 3] : co[j & 3], y = (j < 4) != upper() ? sn[j & 3] : so[j & 3];
                c[j] = at < 2 * half ? x * scale : 1.0f;
                s[j] = at < 2 * half ? y * (at < half ? -scale : scale) : 0.0f;
            }
        }
    }
    // on by as many positions as `by`, a rotor at them with factor 1, stands for: an error of 2^-24 more
    __device__ __forceinline__ void on(const Rotor& by)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float t = fmaf(c[j], by.c[j], -s[j] * by.s[j]);
            s[j] = fmaf(s[j], by.c[j], c[j] * by.s[j]);
            c[j] = t;
        }
    }
    // x, 8 channels; y: their partners (half layout; 0 for channels that are not turned)
    __device__ __forceinline__ void turn(float (&x)[8], const float (&y)[8]) const
    {
        if constexpr (INTERLEAVED) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float a = x[2 * j], b = x[2 * j + 1];
                if (ch * 4 + j < half) {
                    x[2 * j] = fmaf(a, c[j], -b * s[j]);
                    x[2 * j + 1] = fmaf(a, s[j], b * c[j]);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(x[j], c[j], y[j] * s[j]);
        }
    }
};

// 8 values of 16 bits in 32
template <typename T>
__device__ __forceinline__ void widen(const uint4& v, float (&x)[8])
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = Num<T>::unpack(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
template <typename T>
__device__ __forceinline__ uint4 narrow(const float (&x)[8])
{
    return make_uint4(Num<T>::pack(x[0], x[1]), Num<T>::pack(x[2], x[3]), Num<T>::pack(x[4], x[5]),
                      Num<T>::pack(x[6], x[7]));
}

// The partners of channels [8 ch, 8 ch + 8) in the half layout, from the head's row in global memory (16 bytes at a
// time where the halves begin at multiples of 8 channels); 0 for channels that are not turned.
template <typename T>
__device__ __forceinline__ uint4 partners(const RopeDev& rope, const char* row, int ch)
{
    const int h = rope.half, c0 = ch * 8;
    if (c0 >= 2 * h) return make_uint4(0, 0, 0, 0);
    if ((h & 7) == 0) return *reinterpret_cast<const uint4*>(row + (c0 < h ? c0 + h : c0 - h) * 2);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t u[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int c = c0 + 2 * i + e;
            u[e] = c < 2 * h ? *reinterpret_cast<const unsigned short*>(row + (c < h ? c + h : c - h) * 2) : 0;
        }
        w[i] = u[0] | u[1] << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace wk
}  // namespace aladdin
