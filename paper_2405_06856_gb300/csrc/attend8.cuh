// aladdin_worker_attend8: what its kernels share.
//
// As aladdin_worker_attend (attend.cuh), over cached keys and values of 8 bits: k_j = c_j a_b, v_j = d_j e_b with
// e4m3 codes c, d and scales a, e of the block b that slot j lies in, so that
//     s_j = (scale a_b) q . c_j,      out = sum_j (e^(s_j - lse) e_b) d_j.
// Codes are exact in half precision, and so are queries of it. Queries of bfloat16 are multiplied by a power of two
// for each row that brings its largest channel to 2^14 .. 2^15: half precision then holds every channel above 2^-28
// of the largest without loss. Products and sums are 32-bit, and the scales and the row's power multiply the sums.
//
// The second product's weights are rounded to half precision, 2^-11 of each, so what counts is what they refer to: not to
// the largest scale, which may belong to a block without any weight, nor to the largest weight, whose block may have
// next to no scale, but to the largest product of the two. A row keeps M, the maximum of t_j = s_j + log2 e_b (to base 2)
// so far; its weights are 2^(t_j - M + UP), with UP as large as half precision and what M may lag behind allow, results
// count in units of 2^(M - UP), and sums l of the weights without scales in units of 2^(M - d). So a weight is good to 2^-11 of
// itself down to 2^-14 - UP of the largest, and 0 below 2^-25 - UP of it. Any d does that keeps the sums within 32 bits'
// range: it is the logarithm of a scale, and while those of a tile are within 2^FAR of it, as nearly always, a tile
// costs what it would with one scale for all. Others (and new tokens, each of which has a logarithm of its own) take a
// longer way, on which d becomes what M has above the largest s_j. A scale of 0 has the logarithm LOG_ZERO.
// Where scores are so large that logarithms next to them round, sums are rounded such that no weight passes 2^UP.
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

// The power of two that values of which `top` is the largest exponent field in 32 bits are multiplied by, and the one
// that takes it back.
__device__ __forceinline__ float half_factor(int top) { return __uint_as_float((uint32_t)(268 - min(max(top, 15), 254)) << 23); }
__device__ __forceinline__ float half_back(int top) { return __uint_as_float((uint32_t)(min(max(top, 15), 254) - 14) << 23); }

// The largest magnitudes of the lower and of the upper values of words, as bits, and the exponent field in 32 bits of the
// larger one (of half-precision numbers below 2^-14 that of 2^-14).
__device__ __forceinline__ uint32_t largest2(uint32_t top, uint32_t w) { return __vmaxu2(top, w & 0x7fff7fffu); }
template <typename T>
__device__ __forceinline__ int exponent(uint32_t top)
{
    const uint32_t u = max(top & 0xffff, top >> 16);
    if constexpr (std::is_same<T, __half>::value) return (int)max(u >> 10, 1u) + 112;
    return (int)(u >> 7);
}
// The largest exponent field of finite values and `top`.
template <typename T>
__device__ __forceinline__ int finite_exponent(uint32_t w, int top)
{
    w = Num<T>::tame(w);
    if constexpr (!std::is_same<T, __half>::value) return max(top, max((int)(w >> 7 & 0xff), (int)(w >> 23 & 0xff)));
    const float2 v = Num<T>::unpack(w);
    return max(top, max((int)(__float_as_uint(v.x) >> 23 & 0xff), (int)(__float_as_uint(v.y) >> 23 & 0xff)));
}
template <typename T>
__device__ __forceinline__ uint32_t to_half(uint32_t w, float f)
{
    const float2 v = Num<T>::unpack(w);
    return Num<__half>::pack(v.x * f, v.y * f);
}

// ... and back.
template <typename T>
__device__ __forceinline__ uint32_t from_half(uint32_t w, float f)
{
    if constexpr (std::is_same<T, __half>::value) return w;
    const float2 v = Num<__half>::unpack(w);
    return Num<T>::pack(v.x * f, v.y * f);
}

// A row of queries, 4 lanes together, to half precision; returns what its scores are multiplied by.
template <typename T, int N>
__device__ __forceinline__ float half_row(uint2 (&q)[N])
{
    if constexpr (std::is_same<T, __half>::value) return 1.0f;
    uint32_t most = 0;
#pragma unroll
    for (int x = 0; x < N; ++x) most = largest2(largest2(most, q[x].x), q[x].y);
    int top = exponent<T>(most);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const float f = half_factor(top);
#pragma unroll
    for (int x = 0; x < N; ++x) q[x] = make_uint2(to_half<T>(q[x].x, f), to_half<T>(q[x].y, f));
    return half_back(top);
}

// A block's scale; NaN of one that is not finite (infinity would make scores of -inf, which count as not seen).
__device__ __forceinline__ float finite_scale(float k) { return k < INFINITY ? k : NAN; }

constexpr float FAR = 40.0f, LOG_ZERO = -256.0f;

// Logarithm of a block's scale, NaN of what is none.
__device__ __forceinline__ float log_scale(float v)
{
    return v > 0.0f && v < INFINITY ? __log2f(v) : v == 0.0f ? LOG_ZERO : NAN;
}
// 2^d in two factors, neither of which is lost below 2^-126 where the whole is not.
__device__ __forceinline__ float2 unit_of(float d)
{
    const float x = fmaxf(d, -100.0f);
    return make_float2(ex2(x), ex2(d - x));
}

// The axis of all key tiles (attend.cuh), its places dealt out whole: the first `more` workers have one place more than
// the others' `each`. What a cursor needs to know of the requests lies in shared memory.
struct Axis8 {
    int* pre;    // places of the requests before each, and of all
    int* tiles;  // their tiles
    int* lo;     // first new tokens
    int* toks;   // new tokens, 0 of requests that make no sense
    int* len;    // cached tokens
    int total, workers, ov, ct, each, more;

    static constexpr int ints(int n_req) { return 5 * (n_req + 1); }
    __device__ __forceinline__ int places(int c) const { return ov + (c + ct - 1) / ct; }
    __device__ __forceinline__ int tile_at(int z) const { return z <= ov ? 0 : (z - ov) * ct; }
    __device__ __forceinline__ int begin(int i) const { return i * each + min(i, more); }
    __device__ __forceinline__ int worker_of(int x) const
    {
        const int y = x - more * (each + 1);
        return y < 0 ? x / (each + 1) : more + y / each;
    }
    // The first and the last worker that have tiles of the unit under u.
    __device__ __forceinline__ void sharers(const Cursor& u, int& first, int& last) const
    {
        const int n = places(u.c), at = pre[u.r] + (u.h * u.nrt + u.rt) * n;
        first = worker_of(at + ov);
        last = worker_of(at + n - 1);
    }
};

// Key tiles of a row tile: KT keys each, then new tokens in tiles of their own, TN each.
template <int KT, int TN>
__device__ __forceinline__ int key_tiles(int len, int T)
{
    return (len + KT - 1) / KT + (T + TN - 1) / TN;
}

// Lays the requests on the axis, the block's threads together; mem: Axis8::ints, scratch: 96 long longs. One pass with
// three sums: of tiles, of places with `ov` for each unit, and of places of ct tiles. false: nothing to do.
template <int NT, int KT, int TN, int RM>
__device__ __forceinline__ bool plan8(const AttendArgs& a, Axis8& x, int* mem, long long* scratch, int most, int ov, int ct)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.tok.n_req;
    x.pre = mem;
    x.tiles = mem + (n + 1);
    x.lo = mem + 2 * (n + 1);
    x.toks = mem + 3 * (n + 1);
    x.len = mem + 4 * (n + 1);
    int* const small = x.pre;  // places of ct tiles first; replaced where the axis is a large one
    long long base[3] = {0, 0, 0};
    for (int r0 = 0; r0 < n; r0 += NT) {
        const int r = r0 + tid;
        long long v[3] = {0, 0, 0};
        int T = 0, units = 0, c = 0;
        if (r < n) {
            const int lo = a.tok.off[r], hi = a.tok.off[r + 1], len = a.kv.len[r];
            if (lo < 0 || hi < lo || hi > a.tok.n_tok || hi - lo > ALADDIN_TREE_MAX || len < 0 || len > a.kv.cap) {
                if (blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
            } else {
                T = hi - lo;
            }
            x.lo[r] = lo;
            x.toks[r] = T;
            x.len[r] = len;
            if (T) {
                c = key_tiles<KT, TN>(len, T);
                units = (T * a.kv.group + RM - 1) / RM * a.kv.kv_heads;
            }
            v[0] = (long long)units * c;
            v[1] = (long long)units * (ov + c);
            v[2] = (long long)units * ((c + ct - 1) / ct);
        }
        long long mine[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            mine[k] = v[k];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, v[k], o);
                if (lane >= o) v[k] += u;
            }
            if (lane == 31) scratch[k * 32 + warp] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            long long before = base[k];
#pragma unroll
            for (int w = 0; w < NT / 32; ++w) {
                const long long y = scratch[k * 32 + w];
                before += w < warp ? y : 0;
                base[k] += y;
            }
            v[k] += before - mine[k];
        }
        if (r < n) {
            x.tiles[r] = (int)v[0];
            small[r] = (int)v[2];
        }
        __syncthreads();
    }
    if (base[1] > 0x7fffffffll || base[0] <= 0) {
        if (base[0] > 0 && blockIdx.x == 0 && tid == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        return false;
    }
    if (tid == 0) x.tiles[n] = (int)base[0];
    const bool few = base[0] <= (long long)ct * most;
    x.ov = few ? 0 : ov;
    x.ct = few ? ct : 1;
    x.total = (int)(few ? base[2] : base[1]);
    if (tid == 0) small[n] = x.total;
    __syncthreads();
    if (!few) {
        // a unit has ov places more than tiles: so many for all units before
        for (int r = tid; r < n; r += NT) x.pre[r] = x.tiles[r];
        __syncthreads();
        if (ov) {
            long long sum = 0;  // of units
            for (int r0 = 0; r0 < n; r0 += NT) {
                const int r = r0 + tid;
                int v = r < n && x.toks[r] ? (x.toks[r] * a.kv.group + RM - 1) / RM * a.kv.kv_heads : 0;
                const int mine = v;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int u = __shfl_up_sync(0xffffffffu, v, o);
                    if (lane >= o) v += u;
                }
                if (lane == 31) scratch[warp] = v;
                __syncthreads();
                long long before = sum;
#pragma unroll
                for (int w = 0; w < NT / 32; ++w) {
                    before += w < warp ? scratch[w] : 0;
                    sum += scratch[w];
                }
                if (r < n) x.pre[r] += (int)(before + v - mine) * ov;
                __syncthreads();
            }
        }
    }
    x.workers = min(most, x.total);
    x.each = x.total / x.workers;
    x.more = x.total - x.each * x.workers;
    return true;
}

template <int KT, int TN, int RM>
__device__ __forceinline__ void enter8(const AttendArgs& a, const Axis8& x, Cursor& u, int r)
{
    u.r = r;
    u.lo = x.lo[r];
    u.T = x.toks[r];
    u.len = x.len[r];
    u.c = key_tiles<KT, TN>(u.len, u.T);
    u.nrt = (u.T * a.kv.group + RM - 1) / RM;
}

// The cursor at place y < total; returns the tiles in front of it.
template <int KT, int TN, int RM>
__device__ __forceinline__ int locate8(const AttendArgs& a, const Axis8& x, Cursor& u, int y)
{
    const int r = plan_find(x.pre, a.tok.n_req, y);
    enter8<KT, TN, RM>(a, x, u, r);
    const int n = x.places(u.c), z = y - x.pre[r], unit = z / n;
    u.tile = x.tile_at(z - unit * n);
    u.h = unit / u.nrt;
    u.rt = unit - u.h * u.nrt;
    return x.tiles[r] + unit * u.c + u.tile;
}

// Worker i's first tile under u; returns the number of its tiles.
template <int KT, int TN, int RM>
__device__ __forceinline__ int range8(const AttendArgs& a, const Axis8& x, Cursor& u, int i)
{
    const int end = x.begin(i + 1);
    const int t1 = end < x.total ? locate8<KT, TN, RM>(a, x, u, end) : x.tiles[a.tok.n_req];
    return t1 - locate8<KT, TN, RM>(a, x, u, x.begin(i));
}

// To the next unit.
template <int KT, int TN, int RM>
__device__ __forceinline__ void next_unit8(const AttendArgs& a, const Axis8& x, Cursor& u)
{
    u.tile = 0;
    if (++u.rt < u.nrt) return;
    u.rt = 0;
    if (++u.h < a.kv.kv_heads) return;
    u.h = 0;
    int r = u.r + 1;
    while (r < a.tok.n_req && x.toks[r] == 0) ++r;
    if (r < a.tok.n_req) enter8<KT, TN, RM>(a, x, u, r);
}
// To the next tile.
template <int KT, int TN, int RM>
__device__ __forceinline__ void advance8(const AttendArgs& a, const Axis8& x, Cursor& u)
{
    if (++u.tile == u.c) next_unit8<KT, TN, RM>(a, x, u);
}

// A warp says that its part of a unit is written, and learns how many have said so before; the last one reads what they
// wrote behind a fence of its own. counter: of the unit, zero between calls. The number is not waited for here.
__device__ __forceinline__ int arrive_at(int* counter)
{
    int before;
    asm volatile("fence.acq_rel.gpu;\n atom.add.relaxed.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
    return before;
}

// What the tokens of the request under u see, themselves among them; all lanes together. A parent that is not an earlier
// token counts as none and is recorded. (A lane holds two tokens; every round joins what a token sees with what the one at
// the end of it sees: the walk up by loads, one after the other, took 10 times as long.)
struct Ancestors {
    unsigned long long see[2];

    // of token t, each lane its own
    __device__ __forceinline__ unsigned long long of(int i) const
    {
        const unsigned long long x = __shfl_sync(0xffffffffu, see[0], i & 31), y = __shfl_sync(0xffffffffu, see[1], i & 31);
        return i < 0 ? 0ull : i < 32 ? x : y;
    }
    __device__ __forceinline__ Ancestors(const AttendArgs& a, const Cursor& u, int lane)
    {
        int up[2];
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
    }
};

}  // namespace wk
}  // namespace aladdin
