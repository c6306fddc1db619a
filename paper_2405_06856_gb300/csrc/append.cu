// aladdin_worker_append, aladdin_worker_append8: new tokens enter the paged cache, their keys rotated
// on the way (rope.cuh).
//
// Request r appends tokens i = 0 .. A: token i takes slot len + i and position next + i. In 16 bits a unit is some rows
// (heads' keys or values) of one token. In 8 bits it is a block of slots of one head, keys or values, by one warp: of the
// new values x of the block
//     scale = 2^j, the least j >= -126 with max |x| <= 448 2^j (finite values), or the scale that the block
//     has for the tokens that it holds, where that is larger;  code = e4m3(x / scale).
// With scales that are powers of two e4m3, a floating type, loses nothing but below its smallest normal
// number, 2^-6 of the scale: a scale that grows lets codes be rounded again without loss, and blocks do
// not depend on how their tokens came in. The two passes, for the maximum and for the codes, both
// read the new rows; the second finds them in the first-level cache.
//
// The kernels lay the requests' units on one axis (a prefix sum by each CTA) and go over it with all warps of the GPU. The
// last CTA to finish advances the lengths.
#include "rope.cuh"

namespace aladdin {
namespace wk {
namespace {

constexpr int WARPS = 8, NT = WARPS * 32;

// Tokens that request r appends; -1 where its offsets, length or choice make no sense.
__device__ __forceinline__ int appended(const AppendArgs& a, int r)
{
    const int lo = a.tok.off[r], hi = a.tok.off[r + 1], len = a.kv.len[r];
    const int a0 = a.acc_off ? a.acc_off[r] : lo, a1 = a.acc_off ? a.acc_off[r + 1] : hi;
    bool ok = lo >= 0 && hi >= lo && hi <= a.tok.n_tok && len >= 0 && a0 >= 0 && a1 >= a0 && a1 <= a.n_acc &&
              (!a.acc_off || a1 - a0 <= ALADDIN_TREE_MAX) && (long long)len + (a1 - a0) <= a.kv.cap;
    if (ok && a.acc_off) {
#pragma unroll 4
        for (int i = a0; i < a1; ++i) ok &= (unsigned)a.acc[i] < (unsigned)(hi - lo);
    }
    return ok ? a1 - a0 : -1;
}

// Lays the requests on the axis, per(r, A) units each; returns the number of all.
template <typename F>
__device__ __forceinline__ int lay(const AppendArgs& a, int* pre, long long* scratch, F per)
{
    const int all = plan_prefix<NT>(a.tok.n_req, pre, scratch, [&](int r) -> long long {
        const int A = appended(a, r);
        if (A < 0 && blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        return A > 0 ? per(r, A) : 0;
    });
    if (all < 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
    return all;
}

// Every CTA has read the lengths: the last one to come here advances those of the requests with units.
__device__ __forceinline__ void leave(const AppendArgs& a, const int* pre, int all, int* last)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        *last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!*last) return;
    if (threadIdx.x == 0) *a.arrived = 0;
    if (all <= 0) return;
    for (int r = threadIdx.x; r < a.tok.n_req; r += NT) {
        if (pre[r + 1] == pre[r]) continue;
        const int A = a.acc_off ? a.acc_off[r + 1] - a.acc_off[r] : a.tok.off[r + 1] - a.tok.off[r];
        a.kv.len[r] += A;
        if (a.kv.next) a.kv.next[r] += A;
    }
}

// Index of the i-th token that request r appends among all new tokens.
__device__ __forceinline__ long long source(const AppendArgs& a, int r, int i)
{
    return a.tok.off[r] + (a.acc_off ? a.acc[a.acc_off[r] + i] : i);
}

constexpr int ROWS = 4;  // rows in flight of a lane

// 16 bits: 2 H rows a token, in `parts` parts.
template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(NT) k_append(AppendArgs a, int parts)
{
    constexpr int CH = D / 8, RPW = 32 / CH;
    extern __shared__ int pre[];
    __shared__ long long scratch[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = a.kv.kv_heads;
    const int all = lay(a, pre, scratch, [&](int, int A) { return (long long)A * parts; });
    const int sub = lane / CH, ch = lane - sub * CH;
    Turns<INTERLEAVED> turns;
    if (a.rope.half) turns.load(a.rope, ch);
    const int per = ((2 * H + parts - 1) / parts + RPW - 1) / RPW * RPW;
    for (long long u = blockIdx.x * WARPS + warp; u < all; u += gridDim.x * WARPS) {
        const int r = plan_find(pre, a.tok.n_req, (int)u), y = (int)u - pre[r], i = y / parts, part = y - i * parts;
        const int slot = a.kv.len[r] + i, at = slot & (a.kv.page - 1);
        const int p = (int)((unsigned)(a.kv.next ? a.kv.next[r] : a.kv.len[r]) + (unsigned)i);
        const int page = a.kv.table[r * a.kv.table_stride + (slot >> a.kv.page_shift)];
        if ((unsigned)page >= (unsigned)a.kv.pages) {
            if (lane == 0) atomicOr(a.err, WORKER_BAD_INPUT);
            continue;
        }
        const long long t = source(a, r, i);
        const char* const k = a.tok.k + t * a.tok.k_stride * 2;
        const char* const v = a.tok.v + t * a.tok.v_stride * 2;
        const long long dst = page * a.kv.page_stride + at * a.kv.token_stride;
        const int row0 = part * per, row1 = min(2 * H, row0 + per);
        for (int row = row0; row < row1; row += RPW * ROWS) {
            uint4 x[ROWS], z[ROWS];
#pragma unroll
            for (int e = 0; e < ROWS; ++e) {
                const int h = row + e * RPW + sub;
                if (sub < RPW && h < row1) {
                    const char* const src = h < H ? k + (long long)h * D * 2 : v + (long long)(h - H) * D * 2;
                    x[e] = *reinterpret_cast<const uint4*>(src + ch * 16);
                    if (!INTERLEAVED && a.rope.half && h < H) z[e] = partners<T>(a.rope, src, ch);
                }
            }
#pragma unroll
            for (int e = 0; e < ROWS; ++e) {
                const int h = row + e * RPW + sub;
                if (sub < RPW && h < row1) {
                    if (a.rope.half && h < H) {
                        float f[8], g[8];
                        widen<T>(x[e], f);
                        if (!INTERLEAVED) widen<T>(z[e], g);
                        turn<INTERLEAVED>(a.rope, turns, p, ch, f, g);
                        x[e] = narrow<T>(f);
                    }
                    const int head = h < H ? h : h - H;
                    *reinterpret_cast<uint4*>((h < H ? a.kv.k : a.kv.v) + (dst + head * a.kv.head_stride + ch * 8) * 2) = x[e];
                    if (h < H && ch == 0) {
                        const long long m = ((long long)page * H + h) * a.kv.page + at;
                        if (a.kv.pos) a.kv.pos[m] = p;
                        if (a.kv.weight) a.kv.weight[m] = 0.0f;
                    }
                }
            }
        }
    }
    leave(a, pre, all, reinterpret_cast<int*>(scratch));
}

// ---- 8 bits

// Two e4m3 codes of two 32-bit values, the first in the lower byte; NaN gives NaN.
__device__ __forceinline__ uint32_t codes2(float lo, float hi)
{
    unsigned short u;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(u) : "f"(hi), "f"(lo));
    return u;
}
__device__ __forceinline__ float2 values2(uint32_t u)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)u));
    return __half22float2(*reinterpret_cast<__half2*>(&h));
}

// The least power of two, 2^-126 at least, of which m (finite, >= 0) is 448 = 1.75 2^8 times at most.
__device__ __forceinline__ float scale_of(float m)
{
    const uint32_t u = __float_as_uint(m);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);  // (of subnormal numbers less than 1)
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(NT) k_append8(AppendArgs a)
{
    constexpr int CH = D / 8, RPW = 32 / CH;
    extern __shared__ int pre[];
    __shared__ long long scratch[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = a.kv.kv_heads;
    const int shift = a.scales.block_shift, block = 1 << shift;
    const int all = lay(a, pre, scratch, [&](int r, int A) {
        const int len = a.kv.len[r];
        return (long long)(((len + A - 1) >> shift) - (len >> shift) + 1) * (2 * H);
    });
    const int sub = lane / CH, ch = lane - sub * CH;
    Turns<INTERLEAVED> turns;
    if (a.rope.half) turns.load(a.rope, ch);
    for (long long u = blockIdx.x * WARPS + warp; u < all; u += gridDim.x * WARPS) {
        const int r = plan_find(pre, a.tok.n_req, (int)u), y = (int)u - pre[r], b = y / (2 * H), hv = y - b * (2 * H);
        const bool values = hv >= H;
        const int h = values ? hv - H : hv, len = a.kv.len[r];
        const int A = a.acc_off ? a.acc_off[r + 1] - a.acc_off[r] : a.tok.off[r + 1] - a.tok.off[r];
        const int first = ((len >> shift) + b) << shift;               // the block's first slot
        const int lo = max(first, len), hi = min(first + block, len + A);  // its new slots
        const int page = a.kv.table[r * a.kv.table_stride + (first >> a.kv.page_shift)];
        if ((unsigned)page >= (unsigned)a.kv.pages) {
            if (lane == 0) atomicOr(a.err, WORKER_BAD_INPUT);
            continue;
        }
        const int at = first & (a.kv.page - 1), p0 = a.kv.next ? a.kv.next[r] : len;
        const char* const src = (values ? a.tok.v : a.tok.k) + (h * D + ch * 8) * 2;
        const long long stride = values ? a.tok.v_stride : a.tok.k_stride;
        const bool turned = !values && a.rope.half;
        // row `slot` of the new ones in 32 bits
        auto load = [&](int slot, float (&x)[8]) {
            const char* const row = src + source(a, r, slot - len) * stride * 2;
            widen<T>(*reinterpret_cast<const uint4*>(row), x);
            if (turned) {
                float z[8];
                if (!INTERLEAVED) widen<T>(partners<T>(a.rope, row - ch * 16, ch), z);
                turn<INTERLEAVED>(a.rope, turns, (int)((unsigned)p0 + (unsigned)(slot - len)), ch, x, z);
            }
        };
        float most = 0.0f;
#pragma unroll 2
        for (int slot = lo + sub; slot < hi; slot += RPW) {
            if (sub >= RPW) break;
            float x[8];
            load(slot, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float m = fabsf(x[j]);
                if (m < INFINITY) most = fmaxf(most, m);
            }
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
        float* const held = (values ? a.scales.v : a.scales.k) +
                            (((long long)page * H + h) * a.scales.per_page + (at >> shift));
        float scale = scale_of(most);
        char* const dst = (values ? a.kv.v : a.kv.k) + page * a.kv.page_stride + h * a.kv.head_stride +
                          at * a.kv.token_stride + ch * 8;
        if (lo > first) {
            const float old = *held;
            if (scale > old) {
                const float f = old / scale;
                for (int slot = first + sub; slot < lo && sub < RPW; slot += RPW) {
                    uint2* const d = reinterpret_cast<uint2*>(dst + (slot - first) * a.kv.token_stride);
                    const uint2 c = *d;
                    uint32_t w[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 z = values2((j < 2 ? c.x : c.y) >> (j & 1) * 16);
                        w[j] = codes2(z.x * f, z.y * f);
                    }
                    *d = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
                }
            } else {
                scale = old;
            }
        }
        const float inv = 1.0f / scale;
#pragma unroll 2
        for (int slot = lo + sub; slot < hi; slot += RPW) {
            if (sub >= RPW) break;
            float x[8];
            load(slot, x);
            // (x - x: nothing, or NaN for what is not finite)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = fmaf(x[j], inv, x[j] - x[j]);
            *reinterpret_cast<uint2*>(dst + (slot - first) * a.kv.token_stride) =
                make_uint2(codes2(x[0], x[1]) | codes2(x[2], x[3]) << 16, codes2(x[4], x[5]) | codes2(x[6], x[7]) << 16);
        }
        __syncwarp();
        if (lane == 0) *held = scale;
    }
    leave(a, pre, all, reinterpret_cast<int*>(scratch));
}

template <typename T, int D, bool INTERLEAVED>
cudaError_t launch_kind(const AppendArgs& a, int sms, cudaStream_t st)
{
    constexpr int RPW = 32 / (D / 8);
    const int smem = (a.tok.n_req + 1) * (int)sizeof(int), H = a.kv.kv_heads;
    // CTAs that have a unit, 4 an SM at most
    auto ctas = [&](long long units) {
        const long long want = (units + WARPS - 1) / WARPS;
        return (int)(want < 4ll * sms ? want : 4ll * sms);
    };
    if (a.scales.k) {
        // (a request's tokens enter two blocks more than they fill, at most)
        k_append8<T, D, INTERLEAVED><<<ctas((((long long)a.n_acc >> a.scales.block_shift) + 2ll * a.tok.n_req) * 2 * H), NT, smem, st>>>(a);
    } else {
        const long long want = ((long long)sms * 32 + a.n_acc - 1) / a.n_acc;
        const int most = (2 * H + RPW * ROWS - 1) / (RPW * ROWS), parts = (int)(want < most ? want : most);
        k_append<T, D, INTERLEAVED><<<ctas((long long)a.n_acc * parts), NT, smem, st>>>(a, parts);
    }
    return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch(const AppendArgs& a, int sms, cudaStream_t st)
{
    return a.rope.interleaved ? launch_kind<T, D, true>(a, sms, st) : launch_kind<T, D, false>(a, sms, st);
}

template <typename T>
cudaError_t launch_dim(const AppendArgs& a, int dim, int sms, cudaStream_t st)
{
    switch (dim) {
        case 64: return launch<T, 64>(a, sms, st);
        case 96: return launch<T, 96>(a, sms, st);
        case 128: return launch<T, 128>(a, sms, st);
        case 256: return launch<T, 256>(a, sms, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace
}  // namespace wk

cudaError_t launch_append(const AppendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
