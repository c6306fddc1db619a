// aladdin_worker_attend: what its kernels (attend_few.cu, attend_many.cu) share.
//
// Request r has T new tokens, a tree (parent[t] < t or -1), and len cached
// tokens. Row (t, head g of key head h's group) has the scores
//     s_j = scale q . k_j,   j over the cached tokens, t's ancestors and t,
// and the results out = sum_j e^(s_j - lse) v_j, lse = log sum_j e^s_j.
//
// The rows of one (request, key head) share its keys, so they form one side of a
// matrix product with tiles of keys and, after the softmax, with tiles of values.
// The keys of a row tile, cached then new, are cut into tiles; the tiles of all
// (request, head, row tile) units lie on one axis, which the workers share
// evenly: each runs through a contiguous range, so that ragged requests and few
// long ones load every SM alike, and its copies run ahead across the units. A
// softmax goes over its tiles once with a running maximum and sum in 32 bits
// (base 2: the scores are multiplied by scale log2 e); the weights are rounded to
// the values' type for the second product, as its operands have to be. A unit that
// workers share leaves a partial sum, maximum and accumulator from each; the one
// that arrives last adds them in the order of their keys, so that results do not
// depend on the order of arrival.
#pragma once

#include "worker_dev.cuh"

namespace aladdin {
namespace wk {

// Where on the axis a worker (a warp, a CTA) is: KT keys a tile, RM rows a row tile.
struct Cursor {
    int r, h, rt, tile;   // request, key head, row tile, key tile
    int lo, T, len;       // its first new token, new tokens, cached tokens
    int c, nrt;           // key tiles, row tiles
};

template <int KT, int RM>
__device__ __forceinline__ void enter(const AttendArgs& a, Cursor& u, int r)
{
    u.r = r;
    u.lo = a.tok.off[r];
    u.T = a.tok.off[r + 1] - u.lo;
    u.len = a.kv.len[r];
    u.c = (u.len + u.T + KT - 1) / KT;
    u.nrt = (u.T * a.kv.group + RM - 1) / RM;
}

// The axis. A unit of c tiles takes `ov` + ceil(c / ct) places: `ov` stand for what a
// unit costs beside its tiles (a worker whose range ends within them has no tile
// of it), then ct tiles a place. Large calls count an overhead and single tiles;
// calls that give every worker ct tiles on average or fewer, places of ct and no overhead. Where
// those have no more places than workers, each worker has one at most, and the split of a
// unit does not depend on the others; with more units of few tiles than workers it does.
struct Axis {
    const int* pre;    // places of the requests before each, and of all
    const int* tiles;  // their tiles
    int total, workers, ov, ct;

    __device__ __forceinline__ int places(int c) const { return ov + (c + ct - 1) / ct; }
    // The first tile of a unit at its z-th place or behind it.
    __device__ __forceinline__ int tile_at(int z) const { return z <= ov ? 0 : (z - ov) * ct; }
    __device__ __forceinline__ int begin(int i) const { return (int)((long long)total * i / workers); }
    // The worker whose range holds place x (every worker has one: workers <= total).
    __device__ __forceinline__ int worker_of(int x) const
    {
        int i = (int)((long long)x * workers / total);
        while (i + 1 < workers && begin(i + 1) <= x) ++i;
        while (begin(i) > x) --i;
        return i;
    }
    // The first and the last worker that have tiles of the unit under u.
    __device__ __forceinline__ void sharers(const Cursor& u, int& first, int& last) const
    {
        const int n = places(u.c), at = pre[u.r] + (u.h * u.nrt + u.rt) * n;
        first = worker_of(at + ov);
        last = worker_of(at + n - 1);
    }
};

// Lays n requests on the axis, the block's threads together; pre and tiles hold n + 1
// entries each. of(r, c) gives the units of request r and sets c to the tiles of one.
// false: nothing to do.
template <int NT, typename F>
__device__ __forceinline__ bool plan(int n, Axis& x, int* pre, int* tiles, long long* scratch, int most, int ov,
                                     int ct, unsigned* err, F of)
{
    const int all = plan_prefix<NT>(n, tiles, scratch, [&](int r) -> long long {
        int c;
        const int units = of(r, c);
        return (long long)units * c;
    });
    x.pre = pre;
    x.tiles = tiles;
    const bool small = all <= (long long)ct * most;
    x.ov = small ? 0 : ov;
    x.ct = small ? ct : 1;
    x.total = all <= 0 ? all : plan_prefix<NT>(n, pre, scratch, [&](int r) -> long long {
        int c;
        const int units = of(r, c);
        return units ? (long long)units * x.places(c) : 0;
    });
    if (x.total <= 0) {
        if (x.total < 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(err, WORKER_BAD_INPUT);
        return false;
    }
    x.workers = min(most, x.total);
    return true;
}

// The attention's requests: units of a key head's row tiles. A request whose offsets or
// length make no sense has none and is recorded.
template <int KT, int RM>
__device__ __forceinline__ int attend_units(const AttendArgs& a, int r, int& c)
{
    const int lo = a.tok.off[r], hi = a.tok.off[r + 1], len = a.kv.len[r];
    if (lo < 0 || hi < lo || hi > a.tok.n_tok || hi - lo > ALADDIN_TREE_MAX || len < 0 || len > a.kv.cap) {
        if (blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        c = 0;
        return 0;
    }
    c = (len + hi - lo + KT - 1) / KT;
    return ((hi - lo) * a.kv.group + RM - 1) / RM * a.kv.kv_heads;
}

// The cursor at place x < total; returns the tiles in front of it.
template <int KT, int RM>
__device__ __forceinline__ int locate(const AttendArgs& a, const Axis& ax, Cursor& u, int x)
{
    const int r = plan_find(ax.pre, a.tok.n_req, x);
    enter<KT, RM>(a, u, r);
    const int n = ax.places(u.c), y = x - ax.pre[r], unit = y / n;
    u.tile = ax.tile_at(y - unit * n);
    u.h = unit / u.nrt;
    u.rt = unit - u.h * u.nrt;
    return ax.tiles[r] + unit * u.c + u.tile;
}

// Worker i's first tile under u; returns the number of its tiles.
template <int KT, int RM>
__device__ __forceinline__ int range(const AttendArgs& a, const Axis& ax, Cursor& u, int i)
{
    const int end = ax.begin(i + 1);
    const int t1 = end < ax.total ? locate<KT, RM>(a, ax, u, end) : ax.tiles[a.tok.n_req];
    return t1 - locate<KT, RM>(a, ax, u, ax.begin(i));
}

// To the next tile; pre[r] == pre[r + 1] for requests without tiles.
template <int KT, int RM>
__device__ __forceinline__ void advance(const AttendArgs& a, Cursor& u, const int* pre)
{
    if (++u.tile < u.c) return;
    u.tile = 0;
    if (++u.rt < u.nrt) return;
    u.rt = 0;
    if (++u.h < a.kv.kv_heads) return;
    u.h = 0;
    int r = u.r + 1;
    while (r < a.tok.n_req && pre[r + 1] == pre[r]) ++r;
    if (r < a.tok.n_req) enter<KT, RM>(a, u, r);
}

// The tokens that token t of the request under u sees, itself among them. A parent
// that is not an earlier token counts as none and is recorded.
__device__ __forceinline__ unsigned long long ancestors(const AttendArgs& a, const Cursor& u, int t)
{
    unsigned long long see = 0;
    while (t >= 0) {
        see |= 1ull << t;
        int p = a.tok.parent ? a.tok.parent[u.lo + t] : t - 1;
        if (p < -1 || p >= t) {
            atomicOr(a.err, WORKER_BAD_INPUT);
            p = -1;
        }
        t = p;
    }
    return see;
}

// A worker's partial results of a unit: RM (maximum, sum) pairs, then RM x D
// accumulators. Slot 1: of a unit that starts in its range, slot 0: of one that
// started before.
template <int D, int RM>
__device__ __forceinline__ float* part_of(const AttendArgs& a, int worker, int slot)
{
    return a.part + ((size_t)worker * 2 + slot) * (size_t)(RM * (D + 2));
}

// Four rows from row0, from row0 + step, ... below live of the unit under u, whose
// partial results the workers first .. last left; one warp's lanes together. A
// lane weighs the partials (a worker a lane), then sums four columns of four rows.
template <typename T, int D, int RM>
__device__ __forceinline__ void join_rows(const AttendArgs& a, const Cursor& u, int first, int last, int row0,
                                          int live, int step, int lane)
{
    constexpr int NV = (D / 4 + 31) / 32;
    const int G = a.kv.group, H = a.kv.kv_heads;
    for (int r0 = row0; r0 < live; r0 += step) {
        float ref[4], sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int y = 0; y < 4; ++y) ref[y] = -INFINITY;
        for (int i = first + lane; i <= last; i += 32) {
            const float* p = part_of<D, RM>(a, i, i == first);
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (r0 + y < live) ref[y] = fmaxf(ref[y], __ldcg(p + (r0 + y) * 2));
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
#pragma unroll
            for (int x = 16; x; x >>= 1) ref[y] = fmaxf(ref[y], __shfl_xor_sync(0xffffffffu, ref[y], x));
            if (ref[y] == -INFINITY) ref[y] = 0.0f;
        }
        float4 acc[4][NV];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int x = 0; x < NV; ++x) acc[y][x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int i0 = first; i0 <= last; i0 += 32) {
            float f[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (i0 + lane <= last) {
                const float* p = part_of<D, RM>(a, i0 + lane, i0 + lane == first);
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    if (r0 + y < live) {
                        const float2 v = __ldcg(reinterpret_cast<const float2*>(p + (r0 + y) * 2));
                        f[y] = ex2(v.x - ref[y]);
                        sum[y] += v.y * f[y];
                    }
                }
            }
            const int n = min(32, last - i0 + 1);
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                const float* p = part_of<D, RM>(a, i0 + i, i0 + i == first) + RM * 2 + r0 * D;
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float w = __shfl_sync(0xffffffffu, f[y], i);
#pragma unroll
                    for (int x = 0; x < NV; ++x) {
                        const int col = (x * 32 + lane) * 4;
                        if (r0 + y < live && (D % 128 == 0 || col < D)) {
                            const float4 v = __ldcg(reinterpret_cast<const float4*>(p + y * D + col));
                            acc[y][x].x += w * v.x;
                            acc[y][x].y += w * v.y;
                            acc[y][x].z += w * v.z;
                            acc[y][x].w += w * v.w;
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
#pragma unroll
            for (int x = 16; x; x >>= 1) sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], x);
            if (r0 + y >= live) break;
            const int rho = u.rt * RM + r0 + y, t = rho / G, head = u.h * G + rho - t * G;
            const float inv = sum[y] > 0.0f || sum[y] != sum[y] ? 1.0f / sum[y] : 0.0f;
#pragma unroll
            for (int x = 0; x < NV; ++x) {
                const int col = (x * 32 + lane) * 4;
                const float4 v = acc[y][x];
                if (D % 128 == 0 || col < D)
                    *reinterpret_cast<uint2*>(a.out +
                                              ((u.lo + t) * a.out_stride + (long long)head * D + col) * 2) =
                        make_uint2(Num<T>::pack(v.x * inv, v.y * inv), Num<T>::pack(v.z * inv, v.w * inv));
            }
            if (lane == 0 && a.lse)
                a.lse[(long long)(u.lo + t) * (H * G) + head] = (ref[y] + log2f(sum[y])) * LN2;
        }
    }
}

// The smallest normal number: what multiplies results that are not finite and would be lost with 0.
constexpr float NORMAL = 1.17549435e-38f;

// What a worker's partial results of a row, (maximum, sum), are multiplied by. A negative sum: of results that are not finite
// for their values, which count whatever their weight.
__device__ __forceinline__ float part_factor(float2 ml, float ref)
{
    const float f = ex2(ml.x - ref);
    return __float_as_int(ml.y) < 0 ? fmaxf(f, NORMAL) : f;
}

// Row rr (of token t, query head hd) of the unit under u, whose partial results the workers first .. last left with four
// columns of all rows together; one thread.
template <typename T, int D, int RM>
__device__ __forceinline__ void join_row(const AttendArgs& a, const Cursor& u, int first, int last, int rr, int t, int hd)
{
    float top = -INFINITY, sum = 0.0f;
#pragma unroll 4
    for (int i = first; i <= last; ++i)
        top = fmaxf(top, __ldcg(part_of<D, RM>(a, i, i == first) + rr * 2));
    const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
    for (int i = first; i <= last; ++i) {
        const float2 v = __ldcg(
            reinterpret_cast<const float2*>(part_of<D, RM>(a, i, i == first) + rr * 2));
        sum += fabsf(v.y) * part_factor(v, ref);
    }
    const float inv = 1.0f / sum;
    const auto of = [&](float x) { return sum == 0.0f ? 0.0f : x * inv; };
    uint4* const d = reinterpret_cast<uint4*>(
        a.out + ((u.lo + t) * a.out_stride + (long long)hd * D) * 2);
#pragma unroll 2
    for (int c = 0; c < D / 32; ++c) {
        float4 acc[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) acc[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
        for (int i = first; i <= last; ++i) {
            const float* const p = part_of<D, RM>(a, i, i == first);
            const float f = part_factor(__ldcg(reinterpret_cast<const float2*>(p + rr * 2)), ref);
            const float4* const q = reinterpret_cast<const float4*>(p + RM * 2) + c * 8 * RM + rr;
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const float4 v = __ldcg(q + x * RM);
                acc[x].x += f * v.x;
                acc[x].y += f * v.y;
                acc[x].z += f * v.z;
                acc[x].w += f * v.w;
            }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float4 y = acc[x * 2], z = acc[x * 2 + 1];
            d[c * 4 + x] = make_uint4(Num<T>::pack(of(y.x), of(y.y)), Num<T>::pack(of(y.z), of(y.w)),
                                      Num<T>::pack(of(z.x), of(z.y)), Num<T>::pack(of(z.z), of(z.w)));
        }
    }
    if (a.lse) a.lse[(long long)(u.lo + t) * (a.kv.kv_heads * a.kv.group) + hd] = (ref + log2f(sum)) * LN2;
}

}  // namespace wk
}  // namespace aladdin
