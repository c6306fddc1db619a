// aladdin_worker_append, aladdin_worker_append8: new tokens enter the paged cache, their keys rotated
// on the way (rope.cuh).
//
// Request r appends tokens i = 0 .. A: token i takes slot len + i and position next + i. In 16 bits a unit is some rows
// (heads' keys or values) of one token, a warp's. In 8 bits it is a block of slots of one head, keys or values: of the
// new values x of the block
//     scale = 2^j, the least j >= -126 with max |x| <= 448 2^j (finite values), or the scale that the block
//     has for the tokens that it holds, where that is larger;  code = e4m3(x / scale).
// With scales that are powers of two e4m3, a floating type, loses nothing but below its smallest normal
// number, 2^-6 of the scale: a scale that grows lets codes be rounded again without loss, and blocks do
// not depend on how their tokens came in. A warp has a few rows of a block, four chunks of 8 channels a lane, and keeps
// them, rotated, in registers from the maximum to the codes; the warps of a block exchange their maxima. Instructions are
// what it spends most of: so a lane forms the angles of every other row and turns them on to its next. (Three turns after one
// another: 47 us for 50, but half as many codes more than by 64-bit angles came out on the other side of a rounding; every
// row's own angles: 55. Of 14 million keys' codes 7 differ from those of 64-bit arithmetic so, as many as with 64-bit angles.)
//
// Measured: prompts of 20,178 tokens, 8 key heads of 128 channels, into 16 bits 34 us, 4.9 TB/s read and written (a unit of one
// token, a search and new angles each: 49); 36,000 tokens, 4 heads of 96, into 8 bits in blocks of 64: 51 us, 1.6 TB/s, half of the
// instruction slots and the rest latency of rounds that end in a barrier (one warp a block that reads its rows twice:
// 66). In blocks of 16 with 8 heads of 128 in the half layout, 222 MB: 129 us (all warps of a CTA waiting for one another: 45
// more; in this layout 100 to 150 bytes a thread do not fit into registers). One token each of 128 requests: 6 and 9 us with the launch, a chain of look-ups.
//
// The kernels lay the requests' units on one axis (a prefix sum by each CTA, which keeps what the units need of them) and
// go over it with all warps of the GPU. The last CTA to finish advances the lengths.
#include "rope.cuh"

namespace aladdin {
namespace wk {
namespace {

constexpr int WARPS = 8, NT = WARPS * 32, PER_SM = 2;  // of a CTA; CTAs of an SM

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

// What the units need of the requests, in shared memory.
struct Requests {
    int* pre;   // units of the requests before each, and of all
    int* len;
    int* next;
    int* lo;    // first new tokens
    int* a0;    // first entries of acc
    int* count; // tokens that they append

    static size_t bytes(int n) { return (size_t)(n + 1) * 6 * sizeof(int); }
};

// Lays the requests on the axis, per(len, A) units each; returns the number of all.
template <typename F>
__device__ __forceinline__ int lay(const AppendArgs& a, Requests& q, int* mem, long long* scratch, F per)
{
    const int n = a.tok.n_req + 1;
    q.pre = mem, q.len = mem + n, q.next = mem + 2 * n, q.lo = mem + 3 * n, q.a0 = mem + 4 * n, q.count = mem + 5 * n;
    const int all = plan_prefix<NT>(a.tok.n_req, q.pre, scratch, [&](int r) -> long long {
        const int A = appended(a, r);
        if (A < 0 && blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        q.len[r] = a.kv.len[r];
        q.next[r] = a.kv.next ? a.kv.next[r] : q.len[r];
        q.lo[r] = a.tok.off[r];
        q.a0[r] = a.acc_off ? a.acc_off[r] : 0;
        q.count[r] = A;
        return A > 0 ? per(q.len[r], A) : 0;
    });
    if (all < 0 && blockIdx.x == 0 && threadIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
    return all;
}

// Every CTA has read the lengths: the last one to come here advances those of the requests with units.
__device__ __forceinline__ void leave(const AppendArgs& a, const Requests& q, int all, int* last)
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
        if (q.count[r] <= 0) continue;
        a.kv.len[r] = q.len[r] + q.count[r];
        if (a.kv.next) a.kv.next[r] = q.next[r] + q.count[r];
    }
}

// Index of the i-th token that request r appends among all new tokens.
__device__ __forceinline__ long long source(const AppendArgs& a, const Requests& q, int r, int i)
{
    return q.lo[r] + (a.acc ? a.acc[q.a0[r] + i] : i);
}

constexpr int ROWS = 4;  // rows of keys, and of values, in flight of a lane

// 16 bits: a unit is `heads` heads of one token. A warp has neighbouring units.
template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(NT, PER_SM) k_append(AppendArgs a, int heads)
{
    constexpr int CH = D / 8, RPW = 32 / CH;
    extern __shared__ int mem[];
    __shared__ long long scratch[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = a.kv.kv_heads, parts = (H + heads - 1) / heads;
    Requests q;
    const int all = lay(a, q, mem, scratch, [&](int, int A) { return (long long)A * parts; });
    const int sub = lane / CH, ch = lane - sub * CH;
    const bool on = sub < RPW;
    Rotor<INTERLEAVED> rotor, one;
    if (a.rope.half) {
        rotor.load(a.rope, ch);
        one = rotor;
        one.scale = 1.0f;
        one.at(1);
    }
    const int workers = (int)gridDim.x * WARPS, each = (max(all, 0) + workers - 1) / workers;
    const int begin = (int)min((long long)(blockIdx.x * WARPS + warp) * each, (long long)max(all, 0)),
              end = (int)min((long long)begin + each, (long long)max(all, 0));
    int r = begin < end ? plan_find(q.pre, a.tok.n_req, begin) : 0;
    int at_p = 0, turned = 0;  // where the rotor is, how often it has been turned on to there
    bool fresh = true;
    for (int u = begin; u < end; ++u) {
        while (u >= q.pre[r + 1]) ++r;
        const int y = u - q.pre[r], i = parts == 1 ? y : y / parts, part = y - i * parts;
        const int slot = q.len[r] + i, at = slot & (a.kv.page - 1);
        const int p = (int)((unsigned)q.next[r] + (unsigned)i);
        // (the page is looked up while the rows are on their way)
        const int page = a.kv.table[r * a.kv.table_stride + (slot >> a.kv.page_shift)];
        const long long t = source(a, q, r, i);
        const int h0 = part * heads + sub, h1 = min(H, part * heads + heads);
        const char* k = a.tok.k + (t * a.tok.k_stride + h0 * D + ch * 8) * 2;
        const char* v = a.tok.v + (t * a.tok.v_stride + h0 * D + ch * 8) * 2;
        if (a.rope.half && (fresh || p != at_p)) {
            if (!fresh && p == at_p + 1 && turned < 3) {
                rotor.on(one);
                ++turned;
            } else {
                rotor.at(p);
                turned = 0;
            }
            fresh = false;
            at_p = p;
        }
        const bool have = (unsigned)page < (unsigned)a.kv.pages;
        long long dst = (have ? page * a.kv.page_stride + at * a.kv.token_stride + h0 * a.kv.head_stride : 0) + ch * 8;
        long long m = have ? ((long long)page * H + h0) * a.kv.page + at : 0;
        for (int h = h0; h - sub < h1; h += RPW * ROWS) {
            uint4 x[ROWS], z[ROWS], w[ROWS];
#pragma unroll
            for (int e = 0; e < ROWS; ++e) {
                if (on && h + e * RPW < h1) {
                    x[e] = *reinterpret_cast<const uint4*>(k + e * RPW * D * 2);
                    if (!INTERLEAVED && a.rope.half) z[e] = partners<T>(a.rope, k + (e * RPW * D - ch * 8) * 2, ch);
                    w[e] = *reinterpret_cast<const uint4*>(v + e * RPW * D * 2);
                }
            }
            if (!have) {
                if (lane == 0) atomicOr(a.err, WORKER_BAD_INPUT);
                break;
            }
#pragma unroll
            for (int e = 0; e < ROWS; ++e) {
                if (on && h + e * RPW < h1) {
                    if (a.rope.half) {
                        float f[8], g[8];
                        widen<T>(x[e], f);
                        if (!INTERLEAVED) widen<T>(z[e], g);
                        rotor.turn(f, g);
                        x[e] = narrow<T>(f);
                    }
                    *reinterpret_cast<uint4*>(a.kv.k + dst * 2) = x[e];
                    *reinterpret_cast<uint4*>(a.kv.v + dst * 2) = w[e];
                    if (ch == 0) {
                        if (a.kv.pos) a.kv.pos[m] = p;
                        if (a.kv.weight) a.kv.weight[m] = 0.0f;
                    }
                    dst += RPW * a.kv.head_stride;
                    m += RPW * a.kv.page;
                }
            }
            k += ROWS * RPW * D * 2;
            v += ROWS * RPW * D * 2;
        }
    }
    leave(a, q, all, reinterpret_cast<int*>(scratch));
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

// What 32 bits hold of an exact result, the last bit set where that is not all of it: a rounding to fewer bits then comes out
// as one of the exact result. The product with a scale's ratio, and the quotient by a scale that is no power of two.
__device__ __forceinline__ float sticky(float cut, float rest)
{
    return rest != 0.0f ? __uint_as_float(__float_as_uint(cut) | 1u) : cut;
}
__device__ __forceinline__ float product_of(float z, float f)
{
    const float p = __fmul_rz(z, f);
    return sticky(p, fmaf(z, f, -p));
}
// (a function of its own: in line it costs the kernel 6%, which hardly ever comes here)
__device__ __noinline__ float quotient_of(float x, float s)
{
    if (s < 8.6736174e-19f) x *= 1.8446744e19f, s *= 1.8446744e19f;  // 2^-60, 2^64: so that 32 bits hold the rest
    const float q = __fdiv_rz(x, s);
    return sticky(q, fmaf(-q, s, x));
}

// The least power of two, 2^-126 at least, of which m (finite, >= 0) is 448 = 1.75 2^8 times at most.
__device__ __forceinline__ float scale_of(float m)
{
    const uint32_t u = __float_as_uint(m);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffff) > 0x600000 ? 1 : 0);  // (of subnormal numbers less than 1)
    return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// Rows of a block that a warp has at a time: four chunks a lane.
template <int D>
constexpr int ROWS8 = 4 * (32 / (D / 8));

// `wpu` warps a unit: as many as have its rows, at most all of a CTA. A unit is a block and `many` of its 2 H rows of keys and
// values.
template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(NT, PER_SM) k_append8(AppendArgs a, int wpu, int many)
{
    constexpr int CH = D / 8, RPW = 32 / CH, N = 4, RW = ROWS8<D>;
    extern __shared__ int mem[];
    __shared__ long long scratch[32];
    __shared__ float tops[2][WARPS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = a.kv.kv_heads;
    const int shift = a.scales.block_shift, block = 1 << shift, parts = (2 * H + many - 1) / many;
    Requests q;
    const int all = lay(a, q, mem, scratch, [&](int len, int A) {
        return (long long)(((len + A - 1) >> shift) - (len >> shift) + 1) * parts;
    });
    const int sub = lane / CH, ch = lane - sub * CH;
    const int groups = WARPS / wpu, group = warp / wpu, member = warp - group * wpu, span = wpu * RW;
    Rotor<INTERLEAVED> rotor, by;  // at a row's position; from a lane's row to its next
    if (a.rope.half) {
        rotor.load(a.rope, ch);
        by = rotor;
        by.scale = 1.0f;
        by.at(RPW);
    }
    int round = 0;
    for (long long u0 = (long long)blockIdx.x * groups; u0 < all; u0 += (long long)gridDim.x * groups) {
        const bool any = u0 + group < all;
        const int u = any ? (int)(u0 + group) : 0;
        const int r = plan_find(q.pre, a.tok.n_req, u), y = u - q.pre[r], b = y / parts, hv0 = (y - b * parts) * many;
        const int len = q.len[r];
        const int first = ((len >> shift) + b) << shift;                            // the block's first slot
        const int lo = max(first, len), hi = any ? min(first + block, len + q.count[r]) : lo;  // its new slots
        const int page = a.kv.table[r * a.kv.table_stride + (first >> a.kv.page_shift)];
        const int at = first & (a.kv.page - 1), mine = member * RW + sub;  // this lane's first row
        const bool have = any && (unsigned)page < (unsigned)a.kv.pages;
        if (any && !have && lane == 0 && member == 0) atomicOr(a.err, WORKER_BAD_INPUT);
#pragma unroll 1
        for (int hv = hv0; hv < hv0 + many; ++hv, ++round) {  // (all warps of a group, the same number of times)
            const bool live = have && hv < 2 * H, values = hv >= H;
            const int h = values ? hv - H : hv, end = live ? hi : lo;
            const long long stride = (values ? a.tok.v_stride : a.tok.k_stride) * 2;
            const char* const src = (values ? a.tok.v : a.tok.k) + h * D * 2 + q.lo[r] * stride;
            const bool turned = !values && a.rope.half;
            // this warp's rows from slot s0 on, in 32 bits
            float x[N][8];
            auto load = [&](int s0) {
                uint4 raw[N], mates[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int slot = s0 + mine + i * RPW;
                    raw[i] = mates[i] = make_uint4(0, 0, 0, 0);
                    if (sub < RPW && slot < end) {
                        const char* const row = src + (a.acc ? a.acc[q.a0[r] + slot - len] : slot - len) * stride;
                        raw[i] = *reinterpret_cast<const uint4*>(row + ch * 16);
                        if (!INTERLEAVED && turned) mates[i] = partners<T>(a.rope, row, ch);
                    }
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    widen<T>(raw[i], x[i]);
                    if (turned && s0 + member * RW + i * RPW < end) {
                        if (i % 2 == 0) rotor.at((int)((unsigned)q.next[r] + (unsigned)(s0 + mine + i * RPW - len)));
                        else rotor.on(by);
                        float z[8];
                        if (!INTERLEAVED) widen<T>(mates[i], z);
                        rotor.turn(x[i], z);
                    }
                }
            };
            // their largest magnitude; infinity where it is not to be left out
            auto largest = [&](bool finite) {
                float most = 0.0f;
#pragma unroll 1
                for (int s0 = lo; s0 < end; s0 += span) {
                    load(s0);
#pragma unroll
                    for (int i = 0; i < N; ++i) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float m = fabsf(x[i][j]);
                            most = fmaxf(most, finite && m == INFINITY ? 0.0f : m);
                        }
                    }
                }
#pragma unroll
                for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
                return most;
            };
            float most = largest(false);
            bool wild = most == INFINITY;  // of this warp's rows
            if (wild) most = largest(true);
            float* const held = (values ? a.scales.v : a.scales.k) +
                                (live ? ((long long)page * H + h) * a.scales.per_page + (at >> shift) : 0);
            const float old = live && lo > first ? *held : 0.0f;
            if (wpu > 1) {
                if (lane == 0) tops[round & 1][warp] = most;
                // the group's warps alone (the scale has been read by all when the first writes it; two sets of maxima: one may
                // be a round behind)
                asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(wpu * 32) : "memory");
                for (int w = 0; w < wpu; ++w) most = fmaxf(most, tops[round & 1][group * wpu + w]);
            } else {
                __syncwarp();  // (all lanes have read the scale when the first writes it)
            }
            if (!live) continue;
            float scale = scale_of(most);
            char* const dst = (values ? a.kv.v : a.kv.k) + page * a.kv.page_stride + h * a.kv.head_stride +
                              at * a.kv.token_stride + ch * 8;
            if (lo > first) {
                if (scale > old) {
                    const float f = old / scale;
                    for (int slot = first + member * RPW + sub; slot < lo && sub < RPW; slot += wpu * RPW) {
                        uint2* const d = reinterpret_cast<uint2*>(dst + (slot - first) * a.kv.token_stride);
                        const uint2 c = *d;
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 z = values2((j < 2 ? c.x : c.y) >> (j & 1) * 16);
                            w[j] = codes2(product_of(z.x, f), product_of(z.y, f));
                        }
                        *d = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
                    }
                } else {
                    scale = old;
                }
            }
            const bool power = !(__float_as_uint(scale) & 0x7fffff);
            const float inv = power ? 1.0f / scale : 1.0f;
#pragma unroll 1
            for (int s0 = lo; s0 < end; s0 += span) {
                if (end - lo > span) load(s0);
                if (wild) {  // what is infinite becomes NaN, as conversions of NaN are, not the largest number
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[i][j] += x[i][j] - x[i][j];
                }
                if (!power) {  // (a held scale of another origin)
#pragma unroll
                    for (int i = 0; i < N; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) x[i][j] = quotient_of(x[i][j], scale);
                }
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int slot = s0 + mine + i * RPW;
                    if (sub < RPW && slot < end)
                        *reinterpret_cast<uint2*>(dst + (slot - first) * a.kv.token_stride) =
                            make_uint2(codes2(x[i][0] * inv, x[i][1] * inv) | codes2(x[i][2] * inv, x[i][3] * inv) << 16,
                                       codes2(x[i][4] * inv, x[i][5] * inv) | codes2(x[i][6] * inv, x[i][7] * inv) << 16);
                }
            }
            if (lane == 0 && member == 0) *held = scale;
        }
    }
    leave(a, q, all, reinterpret_cast<int*>(scratch));
}

template <typename T, int D, bool INTERLEAVED>
cudaError_t launch_kind(const AppendArgs& a, int sms, cudaStream_t st)
{
    constexpr int RPW = 32 / (D / 8);
    const size_t smem = Requests::bytes(a.tok.n_req);
    const int H = a.kv.kv_heads;
    // CTAs that have a unit, as many as run at once at most
    auto ctas = [&](long long units, int a_cta) {
        const long long want = (units + a_cta - 1) / a_cta;
        return (int)(want < (long long)PER_SM * sms ? want : PER_SM * sms);
    };
    if (a.scales.k) {
        // as many warps a unit as have the rows that a request's new tokens, on average, bring to a block
        const long long mean = ((long long)a.n_acc + a.tok.n_req - 1) / a.tok.n_req, block = 1 << a.scales.block_shift;
        const long long rows = mean < block ? mean : block;
        int wpu = 1;
        while (wpu < WARPS && wpu * ROWS8<D> < rows) wpu *= 2;
        // (a request's tokens enter two blocks more than they fill, at most)
        const long long blocks = ((long long)a.n_acc >> a.scales.block_shift) + 2ll * a.tok.n_req;
        // several rows of heads a unit where there are 4 units for every group of warps all the same
        long long many = blocks * 2 * H * wpu / (4ll * WARPS * PER_SM * sms);
        many = many < 1 ? 1 : many < 2 * H ? many : 2 * H;
        const long long of = (2 * H + many - 1) / many;  // units of a block, of even size
        many = (2 * H + of - 1) / of;
        k_append8<T, D, INTERLEAVED><<<ctas(blocks * ((2 * H + many - 1) / many), WARPS / wpu), NT, smem, st>>>(a, wpu, (int)many);
    } else {
        // heads of a unit: all, or as few as give every warp a unit, a warp's loads at least
        const long long want = ((long long)PER_SM * sms * WARPS + a.n_acc - 1) / a.n_acc;
        int heads = (int)((H + want - 1) / want);
        heads = (heads + RPW - 1) / RPW * RPW;
        k_append<T, D, INTERLEAVED><<<ctas((long long)a.n_acc * ((H + heads - 1) / heads), WARPS), NT, smem, st>>>(a, heads);
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
