// aladdin_worker_attend8 where the rows of a (request, key head) are few. See attend8.cuh for the operator.
//
// Every cached byte is read once and next to nothing is computed with it: what counts is bytes in flight
// and few instructions a byte. As in the attention over 16 bits, every warp works alone on a range of the axis of
// all key tiles, with a few tiles of shared memory that it fills by asynchronous copies ahead, and the products
// are formed transposed: keys by rows, then channels by rows, 8 rows an operand. The codes become half-precision operands
// in registers, one conversion for two values (products of e4m3 take conversions and 32-bit additions of their own on
// this GPU: 60 us for 57). No lane needs another one's codes:
//   scores    the index that is summed over, the channels, may be taken in any order, the same for both operands:
//             a lane takes runs of 4 channels, so that the two halves of a word are the pairs that it needs;
//   results   a lane takes the same channels of 16 keys' 2t, 2t + 1, 2t + 8, 2t + 9 and interleaves the bytes
//             of two keys; which of its channels stands for which row of the operand is its own choice again, so that
//             a lane ends with runs of channels of two rows and writes them as they are.
// Chunks of 16 bytes are exchanged within a tile so that the loads of both meet different banks.
//
// New tokens have tiles of their own, 16 bits wide. Their scores are matrix products in the worker's type; their values,
// few a row, are added in 32 bits one by one, which leaves out what a row does not see even where it is
// not finite.
//
// Measured: two requests of 110,108 cached tokens, 32 heads of 64 channels in f16, scales for 64 tokens: 86 us, 5.2 TB/s of
// 6.75 that a copy reaches; 128 requests of 83,336 tokens, 32 query and 8 key heads of 128 channels in bf16: 48 us, 3.6
// TB/s. There 6 us go by until the first codes are there and 10 to 15 in the ends of units, where what another SM wrote is
// 1,500 cycles away; in between two warps a scheduler wait for their own results, and for instructions: code that few tiles need
// costs all of them where it lies between theirs.
#include "attend8.cuh"

namespace aladdin {
namespace wk {
namespace {

template <int D, int NB>
struct Few8 {
    static constexpr int TK = D == 64 ? 64 : D == 256 ? 16 : 32;      // cached keys of a tile
    static constexpr int TN = TK / 2;                                 // new keys of a tile
    static constexpr int KB = TK / 16;                                // blocks of 16 keys
    // of a CTA, one CTA an SM (two long requests with 64 channels: 8 warps 92 us, 12 warps 85; 128 channels need more
    // registers than 12 warps have)
    static constexpr int WARPS = D == 64 && NB == 1 ? 12 : 8;
    static constexpr int S = WARPS == 8 ? 3 : 2;                      // tiles of a warp
    static constexpr int TILE = 2 * TK * D;                           // keys, then values
    static constexpr int SLOT = TILE + 32;                            // and the scales of 16 keys each, then of 16 values
    typedef typename std::conditional<TK == 64, unsigned long long, unsigned>::type Mask;  // a bit for each key
    static constexpr Mask FULL = TK == 16 ? (Mask)0xffff : ~(Mask)0;
    static constexpr int oks = WARPS * S * SLOT;                      // masks of tiles
    static constexpr int ds = oks + WARPS * S * 8;                    // the rows' d, where they differ
    static constexpr int pending = ds + WARPS * NB * 8 * 4;           // a warp's Pending
    static constexpr int pre = pending + WARPS * 24;
    static constexpr int scratch = 0;                                 // of the plan, in front of all tiles
    // (up to 196 KB, some 70 requests, leave the cache of the SM twice as much as more would, which registers in local memory
    // need: 64 requests of 1,000 tokens, 256 channels, 99 us for 61)
    static constexpr int bytes(int n_req) { return pre + Axis8::ints(n_req) * 4; }

    // byte of chunk c (16 bytes) of a tile's row, keys and values
    static __device__ __forceinline__ int key_at(int row, int c)
    {
        return row * D + (D % 128 == 0 ? c ^ (row & 1) << 2 : c) * 16;
    }
    static __device__ __forceinline__ int value_at(int row, int c)
    {
        if (D == 64) return (row >> 1) * 128 + (((row & 1) * 4 + c) ^ (row >> 1 & 3) << 1) * 16;
        return row * D + (D % 128 == 0 ? c ^ (row >> 1 & 3) << 1 : c) * 16;
    }
    // first of the 4 channels that lane t of 4 has in the x-th product of 16 channels
    static __device__ __forceinline__ int key_channel(int x, int t)
    {
        return D == 96 ? 32 * (x / 2) + 8 * t + 4 * (x % 2) : 64 * (x / 4) + 16 * t + 4 * (x % 4);
    }
    // first of the 4 channels of the w-th word that lane g of 8 has of a value
    static __device__ __forceinline__ int value_channel(int w, int g)
    {
        if (D == 96) return 32 * w + 4 * g;
        if (D == 64) return 8 * g + 4 * w;
        return 128 * (w / 4) + 16 * g + 4 * (w % 4);
    }
};

// Keys of a place in calls that give every warp few tiles, and what a unit costs beside
// its tiles, in keys.
constexpr int PLACE_KEYS = 64, UNIT_KEYS = 64;

// Room of the weights in half precision (attend8.cuh): a row's maximum does not lag.
constexpr float UP = 15.0f;

// The largest of the 8 lanes that hold a row.
__device__ __forceinline__ float row_max(float v)
{
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, x));
    return v;
}

// What a tile of cached keys whose logarithms are not all near d works on: a lane's scores as they are, their logarithms, its
// rows' state, what their results are multiplied by, and the d of all rows.
template <int KB, int NB>
struct Far {
    float s[KB][NB][4], lv[KB], M[NB][2], l[NB][2], d[NB][2], f[NB][2], all;
};

// Weights in the place of scores; whether the rows have a d each from here on, in row_d.
template <int KB, int NB>
__device__ __noinline__ bool far_tile(Far<KB, NB>& t, float* row_d)
{
    const int lane = threadIdx.x & 31, gq = lane >> 2, tq = lane & 3;
    float least = INFINITY, most = -INFINITY;
#pragma unroll 1
    for (int r = 0; r < NB * 2; ++r) {
        const int y = r >> 1, e = r & 1;
        const float before = t.d[y][e], m = t.M[y][e] - before;
        float top = -INFINITY, with = -INFINITY;
#pragma unroll
        for (int x = 0; x < KB; ++x) top = fmaxf(top, fmaxf(t.s[x][y][e], t.s[x][y][e + 2]));
        const float to = fmaxf(m, row_max(top)), base = to == -INFINITY ? 0.0f : to;
        // (differences first: next to scores of any size logarithms would be lost)
#pragma unroll
        for (int x = 0; x < KB; ++x) with = fmaxf(with, (fmaxf(t.s[x][y][e], t.s[x][y][e + 2]) - base) + t.lv[x]);
        const float by = m - base, next = fmaxf(fmaxf(before + by, row_max(with)), 2 * LOG_ZERO);
        float l = t.l[y][e] * ex2(by);
#pragma unroll
        for (int x = 0; x < KB; ++x) {
#pragma unroll
            for (int z = 0; z < 4; z += 2) {
                const float w = t.s[x][y][e + z] - base;
                l += ex2(w);
                t.s[x][y][e + z] = ex2(w + (t.lv[x] - next + UP));
            }
        }
        t.f[y][e] = ex2(by + (before - next));
        t.l[y][e] = l;
        t.M[y][e] = to == -INFINITY ? to : __fadd_ru(to, next);
        t.d[y][e] = next;
        least = fminf(least, next);
        most = fmaxf(most, next);
    }
#pragma unroll
    for (int x = 1; x < 4; x <<= 1) {
        least = fminf(least, __shfl_xor_sync(0xffffffffu, least, x));
        most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
    }
    // one d for all rows again, where it does
    const bool single = most - least > FAR;
    __syncwarp();
#pragma unroll 1
    for (int r = 0; r < NB * 2; ++r) {
        const int y = r >> 1, e = r & 1;
        if (!single) t.l[y][e] *= ex2(least - t.d[y][e]);
        else if (gq == 0) row_d[y * 8 + tq * 2 + e] = t.d[y][e];
    }
    __syncwarp();
    t.all = least;
    return single;
}

// A unit whose partial results the workers first .. last left.
struct Pending {
    int h, rt, lo, T;  // of its Cursor
    int first, last;
};
static_assert(sizeof(Pending) == 24, "the room for it");

// N consecutive floats that other warps wrote
template <int N>
__device__ __forceinline__ void load_row(float (&v)[N], const float* p)
{
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(p + i));
            v[i] = x.x, v[i + 1] = x.y, v[i + 2] = x.z, v[i + 3] = x.w;
        }
    } else if constexpr (N == 2) {
        const float2 x = __ldcg(reinterpret_cast<const float2*>(p));
        v[0] = x.x, v[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __ldcg(p + i);
    }
}

// The rows below live of a unit; one warp, D / 32 columns a lane. What another SM wrote is 1,500 cycles away: the maxima and sums of up to 32 partial results, one a lane, and
// the columns of up to four of them are on their way together.
template <typename T, int D, int RM>
__device__ __forceinline__ void join_rows8(const AttendArgs& a, const Pending& u, int live, int lane)
{
    const int first = u.first, last = u.last;
    // (fewer together where accumulators and queries take most registers anyway: the kernel around this keeps to registers but
    // with 64 channels and 12 warps, 60 bytes a thread, and with 256 of bfloat16, 350)
    constexpr int N = D / 32, U = D == 256 ? 1 : D * RM > 8 * 128 ? 2 : 4, ROWS = 4;
    const int G = a.kv.group;
#pragma unroll 1
    for (int r0 = 0; r0 < live; r0 += ROWS) {
        float ref[ROWS], sum[ROWS], acc[ROWS][N];
#pragma unroll
        for (int y = 0; y < ROWS; ++y) {
            ref[y] = -INFINITY;
            sum[y] = 0.0f;
#pragma unroll
            for (int x = 0; x < N; ++x) acc[y][x] = 0.0f;
        }
#pragma unroll 1
        for (int i0 = first; i0 <= last; i0 += 32) {
            const int count = min(32, last - i0 + 1), mine = i0 + min(lane, count - 1);
            float2 ml[ROWS];
            {
                const float* const p = part_of<D, RM>(a, mine, mine == first);
#pragma unroll
                for (int y = 0; y < ROWS; ++y)
                    ml[y] = __ldcg(reinterpret_cast<const float2*>(p + min(r0 + y, live - 1) * 2));
            }
            float f[ROWS];
#pragma unroll 1
            for (int k0 = 0; k0 < count; k0 += U) {
                float v[U][ROWS][N];
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    const int i = i0 + min(k0 + k, count - 1);
                    const float* const p = part_of<D, RM>(a, i, i == first) + RM * 2 + lane * N;
#pragma unroll
                    for (int y = 0; y < ROWS; ++y) load_row(v[k][y], p + min(r0 + y, live - 1) * D);
                }
                if (k0 == 0) {
                    // this lane's factor to the largest maximum so far, and what came before to that
#pragma unroll
                    for (int y = 0; y < ROWS; ++y) {
                        float top = fmaxf(ref[y], ml[y].x);
#pragma unroll
                        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                        const float base = top == -INFINITY ? 0.0f : top, g = ex2(ref[y] - base);
                        f[y] = lane < count ? part_factor(ml[y], base) : 0.0f;
                        sum[y] = sum[y] * g + (lane < count ? fabsf(ml[y].y) * f[y] : 0.0f);
#pragma unroll
                        for (int x = 0; x < N; ++x) acc[y][x] *= g;
                        ref[y] = top;
                    }
                }
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    if (k0 + k >= count) break;
#pragma unroll
                    for (int y = 0; y < ROWS; ++y) {
                        const float w = __shfl_sync(0xffffffffu, f[y], k0 + k);
#pragma unroll
                        for (int x = 0; x < N; ++x) acc[y][x] += w * v[k][y][x];
                    }
                }
            }
        }
#pragma unroll
        for (int y = 0; y < ROWS; ++y) {
#pragma unroll
            for (int x = 16; x; x >>= 1) sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], x);
            const int rr = r0 + y;
            if (rr >= live) break;
            const int rho = u.rt * RM + rr, t = rho / G, head = u.h * G + rho - t * G;
            const float inv = 1.0f / sum[y];
            const auto of = [&](float x) { return sum[y] == 0.0f ? 0.0f : x * inv; };
            char* const d = a.out + ((u.lo + t) * a.out_stride + (long long)head * D + lane * N) * 2;
            if constexpr (N % 2 == 0) {
#pragma unroll
                for (int x = 0; x < N; x += 2)
                    *reinterpret_cast<uint32_t*>(d + x * 2) = Num<T>::pack(of(acc[y][x]), of(acc[y][x + 1]));
            } else {
#pragma unroll
                for (int x = 0; x < N; ++x)
                    *reinterpret_cast<unsigned short*>(d + x * 2) = (unsigned short)Num<T>::pack(of(acc[y][x]), 0.0f);
            }
            if (lane == 0 && a.lse)
                a.lse[(long long)(u.lo + t) * (a.kv.kv_heads * G) + head] =
                    ((ref[y] == -INFINITY ? 0.0f : ref[y]) + log2f(sum[y])) * LN2;
        }
    }
}

// NB: blocks of 8 rows.
template <typename T, int D, int NB>
__global__ void __launch_bounds__(Few8<D, NB>::WARPS * 32, 1) k_attend8_few(Attend8Args a)
{
    constexpr int RM = NB * 8;
    using L = Few8<D, NB>;
    constexpr int TK = L::TK, TN = L::TN, S = L::S, NT = L::WARPS * 32;
    constexpr int KB = L::KB, MO = D / 16, NW = D / 32;  // blocks of 16 keys, of 16 channels; words of a value a lane
    typedef typename L::Mask Mask;
    extern __shared__ __align__(128) char sm[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.kv.group, H = a.kv.kv_heads;
    char* const tiles = sm + warp * S * L::SLOT;
    const uint32_t tiles0 = smem_addr(tiles);
    Mask* const oks = reinterpret_cast<Mask*>(sm + L::oks) + warp * S;
    float* const row_d = reinterpret_cast<float*>(sm + L::ds) + warp * NB * 8;

    Axis8 ax;
    if (!plan8<NT, TK, TN, RM>(a, ax, reinterpret_cast<int*>(sm + L::pre), reinterpret_cast<long long*>(sm + L::scratch),
                               (int)gridDim.x * L::WARPS, UNIT_KEYS / TK, PLACE_KEYS / TK))
        return;
    // neighbouring ranges lie on different SMs
    const int me = warp * gridDim.x + blockIdx.x;
    if (me >= ax.workers) return;
    Cursor C, F;  // the tile computed, the tile fetched
    const int n = range8<TK, TN, RM>(a, ax, C, me);
    F = C;
    // of F's unit: its row of the table, its head in the pool and among the scales
    const int32_t* row_F;
    const char* keys_F;
    auto unit = [&]() {
        row_F = a.kv.table + (long long)F.r * a.kv.table_stride;
        keys_F = a.kv.k + F.h * a.kv.head_stride;
    };
    // the page of 16 keys of the tile under F, as the table has it: of block lane % KB
    int page;
    auto find = [&]() {
        const int key = F.tile * TK + lane % KB * 16;
        page = key < F.len ? row_F[key >> a.kv.page_shift] : -1;
    };
    unit();
    find();
    // this lane's chunks of a tile's rows: 16 bytes of rows row0, row0 + 32 / CH, ..
    constexpr int CH = D / 16, NI = TK * CH / 32;
    auto row_of = [&](int i) { return 32 % CH == 0 ? lane / CH + i * (32 / CH) : (lane + i * 32) / CH; };
    auto chunk_of = [&](int i) { return 32 % CH == 0 ? lane % CH : (lane + i * 32) % CH; };
    const long long from0 = row_of(0) * a.kv.token_stride + chunk_of(0) * 16, apart = a.kv.v - a.kv.k;
    const long long rows_on = (32 % CH == 0 ? 32 / CH : 16) * a.kv.token_stride;  // (D 96: three chunks, then 16 rows on)
    const bool one_page = a.kv.page >= TK;
    // the tile under F into place b; then F goes on
    auto fetch = [&](int b, bool more) {
        const int key0 = F.tile * TK, own = F.len - key0;  // cached keys from the tile's start
        const uint32_t d = tiles0 + b * L::SLOT;
        if (own > 0) {
            const int at = key0 & (a.kv.page - 1), page0 = __shfl_sync(0xffffffffu, page, 0);
            Mask mask = L::FULL;
            if (one_page && own >= TK && (unsigned)page0 < (unsigned)a.kv.pages) {
                const char* k = keys_F + page0 * a.kv.page_stride + at * a.kv.token_stride;
                if constexpr (32 % CH == 0) {
                    k += from0;
                    const char* v = k + apart;
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        cp16(d + L::key_at(row_of(i), chunk_of(i)), k, true);
                        cp16(d + TK * D + L::value_at(row_of(i), chunk_of(i)), v, true);
                        k += rows_on;
                        v += rows_on;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
                        const char* p = k + row_of(i) * a.kv.token_stride + chunk_of(i) * 16;
#pragma unroll
                        for (int g = 0; g < KB; ++g) {
                            cp16(d + L::key_at(g * 16 + row_of(i), chunk_of(i)), p, true);
                            cp16(d + TK * D + L::value_at(g * 16 + row_of(i), chunk_of(i)), p + apart, true);
                            p += rows_on;
                        }
                    }
                }
            } else {
                // rows behind the last key or on other pages (weights of 0 meet the codes of rows that hold no key: zeros)
                const bool have = (unsigned)page < (unsigned)a.kv.pages;
                const unsigned pages = __ballot_sync(0xffffffffu, have);
#pragma unroll 1
                for (int i = 0; i < NI; ++i) {
                    const int row = (lane + i * 32) / CH, ch = (lane + i * 32) % CH;
                    const int p = __shfl_sync(0xffffffffu, page, row >> 4);
                    const bool ok = row < own && (pages >> (row >> 4) & 1);
                    const char* const k =
                        ok ? keys_F + p * a.kv.page_stride + ((key0 + row) & (a.kv.page - 1)) * a.kv.token_stride + ch * 16 : a.kv.k;
                    cp16(d + L::key_at(row, ch), k, ok);
                    cp16(d + TK * D + L::value_at(row, ch), k + apart, ok);
                }
                mask = own >= TK ? L::FULL : ((Mask)1 << own) - 1;
#pragma unroll
                for (int g = 0; g < KB; ++g)
                    if (!(pages >> g & 1)) mask &= ~((Mask)0xffff << (g * 16));
                if (lane < KB && lane * 16 < own && !have) atomicOr(a.err, WORKER_BAD_INPUT);
            }
            if (lane < 2 * KB) {
                const bool ok = (unsigned)page < (unsigned)a.kv.pages;
                const long long e = ok ? ((long long)page * H + F.h) * a.scales.per_page +
                                             (((key0 + lane % KB * 16) & (a.kv.page - 1)) >> a.scales.block_shift)
                                       : 0;
                cp4(d + L::TILE + lane * 4, (lane < KB ? a.scales.k : a.scales.v) + e, ok);
            }
            if (lane == 0) oks[b] = mask;
        } else {
            const int first = (F.tile - (F.len + TK - 1) / TK) * TN;
            constexpr int CH = D / 8;
#pragma unroll 1
            for (int i = 0; i < TN * CH / 32; ++i) {
                const int x = lane + i * 32, row = x / CH, ch = x - row * CH;
                const bool ok = first + row < F.T;
                const long long t = F.lo + (ok ? first + row : 0);
                cp16(d + row * (D * 2) + ch * 16, a.tok.k + (t * a.tok.k_stride + F.h * D + ch * 8) * 2, ok);
                cp16(d + TK * D + row * (D * 2) + ch * 16, a.tok.v + (t * a.tok.v_stride + F.h * D + ch * 8) * 2, ok);
            }
        }
        if (more) {
            advance8<TK, TN, RM>(a, ax, F);
            if (F.tile == 0) unit();
            find();
        }
    };
    const int gq = lane >> 2, tq = lane & 3;
    uint32_t qf[MO][NB][2];   // row gq of every block, in half precision
    float factor[NB][2];      // of the scores of rows 2 tq, 2 tq + 1, to base 2
    // this lane's channels of row gq of block y in the worker's type
    auto query = [&](const Cursor& u, int y, int x) -> uint2 {
        const int rho = u.rt * RM + y * 8 + gq;
        if (rho >= u.T * G) return make_uint2(0u, 0u);
        const int t = rho / G;
        return __ldg(reinterpret_cast<const uint2*>(
            a.tok.q + ((u.lo + t) * a.tok.q_stride + (long long)(u.h * G + rho - t * G) * D + L::key_channel(x, tq)) * 2));
    };

    // the next unit's queries are on their way while one is computed, the first ones in front of all keys
    // (256 channels, and 16 rows of 128, leave no registers for that)
    constexpr bool AHEAD = D * NB < 256;
    uint2 qn[AHEAD ? MO : 1][NB];
    auto queries_of = [&](const Cursor& u) {
        if constexpr (AHEAD) {
#pragma unroll
            for (int y = 0; y < NB; ++y)
#pragma unroll
                for (int x = 0; x < MO; ++x) qn[x][y] = query(u, y, x);
        }
    };
    queries_of(C);
#pragma unroll
    for (int j = 0; j < S - 1; ++j) {
        if (j < n) fetch(j, j + 1 < n);
        cp_commit();
    }

    float o[MO][NB][4], M[NB][2], l[NB][2];  // channels of rows 2 tq, 2 tq + 1, and what attend8.cuh says
    float d = 0.0f;
    bool single = false;                     // whether the rows have a d each
    float unscale[NB];                       // of row gq of every block
    bool fresh = true, wild = false;         // whether the unit's results hold values that are not finite
    int b = 0, tile0 = 0;  // a tile's place; the first tile of the unit that this warp has
    // A unit that warps share and whose part this one has written: a tile later it says so, and at the end of its next
    // unit it looks whether it was the last one to, which joins the parts; neither is waited for while there are tiles.
    Pending& P = *reinterpret_cast<Pending*>(sm + L::pending + warp * 24);
    int pend = 0, p_before = 0;  // 1: written, 2: said

    for (int j = 0; j < n; ++j) {
        __syncwarp();
        if (j + S - 1 < n) fetch(b == 0 ? S - 1 : b - 1, j + S < n);
        cp_commit();
        const int rows = C.T * G - C.rt * RM;
        if (fresh) {
            fresh = wild = single = false;
            tile0 = C.tile;
            d = 0.0f;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int x = 0; x < MO; ++x) o[x][y][0] = o[x][y][1] = o[x][y][2] = o[x][y][3] = 0.0f;
                M[y][0] = M[y][1] = -INFINITY;
                l[y][0] = l[y][1] = 0.0f;
                uint2 q[MO];
#pragma unroll
                for (int x = 0; x < MO; ++x) q[x] = AHEAD ? qn[AHEAD ? x : 0][y] : query(C, y, x);
                float back = half_row<T, MO>(q);
                unscale[y] = back;
#pragma unroll
                for (int x = 0; x < MO; ++x) {
                    qf[x][y][0] = q[x].x;
                    qf[x][y][1] = q[x].y;
                }
                back *= a.scale_log2;
                factor[y][0] = __shfl_sync(0xffffffffu, back, tq * 8);
                factor[y][1] = __shfl_sync(0xffffffffu, back, tq * 8 + 4);
            }
            if (AHEAD && j + C.c - C.tile < n) {  // the range goes on behind this unit
                Cursor u = C;
                next_unit8<TK, TN, RM>(a, ax, u);
                queries_of(u);
            }
        }
        cp_wait<S - 1>();
        __syncwarp();
        const char* const slot = tiles + b * L::SLOT;
        const bool cached = C.tile * TK < C.len;
        const int first = cached ? 0 : (C.tile - (C.len + TK - 1) / TK) * TN;  // the first new token

        float s[KB][NB][4];  // keys gq, gq + 8 of a block by rows 2 tq, 2 tq + 1
        float lv[KB];          // logarithms of the scales of the blocks' values, or of what key gq of a block has for one
        float hi = -INFINITY;  // the largest
        unsigned seen = 0;     // by the rows, of this lane's new keys
        bool odd = true;       // whether a row's d is not within reach of all of them (attend8.cuh)
        if (cached) {
            // (a block without keys has no part, and one whose scale is none makes its scores NaN)
            const Mask okm = oks[b];
            const float* const scales = reinterpret_cast<const float*>(slot + L::TILE);
            float lo = INFINITY;
#pragma unroll
            for (int x = 0; x < KB; ++x) {
                lv[x] = log_scale(scales[KB + x]);
                hi = fmaxf(hi, lv[x]);
                lo = fminf(lo, lv[x]);
            }
            if (okm != L::FULL) {
                hi = -INFINITY, lo = INFINITY;
#pragma unroll
                for (int x = 0; x < KB; ++x) {
                    if (okm >> (x * 16) & 1) hi = fmaxf(hi, lv[x]), lo = fminf(lo, lv[x]);
                }
                if (hi == -INFINITY) hi = d;
#pragma unroll
                for (int x = 0; x < KB; ++x) lv[x] = okm >> (x * 16) & 1 ? lv[x] : hi;
            }
            if (C.tile == tile0) d = hi;
            odd = single || hi > d + FAR || lo < d - FAR;
        }
        if (cached) {
            const Mask okm = oks[b];
            const float* const scales = reinterpret_cast<const float*>(slot + L::TILE);
#pragma unroll
            for (int x = 0; x < KB; ++x) {
                // scores come with their scale's logarithm, from the largest one on, where that is in reach
                const float with = lv[x] - (odd ? lv[x] : hi);
#pragma unroll
                for (int y = 0; y < NB; ++y) s[x][y][0] = s[x][y][1] = s[x][y][2] = s[x][y][3] = 0.0f;
                constexpr int CW = D == 96 ? 2 : 4;  // words of a load
#pragma unroll
                for (int i = 0; i < MO / CW; ++i) {
                    uint32_t w[2][CW];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = x * 16 + e * 8 + gq;
                        if constexpr (D == 96) {
                            const uint2 v = *reinterpret_cast<const uint2*>(slot + row * D + i * 32 + tq * 8);
                            w[e][0] = v.x, w[e][1] = v.y;
                        } else {
                            const uint4 v = *reinterpret_cast<const uint4*>(slot + L::key_at(row, i * 4 + tq));
                            w[e][0] = v.x, w[e][1] = v.y, w[e][2] = v.z, w[e][3] = v.w;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < CW; ++c) {
                        const uint32_t f[4] = {half2_lo(w[0][c]), half2_lo(w[1][c]), half2_hi(w[0][c]), half2_hi(w[1][c])};
#pragma unroll
                        for (int y = 0; y < NB; ++y) Num<__half>::mma(s[x][y], f, qf[i * CW + c][y][0], qf[i * CW + c][y][1]);
                    }
                }
                const float ks = finite_scale(scales[x]);
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    const float k0 = ks * factor[y][0], k1 = ks * factor[y][1];
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[x][y][e] = fmaf(s[x][y][e], e & 1 ? k1 : k0, with);
                }
            }
            if (okm != L::FULL) {
#pragma unroll
                for (int x = 0; x < KB; ++x)
#pragma unroll
                    for (int y = 0; y < NB; ++y)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!(okm >> (x * 16 + (e >> 1) * 8 + gq) & 1)) s[x][y][e] = -INFINITY;
            }
        } else {
            // what the rows see (looked for here: between the tiles it would cost registers)
            unsigned long long see[NB][2];
            if (C.T > 1) {
                const Ancestors tree(a, C, lane);
#pragma unroll
                for (int y = 0; y < NB; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int rr = y * 8 + tq * 2 + e;
                        see[y][e] = tree.of(rr < rows ? (C.rt * RM + rr) / G : 0);
                    }
            } else {
#pragma unroll
                for (int y = 0; y < NB; ++y) see[y][0] = see[y][1] = 1;
            }
            // 8 new keys in the place of 16
#pragma unroll
            for (int x = 0; x < KB; ++x) {
                // as if their values, of which the largest finite one counts, were codes of up to 2^9
                lv[x] = -110.0f;  // (2^110 2^UP is what 32-bit weights of them have room for)
                if (first + x * 8 < C.T) {
                    const uint4* const v = reinterpret_cast<const uint4*>(slot + TK * D + (x * 8 + gq) * (D * 2)) + tq;
                    uint32_t most = 0;
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
                        most = largest2(largest2(largest2(largest2(most, v[i * 4].x), v[i * 4].y), v[i * 4].z), v[i * 4].w);
                    if (__any_sync(0xffffffffu, Num<T>::wild(most))) {
                        wild = true;
                        most = 0;
#pragma unroll 1
                        for (int i = 0; i < D / 8; ++i) most = largest2(most, Num<T>::tame(reinterpret_cast<const uint32_t*>(v + i / 4 * 4)[i % 4]));
                    }
                    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = __vmaxu2(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    lv[x] = fmaxf((float)(exponent<T>(most) - 135), -110.0f);
                }
#pragma unroll
                for (int y = 0; y < NB; ++y) s[x][y][0] = s[x][y][1] = s[x][y][2] = s[x][y][3] = 0.0f;
#pragma unroll
                for (int i = 0; i < MO; ++i) {
                    const uint2 v = *reinterpret_cast<const uint2*>(slot + (x * 8 + gq) * (D * 2) + L::key_channel(i, tq) * 2);
                    const uint32_t f[4] = {v.x, 0u, v.y, 0u};
#pragma unroll
                    for (int y = 0; y < NB; ++y) {
                        Num<T>::mma(s[x][y], f, from_half<T>(qf[i][y][0], unscale[y]), from_half<T>(qf[i][y][1], unscale[y]));
                    }
                }
                const int key = first + x * 8 + gq;
#pragma unroll
                for (int y = 0; y < NB; ++y) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const bool is = key < C.T && (see[y][e] >> key & 1);
                        s[x][y][e] = is ? s[x][y][e] * a.scale_log2 : -INFINITY;
                        seen |= (unsigned)is << (x * NB + y) * 2 + e;
                        s[x][y][e + 2] = -INFINITY;
                    }
                }
            }
        }

        if (!odd) {
            float top[NB][2];
            bool higher = false;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float t = -INFINITY;
#pragma unroll
                    for (int x = 0; x < KB; ++x) t = fmaxf(t, fmaxf(s[x][y][e], s[x][y][e + 2]));
                    top[y][e] = __fadd_ru(t, hi);
                    higher = higher || top[y][e] > M[y][e];
                }
            }
            if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
                for (int y = 0; y < NB; ++y) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float to = fmaxf(M[y][e], row_max(top[y][e])), f = to > M[y][e] ? ex2(M[y][e] - to) : 1.0f;
                        M[y][e] = to;
                        l[y][e] *= f;
#pragma unroll
                        for (int x = 0; x < MO; ++x) {
                            o[x][y][e] *= f;
                            o[x][y][e + 2] *= f;
                        }
                    }
                }
            }
            const float up = hi + UP;
            float back[KB];
#pragma unroll
            for (int x = 0; x < KB; ++x) back[x] = ex2(d - UP - lv[x]);
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float at = __fadd_ru(M[y][e] == -INFINITY ? 0.0f : M[y][e], -up);
#pragma unroll
                    for (int x = 0; x < KB; ++x) {
                        s[x][y][e] = ex2(s[x][y][e] - at);
                        s[x][y][e + 2] = ex2(s[x][y][e + 2] - at);
                        l[y][e] += (s[x][y][e] + s[x][y][e + 2]) * back[x];
                    }
                }
            }
        } else if (cached) {
            // (a function of its own, by way of local memory: its code between the tiles' would cost every one of them, 20 rows of 64
            // channels 10%)
            Far<KB, NB> far;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    far.M[y][e] = M[y][e], far.l[y][e] = l[y][e];
                    far.d[y][e] = single ? row_d[y * 8 + tq * 2 + e] : d;
                }
#pragma unroll
                for (int x = 0; x < KB; ++x) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) far.s[x][y][e] = s[x][y][e];
                }
            }
#pragma unroll
            for (int x = 0; x < KB; ++x) far.lv[x] = lv[x];
            far.all = d;
            single = far_tile<KB, NB>(far, row_d);
            d = far.all;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    M[y][e] = far.M[y][e], l[y][e] = far.l[y][e];
                    const float f = far.f[y][e];
#pragma unroll
                    for (int x = 0; x < MO; ++x) {
                        o[x][y][e] *= f;
                        o[x][y][e + 2] *= f;
                    }
                }
#pragma unroll
                for (int x = 0; x < KB; ++x) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[x][y][e] = far.s[x][y][e];
                }
            }
        } else {
            // new tokens have a logarithm each. (Differences first: next to scores of any size logarithms would be lost)
            float f[NB][2], next[NB][2];
            bool moved = false;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float before = single ? row_d[y * 8 + tq * 2 + e] : d, m = M[y][e] - before;
                    float top = -INFINITY, with = -INFINITY;
#pragma unroll
                    for (int x = 0; x < KB; ++x) top = fmaxf(top, s[x][y][e]);
                    const float to = fmaxf(m, row_max(top)), base = to == -INFINITY ? 0.0f : to;
#pragma unroll
                    for (int x = 0; x < KB; ++x) with = fmaxf(with, (s[x][y][e] - base) + lv[x]);
                    const float by = m - base;
                    next[y][e] = fmaxf(fmaxf(before + by, row_max(with)), 2 * LOG_ZERO);
                    f[y][e] = ex2(by + (before - next[y][e]));
                    if (wild) f[y][e] = fmaxf(f[y][e], NORMAL);
                    moved = moved || f[y][e] != 1.0f;
                    l[y][e] *= ex2(by);
                    M[y][e] = to == -INFINITY ? to : __fadd_ru(to, next[y][e]);
#pragma unroll
                    for (int x = 0; x < KB; ++x) {
                        // (their weights stay in 32 bits, and have no scale)
                        const float t = s[x][y][e] - base;
                        l[y][e] += ex2(t);
                        s[x][y][e] = ex2(t + (UP - next[y][e]));
                        // a value that is not finite counts for all rows that see it: no weight of theirs is 0
                        if (wild && (seen >> (x * NB + y) * 2 + e & 1)) s[x][y][e] = fmaxf(s[x][y][e], 1.4e-45f);
                    }
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int y = 0; y < NB; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int x = 0; x < MO; ++x) {
                            o[x][y][e] *= f[y][e];
                            o[x][y][e + 2] *= f[y][e];
                        }
            }
            single = true;
            __syncwarp();
            if (gq == 0) {
#pragma unroll
                for (int y = 0; y < NB; ++y) *reinterpret_cast<float2*>(row_d + y * 8 + tq * 2) = make_float2(next[y][0], next[y][1]);
            }
            __syncwarp();
        }
        if (cached) {
#pragma unroll
            for (int x = 0; x < KB; ++x) {
                uint32_t p[NB][2];
#pragma unroll
                for (int y = 0; y < NB; ++y) {
                    p[y][0] = transpose8(Num<__half>::pack(s[x][y][0], s[x][y][1]));
                    p[y][1] = transpose8(Num<__half>::pack(s[x][y][2], s[x][y][3]));
                }
                constexpr int VW = D == 96 ? 1 : D == 64 ? 2 : 4;  // words of a load
#pragma unroll
                for (int i = 0; i < NW / VW; ++i) {
                    uint32_t w[4][VW];  // keys 2 tq, 2 tq + 1, 2 tq + 8, 2 tq + 9
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int row = x * 16 + (e >> 1) * 8 + tq * 2 + (e & 1);
                        const char* const v = slot + TK * D;
                        if constexpr (D == 96) {
                            w[e][0] = *reinterpret_cast<const uint32_t*>(v + row * D + i * 32 + gq * 4);
                        } else if constexpr (D == 64) {
                            const uint2 z = *reinterpret_cast<const uint2*>(v + L::value_at(row, gq >> 1) + (gq & 1) * 8);
                            w[e][0] = z.x, w[e][1] = z.y;
                        } else {
                            const uint4 z = *reinterpret_cast<const uint4*>(v + L::value_at(row, i * 8 + gq));
                            w[e][0] = z.x, w[e][1] = z.y, w[e][2] = z.z, w[e][3] = z.w;
                        }
                    }
#pragma unroll
                    for (int c = 0; c < VW; ++c) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            // channels 2 h, 2 h + 1 of the word, two keys side by side
                            const uint32_t u = __byte_perm(w[0][c], w[1][c], h ? 0x7362 : 0x5140),
                                           v = __byte_perm(w[2][c], w[3][c], h ? 0x7362 : 0x5140);
                            const uint32_t f[4] = {half2_lo(u), half2_hi(u), half2_lo(v), half2_hi(v)};
#pragma unroll
                            for (int y = 0; y < NB; ++y)
                                Num<__half>::mma(o[(i * VW + c) * 2 + h][y], f, p[y][0], p[y][1]);
                        }
                    }
                }
            }
        } else {
#pragma unroll
            for (int x = 0; x < KB; ++x) {
#pragma unroll 1
                for (int k = 0; k < min(8, C.T - first - x * 8); ++k) {
                    const char* const v = slot + TK * D + (x * 8 + k) * (D * 2);
                    float p[NB][2];
#pragma unroll
                    for (int y = 0; y < NB; ++y)
#pragma unroll
                        for (int e = 0; e < 2; ++e) p[y][e] = __shfl_sync(0xffffffffu, s[x][y][e], k * 4 + tq);
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        const uint2 z = *reinterpret_cast<const uint2*>(v + L::value_channel(w, gq) * 2);
                        const float2 z0 = Num<T>::unpack(z.x), z1 = Num<T>::unpack(z.y);
#pragma unroll
                        for (int y = 0; y < NB; ++y) {
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                if (p[y][e] != 0.0f) {
                                    o[2 * w][y][e] += p[y][e] * z0.x;
                                    o[2 * w][y][e + 2] += p[y][e] * z0.y;
                                    o[2 * w + 1][y][e] += p[y][e] * z1.x;
                                    o[2 * w + 1][y][e + 2] += p[y][e] * z1.y;
                                }
                            }
                        }
                    }
                }
            }
        }

        if (pend == 1) {
            if (lane == 0) p_before = arrive_at(a.arrived + P.first);
            pend = 2;
        }
        if (C.tile + 1 == C.c || j + 1 == n) {
            const bool whole = tile0 == 0 && C.tile + 1 == C.c;
            const int live = min(rows, RM);
            float* const part = part_of<D, RM>(a, me, tile0 == 0 ? 1 : 0);
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[y][e] += __shfl_xor_sync(0xffffffffu, l[y][e], x);
                    const float sum = l[y][e];
                    const float of_row = single ? row_d[y * 8 + tq * 2 + e] : d;
                    const float2 unit = unit_of(of_row);
                    const float small = unit.y * ex2(-UP);
                    const int rr = y * 8 + tq * 2 + e;
                    if (rr < live) {
                        if (!whole) {
                            float* const to = part + RM * 2 + rr * D;
#pragma unroll
                            for (int w = 0; w < NW; ++w)
                                *reinterpret_cast<float4*>(to + L::value_channel(w, gq)) =
                                    make_float4(o[2 * w][y][e] * small * unit.x, o[2 * w][y][e + 2] * small * unit.x,
                                                o[2 * w + 1][y][e] * small * unit.x, o[2 * w + 1][y][e + 2] * small * unit.x);
                            if (gq == 0) *reinterpret_cast<float2*>(part + rr * 2) = make_float2(M[y][e] - of_row, wild ? -sum : sum);
                        } else {
                            const int rho = C.rt * RM + rr, t = rho / G, head = C.h * G + rho - t * G;
                            const float inv = 1.0f / sum * small;
                            const auto of = [&](float x) { return sum == 0.0f ? 0.0f : x * inv * unit.x; };
                            char* const to = a.out + ((C.lo + t) * a.out_stride + (long long)head * D) * 2;
#pragma unroll
                            for (int w = 0; w < NW; ++w)
                                *reinterpret_cast<uint2*>(to + L::value_channel(w, gq) * 2) =
                                    make_uint2(Num<T>::pack(of(o[2 * w][y][e]), of(o[2 * w][y][e + 2])),
                                               Num<T>::pack(of(o[2 * w + 1][y][e]), of(o[2 * w + 1][y][e + 2])));
                            if (gq == 0 && a.lse) a.lse[(long long)(C.lo + t) * (H * G) + head] = (M[y][e] - of_row + log2f(sum)) * LN2;
                        }
                    }
                }
            }
            bool add = !whole;
#pragma unroll 1
            while (pend || add) {
                if (pend) {
                    const Pending p = P;
                    if (__shfl_sync(0xffffffffu, p_before, 0) == p.last - p.first) {
                        if (lane == 0) a.arrived[p.first] = 0;
                        asm volatile("fence.acq_rel.gpu;" ::: "memory");
                        join_rows8<T, D, RM>(a, p, min(p.T * G - p.rt * RM, RM), lane);
                    }
                    pend = 0;
                }
                if (!add) break;
                add = false;
                Pending p = {C.h, C.rt, C.lo, C.T, 0, 0};
                ax.sharers(C, p.first, p.last);
                __syncwarp();
                if (lane == 0) P = p;
                __syncwarp();
                pend = 1;
                if (j + 1 < n) break;
                if (lane == 0) p_before = arrive_at(a.arrived + P.first);
                pend = 2;
            }
            fresh = true;
        }
        if (j + 1 < n) advance8<TK, TN, RM>(a, ax, C);
        if (++b == S) b = 0;
    }
    cp_wait<0>();
}

template <typename T, int D, int NB>
cudaError_t launch_rows(const Attend8Args& a, int sms, cudaStream_t st)
{
    using L = Few8<D, NB>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024 && L::WARPS <= ATTEND_WORKERS_PER_SM, "what a CTA has");
    static_assert(L::WARPS * NB * 8 <= (D < 256 ? 256 : 128), "the partial results' room");
    cudaError_t e = allow_smem<k_attend8_few<T, D, NB>>(most);
    if (e != cudaSuccess) return e;
    k_attend8_few<T, D, NB><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch(const Attend8Args& a, int sms, cudaStream_t st)
{
    if constexpr (D < 256) {
        if ((long long)a.tok.n_tok * a.kv.group > 8ll * a.tok.n_req) return launch_rows<T, D, 2>(a, sms, st);
    }
    return launch_rows<T, D, 1>(a, sms, st);
}

template <typename T>
cudaError_t launch_dim(const Attend8Args& a, int dim, int sms, cudaStream_t st)
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

cudaError_t launch_attend8_few(const Attend8Args& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
