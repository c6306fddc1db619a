// aladdin_worker_accept: the kept tokens of a step enter the cache, and every
// cached token's accumulated weight grows by what the kept rows attended to it.
//
// Request r keeps the tokens acc[0 .. A) of its tree, a path from the root:
// token i takes slot len + i. With weights, slot c of key head h gains
//     sum_{i, g} e^(scale q_ig . k_c - lse_ig),   c <= len + i,
// over the kept tokens i and the group's query heads g: the softmax weights of
// the attention that lse came from, formed again from K alone (half of the
// bytes of the attention) for the rows that stayed, which the attention could
// not know. What counts is bytes in flight, as in the attention of few rows
// (attend_few.cu), and the kernel is built the same way: every warp works alone on
// a range of the axis of all key tiles, copies a few tiles ahead and forms keys by
// rows products with 8 rows an operand; the queries of a unit (request, head) stay
// in registers, up to 8 NB rows, more are read again for every tile. A slot
// belongs to one tile, so each weight is read and written once, sums run in 32 bits
// in a fixed order, and the tile that holds a new slot writes its key, value, weight
// and position. The last CTA to finish advances the lengths.
#include "attend.cuh"

namespace aladdin {
namespace wk {
namespace {

template <int D, int NB>
struct Accept {
    static constexpr int TK = D == 256 || NB == 1 ? 16 : 32;  // keys of a tile
    static constexpr int KB = TK / 16;                   // blocks of 16 keys
    static constexpr int WARPS = NB == 1 && D < 256 ? 16 : 8;  // warps of a CTA, one CTA an SM
    static constexpr int S = D == 64 ? 5 : D == 96 ? 4 : 3;    // tiles of a warp
    static constexpr int PITCH = D * 2 + 16;             // (rows in different banks)
    static constexpr int TILE = TK * PITCH;
    static constexpr int w = WARPS * S * TILE;           // weights of the tiles' keys
    static constexpr int pages = w + WARPS * S * TK * 4; // their pages, 16 keys each
    static constexpr int scratch = (pages + WARPS * S * KB * 4 + 7) / 8 * 8;
    static constexpr int pre = scratch + 32 * 8;
    static constexpr int bytes(int n_req) { return pre + (n_req + 1) * 8; }
};
// Keys of a place in calls that give every warp few tiles, and what a unit costs beside
// its tiles, in keys.
constexpr int PLACE_KEYS = 64, UNIT_KEYS = 64;

struct Unit {
    int r, h, tile;
    int len, A, lo, a0;  // cached, kept; the request's first token and first entry of acc
    int t0, c;           // its first tile, the number of its tiles
};

template <int KT>
__device__ __forceinline__ void enter(const AcceptArgs& a, Unit& u, int r)
{
    u.r = r;
    u.lo = a.tok.off[r];
    u.a0 = a.acc_off ? a.acc_off[r] : u.lo;
    u.A = (a.acc_off ? a.acc_off[r + 1] : a.tok.off[r + 1]) - u.a0;
    u.len = a.kv.len[r];
    u.t0 = a.lse ? 0 : u.len / KT;
    u.c = (u.len + u.A + KT - 1) / KT - u.t0;
}

template <int KT>
__device__ __forceinline__ int locate(const AcceptArgs& a, const Axis& ax, Unit& u, int x)
{
    const int r = plan_find(ax.pre, a.tok.n_req, x);
    enter<KT>(a, u, r);
    const int n = ax.places(u.c), y = x - ax.pre[r];
    u.h = y / n;
    u.tile = ax.tile_at(y - u.h * n);
    return ax.tiles[r] + u.h * u.c + u.tile;
}

template <int KT>
__device__ __forceinline__ void advance(const AcceptArgs& a, Unit& u, const int* pre)
{
    if (++u.tile < u.c) return;
    u.tile = 0;
    if (++u.h < a.kv.kv_heads) return;
    u.h = 0;
    int r = u.r + 1;
    while (r < a.tok.n_req && pre[r + 1] == pre[r]) ++r;
    if (r < a.tok.n_req) enter<KT>(a, u, r);
}

// Index of the i-th kept token of a request among all tokens.
__device__ __forceinline__ int kept(const AcceptArgs& a, const Unit& u, int i)
{
    return u.lo + (a.acc_off ? a.acc[u.a0 + i] : i);
}

template <typename T, int D, int NB>
__global__ void __launch_bounds__(Accept<D, NB>::WARPS * 32, 1) k_accept(AcceptArgs a)
{
    using L = Accept<D, NB>;
    constexpr int TK = L::TK, KB = L::KB, S = L::S, NT = L::WARPS * 32, PITCH = L::PITCH, CH = D / 8, MO = D / 16;
    constexpr int ROWS = NB * 8;  // rows whose queries the registers hold
    extern __shared__ __align__(128) char sm[];
    int* const pre = reinterpret_cast<int*>(sm + L::pre);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.kv.group, H = a.kv.kv_heads;
    const bool weigh = a.lse != nullptr;

    // a request whose offsets, length, kept tokens or pages make no sense keeps
    // nothing and is recorded
    Axis ax;
    const bool work = plan<NT>(
        a.tok.n_req, ax, pre, pre + a.tok.n_req + 1, reinterpret_cast<long long*>(sm + L::scratch),
        (int)gridDim.x * L::WARPS, UNIT_KEYS / TK, PLACE_KEYS / TK, a.err, [&](int r, int& c) -> int {
            const int lo = a.tok.off[r], hi = a.tok.off[r + 1], len = a.kv.len[r];
            const int a0 = a.acc_off ? a.acc_off[r] : lo, a1 = a.acc_off ? a.acc_off[r + 1] : hi;
            bool ok = lo >= 0 && hi >= lo && hi <= a.tok.n_tok && hi - lo <= ALADDIN_TREE_MAX && len >= 0 &&
                      a0 >= 0 && a1 >= a0 && a1 <= a.n_acc && a1 - a0 <= ALADDIN_TREE_MAX &&
                      (long long)len + (a1 - a0) <= a.kv.cap;
            if (ok && a.acc_off)
                for (int i = a0; i < a1; ++i) ok = ok && (unsigned)a.acc[i] < (unsigned)(hi - lo);
            if (ok && a1 > a0)
                for (int p = len >> a.kv.page_shift; p <= (len + a1 - a0 - 1) >> a.kv.page_shift; ++p)
                    ok = ok && (unsigned)a.kv.table[(long long)r * a.kv.table_stride + p] < (unsigned)a.kv.pages;
            c = 0;
            if (!ok) {
                if (blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
                return 0;
            }
            if (a1 == a0) return 0;
            c = (len + a1 - a0 + TK - 1) / TK - (weigh ? 0 : len / TK);
            return H;
        });
    // neighbouring ranges lie on different SMs
    const int me = warp * gridDim.x + blockIdx.x;
    if (work && me < ax.workers) {
        Unit C, F;  // the tile computed, the tile fetched
        int n;
        {
            const int end = ax.begin(me + 1);
            const int t1 = end < ax.total ? locate<TK>(a, ax, C, end) : ax.tiles[a.tok.n_req];
            n = t1 - locate<TK>(a, ax, C, ax.begin(me));
        }
        F = C;
        char* const tiles = sm + warp * S * L::TILE;
        const uint32_t tiles0 = smem_addr(tiles);
        float* const ws = reinterpret_cast<float*>(sm + L::w) + warp * S * TK;
        int* const pgs = reinterpret_cast<int*>(sm + L::pages) + warp * S * KB;
        const int gq = lane >> 2, tq = lane & 3, id = lane >> 3, lr = lane & 7;

        int page[KB];  // the pages of the tile under F, as the table has them
        auto pages = [&]() {
#pragma unroll
            for (int g = 0; g < KB; ++g) {
                const int key = (F.t0 + F.tile) * TK + g * 16;
                page[g] = key < F.len + F.A
                              ? a.kv.table[(long long)F.r * a.kv.table_stride + (key >> a.kv.page_shift)]
                              : 0;
            }
        };
        if (n > 0) pages();
        // the tile under F into place b; then F goes on
        auto fetch = [&](int b, bool more) {
            const int key0 = (F.t0 + F.tile) * TK, own = F.len - key0, all = own + F.A;
            bool valid[KB];
#pragma unroll
            for (int g = 0; g < KB; ++g) {
                valid[g] = (unsigned)page[g] < (unsigned)a.kv.pages;
                if (!valid[g] && lane == 0) atomicOr(a.err, WORKER_BAD_INPUT);
                if (lane == 0) pgs[b * KB + g] = valid[g] ? page[g] : -1;
            }
            if (weigh) {
                const uint32_t kd = tiles0 + b * L::TILE;
                const long long head = (long long)F.h * a.kv.head_stride;
                if (own >= TK && 32 % CH == 0) {
                    constexpr int STEP = 32 / CH;
                    const int r0 = lane / CH, ch = lane % CH;
#pragma unroll
                    for (int g = 0; g < KB; ++g) {
                        const char* k = a.kv.k;
                        if (valid[g])
                            k += (page[g] * a.kv.page_stride + head +
                                  (((key0 + g * 16) & (a.kv.page - 1)) + r0) * a.kv.token_stride + ch * 8) * 2;
                        const long long step = valid[g] ? STEP * a.kv.token_stride * 2 : 0;
#pragma unroll
                        for (int i = 0; i < 16 / STEP; ++i) {
                            cp16(kd + (g * 16 + i * STEP + r0) * PITCH + ch * 16, k, valid[g]);
                            k += step;
                        }
                    }
                } else {
#pragma unroll 2
                    for (int i = 0; i < (TK * CH + 31) / 32; ++i) {
                        const int x = lane + i * 32, row = x / CH, ch = x - row * CH;
                        if ((TK * CH) % 32 && x >= TK * CH) break;
                        const char* k = a.kv.k;
                        bool ok = row < all;
                        if (row < own) {
                            int p = page[0];
                            ok = valid[0];
#pragma unroll
                            for (int g = 1; g < KB; ++g)
                                if (row >> 4 == g) p = page[g], ok = valid[g];
                            if (ok)
                                k += (p * a.kv.page_stride + head + ((key0 + row) & (a.kv.page - 1)) * a.kv.token_stride +
                                      ch * 8) * 2;
                        } else if (ok) {
                            k = a.tok.k + (kept(a, F, row - own) * a.tok.k_stride + F.h * D + ch * 8) * 2;
                        }
                        cp16(kd + row * PITCH + ch * 16, k, ok);
                    }
                }
#pragma unroll
                for (int i = 0; i < (TK + 31) / 32; ++i) {
                    const int row = lane + i * 32;
                    int p = page[0];
                    bool ok = valid[0];
#pragma unroll
                    for (int g = 1; g < KB; ++g)
                        if (row >> 4 == g) p = page[g], ok = valid[g];
                    ok = ok && row < own;
                    if (row < TK)
                        cp4(smem_addr(ws + b * TK + row),
                            a.kv.weight + (ok ? ((long long)p * H + F.h) * a.kv.page + ((key0 + row) & (a.kv.page - 1)) : 0),
                            ok);
                }
            }
            if (more) {
                advance<TK>(a, F, pre);
                pages();
            }
        };
#pragma unroll
        for (int j = 0; j < S - 1; ++j) {
            if (j < n) fetch(j, j + 1 < n);
            cp_commit();
        }

        // rows row0 .. of a unit: row gq of every block, channels 2 tq and 2 tq + 1 of every 8,
        // and the logarithms of the sums of rows 2 tq and 2 tq + 1
        uint32_t qf[MO][NB][2];
        float lse2[NB][2];
        auto queries = [&](const Unit& u, int row0) {
            const int R = u.A * G;
            // (no early end: all loads are on their way together)
            int tok[NB][3];
#pragma unroll
            for (int y = 0; y < NB; ++y)
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    const int row = row0 + y * 8 + (e < 2 ? tq * 2 + e : gq);
                    tok[y][e] = row < R ? kept(a, u, row / G) : -1;
                }
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                const int row = row0 + y * 8 + gq, t = tok[y][2];
                const uint32_t* p = reinterpret_cast<const uint32_t*>(
                    a.tok.q + ((t < 0 ? 0 : t) * a.tok.q_stride + (long long)(u.h * G + row % G) * D) * 2) + tq;
#pragma unroll
                for (int x = 0; x < MO; ++x) {
                    qf[x][y][0] = t >= 0 ? __ldg(p + x * 8) : 0u;
                    qf[x][y][1] = t >= 0 ? __ldg(p + x * 8 + 4) : 0u;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int rr = row0 + y * 8 + tq * 2 + e;
                    // (rows that are none, and rows without an attention, add nothing)
                    lse2[y][e] = tok[y][e] >= 0 ? a.lse[(long long)tok[y][e] * (H * G) + u.h * G + rr % G] : -INFINITY;
                }
            }
#pragma unroll
            for (int y = 0; y < NB; ++y)
#pragma unroll
                for (int e = 0; e < 2; ++e) lse2[y][e] = lse2[y][e] == -INFINITY ? INFINITY : lse2[y][e] * LOG2E;
        };
        bool fresh = true;
        int b = 0;
        for (int j = 0; j < n; ++j) {
            __syncwarp();
            if (j + S - 1 < n) fetch(b == 0 ? S - 1 : b - 1, j + S < n);
            cp_commit();
            const int key0 = (C.t0 + C.tile) * TK, new0 = C.len - key0, R = C.A * G;
            if (weigh && fresh && R <= ROWS) queries(C, 0);
            fresh = false;
            cp_wait<S - 1>();
            __syncwarp();
            // new slots of this tile: keys, values, positions
            if (new0 < TK) {
                const int s0 = max(new0, 0), s1 = min(new0 + C.A, TK);
                for (int x = lane; x < (s1 - s0) * CH; x += 32) {
                    const int row = s0 + x / CH, ch = x % CH, slot = key0 + row;
                    const int p = pgs[b * KB + (row >> 4)], at = slot & (a.kv.page - 1);
                    const long long t = kept(a, C, row - new0);
                    const long long d = (p * a.kv.page_stride + C.h * a.kv.head_stride + at * a.kv.token_stride + ch * 8) * 2;
                    *reinterpret_cast<uint4*>(a.kv.k + d) = *reinterpret_cast<const uint4*>(
                        a.tok.k + (t * a.tok.k_stride + C.h * D + ch * 8) * 2);
                    *reinterpret_cast<uint4*>(a.kv.v + d) = *reinterpret_cast<const uint4*>(
                        a.tok.v + (t * a.tok.v_stride + C.h * D + ch * 8) * 2);
                    if (ch == 0) {
                        const long long m = ((long long)p * H + C.h) * a.kv.page + at;
                        if (a.kv.pos) a.kv.pos[m] = (a.kv.next ? a.kv.next[C.r] : C.len) + row - new0;
                        if (a.kv.weight && !weigh) a.kv.weight[m] = 0.0f;
                    }
                }
            }
            if (weigh) {
                const uint32_t kd = tiles0 + b * L::TILE + ((id & 1) * 8 + lr) * PITCH + (id >> 1) * 16;
                float sum[KB][2];  // keys gq and gq + 8 of every 16
#pragma unroll
                for (int x = 0; x < KB; ++x) sum[x][0] = sum[x][1] = 0.0f;
                for (int row0 = 0; row0 < R; row0 += ROWS) {
                    if (R > ROWS) queries(C, row0);
#pragma unroll
                    for (int x = 0; x < KB; ++x) {
                        uint32_t f[MO][4];
#pragma unroll
                        for (int ks = 0; ks < MO; ++ks) ldmatrix4(f[ks], kd + x * 16 * PITCH + ks * 32);
// two blocks at a time: their products do not wait for one another
#pragma unroll
                        for (int y0 = 0; y0 < NB; y0 += 2) {
                            if (row0 + y0 * 8 >= R) break;
                            constexpr int P = NB > 1 ? 2 : 1;
                            float s[P][4];
#pragma unroll
                            for (int y = 0; y < P; ++y) s[y][0] = s[y][1] = s[y][2] = s[y][3] = 0.0f;
#pragma unroll
                            for (int ks = 0; ks < MO; ++ks)
#pragma unroll
                                for (int y = 0; y < P; ++y)
                                    Num<T>::mma(s[y], f[ks], qf[ks][y0 + y][0], qf[ks][y0 + y][1]);
#pragma unroll
                            for (int y = 0; y < P; ++y) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float v = ex2(fmaf(s[y][e], a.scale_log2, -lse2[y0 + y][e & 1]));
                                    // row i sees the slots up to its own
                                    const int rr = row0 + (y0 + y) * 8 + tq * 2 + (e & 1);
                                    bool sees = rr < R;
                                    if (new0 < TK) sees = sees && x * 16 + (e >> 1) * 8 + gq - new0 <= rr / G;
                                    sum[x][e >> 1] += sees ? v : 0.0f;
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int x = 0; x < KB; ++x) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = sum[x][e];
                        v += __shfl_xor_sync(0xffffffffu, v, 1);
                        v += __shfl_xor_sync(0xffffffffu, v, 2);
                        const int row = x * 16 + e * 8 + gq, p = pgs[b * KB + x];
                        if (tq == 0 && row < new0 + C.A && p >= 0)
                            a.kv.weight[((long long)p * H + C.h) * a.kv.page + ((key0 + row) & (a.kv.page - 1))] =
                                ws[b * TK + row] + v;
                    }
                }
            }
            fresh = C.tile + 1 == C.c;
            if (j + 1 < n) advance<TK>(a, C, pre);
            if (++b == S) b = 0;
        }
        cp_wait<0>();
    }

    // every CTA has read the lengths: the last one to come here advances them
    __syncthreads();
    int* const last = reinterpret_cast<int*>(sm + L::scratch);
    if (tid == 0) {
        __threadfence();
        *last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (*last) {
        if (tid == 0) *a.arrived = 0;
        if (!work) return;
        for (int r = tid; r < a.tok.n_req; r += NT) {
            if (pre[r + 1] == pre[r]) continue;
            const int A = a.acc_off ? a.acc_off[r + 1] - a.acc_off[r] : a.tok.off[r + 1] - a.tok.off[r];
            a.kv.len[r] += A;
            if (a.kv.next) a.kv.next[r] += A;
        }
    }
}

template <typename T, int D, int NB>
cudaError_t launch_rows(const AcceptArgs& a, int sms, cudaStream_t st)
{
    using L = Accept<D, NB>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_accept<T, D, NB>>(most);
    if (e != cudaSuccess) return e;
    k_accept<T, D, NB><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
}

// 8 rows in registers where the mean rows of a request's key head fit them, else as many
// as the registers hold.
template <typename T, int D>
cudaError_t launch(const AcceptArgs& a, int sms, cudaStream_t st)
{
    if ((long long)a.n_acc * a.kv.group <= 8ll * a.tok.n_req) return launch_rows<T, D, 1>(a, sms, st);
    return launch_rows<T, D, D == 256 ? 2 : D == 64 ? 8 : 6>(a, sms, st);
}

template <typename T>
cudaError_t launch_dim(const AcceptArgs& a, int dim, int sms, cudaStream_t st)
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

cudaError_t launch_accept(const AcceptArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
