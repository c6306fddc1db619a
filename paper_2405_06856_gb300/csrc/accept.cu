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
// rows products with 8 rows an operand. The queries of a unit (request, head) stay
// in registers where they are 8 rows, else in shared memory, in a rolled loop (with
// 48 rows in registers the unrolled code did not fit the instruction cache: 89 us
// for 24 requests' trees instead of 72); more rows are read again for every tile. A slot
// belongs to one tile, so each weight is read and written once, sums run in 32 bits
// in a fixed order, and the tile that holds a new slot writes its key, value, weight
// and position. The last CTA to finish advances the lengths.
//
// Measured: one token each of 128 requests, 83,336 cached tokens, 8 key heads of 128: 46 us, 3.9
// TB/s of keys and weights.
#include "attend.cuh"

namespace aladdin {
namespace wk {
namespace {

// FEW: a unit has 8 rows.
template <int D, bool FEW>
struct Accept {
    static constexpr int TK = 16;                        // keys of a tile
    static constexpr int WARPS = FEW && D < 256 ? 16 : 8;  // warps of a CTA, one CTA an SM
    static constexpr int S = D == 64 ? 5 : D == 96 ? 4 : D == 256 && !FEW ? 2 : 3;  // tiles of a warp
    static constexpr int ROWS = FEW ? 8 : D == 256 ? 16 : D == 128 ? 48 : 64;  // rows that are held
    static constexpr int PITCH = D * 2 + 16;             // (rows in different banks)
    static constexpr int TILE = TK * PITCH;
    static constexpr int q = WARPS * S * TILE;           // the warps' rows
    static constexpr int lse = q + (FEW ? 0 : WARPS * ROWS * PITCH);
    static constexpr int w = lse + (FEW ? 0 : WARPS * ROWS * 4);  // weights of the tiles' keys
    static constexpr int pages = w + WARPS * S * TK * 4; // their pages
    static constexpr int scratch = (pages + WARPS * S * 4 + 7) / 8 * 8;
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

template <typename T, int D, bool FEW>
__global__ void __launch_bounds__(Accept<D, FEW>::WARPS * 32, 1) k_accept(AcceptArgs a)
{
    using L = Accept<D, FEW>;
    constexpr int TK = L::TK, S = L::S, NT = L::WARPS * 32, PITCH = L::PITCH, CH = D / 8, MO = D / 16;
    constexpr int ROWS = L::ROWS;
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
        int* const pgs = reinterpret_cast<int*>(sm + L::pages) + warp * S;
        const int gq = lane >> 2, tq = lane & 3, id = lane >> 3, lr = lane & 7;

        int page = 0;  // the page of the tile under F, as the table has it
        auto pages = [&]() {
            const int key = (F.t0 + F.tile) * TK;
            page = a.kv.table[(long long)F.r * a.kv.table_stride + (key >> a.kv.page_shift)];
        };
        if (n > 0) pages();
        // the tile under F into place b; then F goes on
        auto fetch = [&](int b, bool more) {
            const int key0 = (F.t0 + F.tile) * TK, own = F.len - key0, all = own + F.A;
            const bool valid = (unsigned)page < (unsigned)a.kv.pages;
            if (lane == 0) {
                if (!valid) atomicOr(a.err, WORKER_BAD_INPUT);
                pgs[b] = valid ? page : -1;
            }
            if (weigh) {
                const uint32_t kd = tiles0 + b * L::TILE;
                const long long from = page * a.kv.page_stride + (long long)F.h * a.kv.head_stride +
                                       (key0 & (a.kv.page - 1)) * a.kv.token_stride;
                if (own >= TK && 32 % CH == 0) {
                    constexpr int STEP = 32 / CH;
                    const int r0 = lane / CH, ch = lane % CH;
                    const char* k = a.kv.k + (valid ? (from + r0 * a.kv.token_stride + ch * 8) * 2 : 0);
                    const long long step = valid ? STEP * a.kv.token_stride * 2 : 0;
#pragma unroll
                    for (int i = 0; i < TK / STEP; ++i) {
                        cp16(kd + (i * STEP + r0) * PITCH + ch * 16, k, valid);
                        k += step;
                    }
                } else {
#pragma unroll 2
                    for (int i = 0; i < (TK * CH + 31) / 32; ++i) {
                        const int x = lane + i * 32, row = x / CH, ch = x - row * CH;
                        if ((TK * CH) % 32 && x >= TK * CH) break;
                        const char* k = a.kv.k;
                        bool ok = row < all;
                        if (row < own) {
                            ok = valid;
                            if (ok) k += (from + row * a.kv.token_stride + ch * 8) * 2;
                        } else if (ok) {
                            k = a.tok.k + (kept(a, F, row - own) * a.tok.k_stride + F.h * D + ch * 8) * 2;
                        }
                        cp16(kd + row * PITCH + ch * 16, k, ok);
                    }
                }
                if (lane < TK) {
                    const bool ok = valid && lane < own;
                    cp4(smem_addr(ws + b * TK + lane),
                        a.kv.weight + (ok ? ((long long)page * H + F.h) * a.kv.page + ((key0 + lane) & (a.kv.page - 1)) : 0),
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

        // rows row0 .. of a unit: in registers row gq, channels 2 tq and 2 tq + 1 of every 8, and
        // the logarithms of the sums of rows 2 tq and 2 tq + 1, or in this warp's shared memory
        uint32_t qf[FEW ? MO : 1][2];
        float lse2[2];
        char* const qs = sm + L::q + warp * ROWS * PITCH;
        float* const ls = reinterpret_cast<float*>(sm + L::lse) + warp * ROWS;
        // (rows that are none, and rows without an attention, add nothing)
        auto log_sum = [](float s) { return s == -INFINITY ? INFINITY : s * LOG2E; };
        auto queries = [&](const Unit& u, int row0) {
            const int R = u.A * G;
            if constexpr (FEW) {
                int tok[3];
#pragma unroll
                for (int e = 0; e < 3; ++e) {
                    const int row = row0 + (e < 2 ? tq * 2 + e : gq);
                    tok[e] = row < R ? kept(a, u, row / G) : -1;
                }
                const bool ok = tok[2] >= 0;
                const uint32_t* p = reinterpret_cast<const uint32_t*>(
                    a.tok.q + ((ok ? tok[2] : 0) * a.tok.q_stride + (long long)(u.h * G + (row0 + gq) % G) * D) * 2) + tq;
#pragma unroll
                for (int x = 0; x < MO; ++x) {
                    qf[x][0] = ok ? __ldg(p + x * 8) : 0u;
                    qf[x][1] = ok ? __ldg(p + x * 8 + 4) : 0u;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    lse2[e] = tok[e] >= 0 ? a.lse[(long long)tok[e] * (H * G) + u.h * G + (row0 + tq * 2 + e) % G] : -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e) lse2[e] = log_sum(lse2[e]);
            } else {
                __syncwarp();
                const int rows = min(ROWS, R - row0), held = (rows + 15) / 16 * 16;
                const uint32_t qd = smem_addr(qs);
#pragma unroll 4
                for (int x = lane; x < held * CH; x += 32) {
                    const int row = x / CH, ch = x - row * CH;
                    const bool ok = row < rows;
                    const int i = ok ? (row0 + row) / G : 0, g = ok ? row0 + row - i * G : 0;
                    cp16(qd + row * PITCH + ch * 16,
                         a.tok.q + (kept(a, u, i) * a.tok.q_stride + (long long)(u.h * G + g) * D + ch * 8) * 2, ok);
                }
                for (int row = lane; row < held; row += 32) {
                    float s = -INFINITY;
                    if (row < rows) {
                        const int i = (row0 + row) / G;
                        s = a.lse[(long long)kept(a, u, i) * (H * G) + u.h * G + row0 + row - i * G];
                    }
                    ls[row] = log_sum(s);
                }
                cp_commit();
                cp_wait<0>();
                __syncwarp();
            }
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
                    const int p = pgs[b], at = slot & (a.kv.page - 1);
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
                uint32_t f[MO][4];
#pragma unroll
                for (int ks = 0; ks < MO; ++ks) ldmatrix4(f[ks], kd + ks * 32);
                float sum[2] = {0.0f, 0.0f};  // keys gq and gq + 8
                // scores of the keys by rows row, row + 1 (row = the first of a block + 2 tq) join the sums
                auto add = [&](const float(&s)[4], float ls0, float ls1, int row) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = ex2(fmaf(s[e], a.scale_log2, e & 1 ? -ls1 : -ls0));
                        const int rr = row + (e & 1);
                        bool sees = rr < R;  // (a row that is none may hold anything)
                        if (new0 < TK) sees = sees && (e >> 1) * 8 + gq - new0 <= rr / G;
                        sum[e >> 1] += sees ? v : 0.0f;
                    }
                };
                if constexpr (FEW) {
                    // (a kept token more than the mean may bring more than 8 rows: they are read again)
                    for (int row0 = 0; row0 < R; row0 += 8) {
                        if (R > 8) queries(C, row0);
                        float s[2][4] = {};
#pragma unroll
                        for (int ks = 0; ks < MO; ++ks) Num<T>::mma(s[ks & 1], f[ks], qf[ks][0], qf[ks][1]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[0][e] += s[1][e];
                        add(s[0], lse2[0], lse2[1], row0 + tq * 2);
                    }
                } else {
                    for (int row0 = 0; row0 < R; row0 += ROWS) {
                        if (R > ROWS) queries(C, row0);
                        const uint32_t qa = smem_addr(qs) + ((id >> 1) * 8 + lr) * PITCH + (id & 1) * 16;
                        // two blocks of 8 rows at a time: their products do not wait for one another
#pragma unroll 1
                        for (int y = 0; y < min(ROWS, R - row0); y += 16) {
                            float s[2][4] = {};
#pragma unroll
                            for (int ks = 0; ks < MO; ++ks) {
                                uint32_t q[4];
                                ldmatrix4(q, qa + y * PITCH + ks * 32);
                                Num<T>::mma(s[0], f[ks], q[0], q[1]);
                                Num<T>::mma(s[1], f[ks], q[2], q[3]);
                            }
                            const float2 l0 = *reinterpret_cast<const float2*>(ls + y + tq * 2),
                                         l1 = *reinterpret_cast<const float2*>(ls + y + 8 + tq * 2);
                            add(s[0], l0.x, l0.y, row0 + y + tq * 2);
                            add(s[1], l1.x, l1.y, row0 + y + 8 + tq * 2);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float v = sum[e];
                    v += __shfl_xor_sync(0xffffffffu, v, 1);
                    v += __shfl_xor_sync(0xffffffffu, v, 2);
                    const int row = e * 8 + gq, p = pgs[b];
                    if (tq == 0 && row < new0 + C.A && p >= 0)
                        a.kv.weight[((long long)p * H + C.h) * a.kv.page + ((key0 + row) & (a.kv.page - 1))] =
                            ws[b * TK + row] + v;
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

template <typename T, int D, bool FEW>
cudaError_t launch_rows(const AcceptArgs& a, int sms, cudaStream_t st)
{
    using L = Accept<D, FEW>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_accept<T, D, FEW>>(most);
    if (e != cudaSuccess) return e;
    k_accept<T, D, FEW><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
}

// 8 rows in registers where the mean rows of a request's key head fit them (64 requests of about 1,500
// tokens, 8 key heads of 128: 8 rows 59 us in registers and 66 in shared memory, 12 rows 92 and 68).
template <typename T, int D>
cudaError_t launch(const AcceptArgs& a, int sms, cudaStream_t st)
{
    if ((long long)a.n_acc * a.kv.group <= 8ll * a.tok.n_req) return launch_rows<T, D, true>(a, sms, st);
    return launch_rows<T, D, false>(a, sms, st);
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
