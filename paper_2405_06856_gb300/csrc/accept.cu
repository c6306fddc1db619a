// aladdin_worker_accept: the kept tokens of a step enter the cache, and every
// cached token's accumulated weight grows by what the kept rows attended to it.
//
// Request r keeps the tokens acc[0 .. A) of its tree, a path from the root:
// token i takes slot len + i. With weights, slot c of key head h gains
//     sum_{i, g} e^(scale q_ig . k_c - lse_ig),   c <= len + i,
// over the kept tokens i and the group's query heads g: the softmax weights of
// the attention that lse came from, formed again from K alone (half of the
// bytes of the attention) for the rows that stayed, which the attention could
// not know. The tiles of all (request, head) pairs lie on one axis that the
// CTAs share evenly. A slot belongs to one tile, so each weight is read and
// written once, sums run in 32 bits in a fixed order, and the tile that holds
// a new slot writes its key, value, weight and position. The last CTA to
// finish advances the lengths.
#include "worker_dev.cuh"

namespace aladdin {
namespace wk {
namespace {

// Keys of a tile, threads, rows that are staged at a time where a unit has more than 16.
constexpr int KT = 64, NT = 128, QR = 64;

struct Cursor {
    int r, h, tile;
    int len, A, lo, a0;  // cached, kept; the request's first token and first entry of acc
    int t0, c;           // first tile and number of tiles
};

__device__ __forceinline__ void enter(const AcceptArgs& a, Cursor& u, int r)
{
    u.r = r;
    u.lo = a.tok.off[r];
    u.a0 = a.acc_off ? a.acc_off[r] : u.lo;
    u.A = (a.acc_off ? a.acc_off[r + 1] : a.tok.off[r + 1]) - u.a0;
    u.len = a.kv.len[r];
    u.t0 = a.lse ? 0 : u.len / KT;
    u.c = (u.len + u.A + KT - 1) / KT - u.t0;
}

__device__ __forceinline__ void locate(const AcceptArgs& a, Cursor& u, const int* pre, int x)
{
    enter(a, u, plan_find(pre, a.tok.n_req, x));
    const int y = x - pre[u.r];
    u.h = y / u.c;
    u.tile = y - u.h * u.c;
}

__device__ __forceinline__ void advance(const AcceptArgs& a, Cursor& u, const int* pre)
{
    if (++u.tile < u.c) return;
    u.tile = 0;
    if (++u.h < a.kv.kv_heads) return;
    u.h = 0;
    int r = u.r + 1;
    while (r < a.tok.n_req && pre[r + 1] == pre[r]) ++r;
    if (r < a.tok.n_req) enter(a, u, r);
}

// Index of the i-th kept token of a request among all tokens.
__device__ __forceinline__ int kept(const AcceptArgs& a, const Cursor& u, int i)
{
    return a.acc_off ? u.lo + a.acc[u.a0 + i] : u.lo + i;
}

template <int D>
struct Smem {
    static constexpr int S = D == 256 ? 3 : 4;           // tiles in flight
    static constexpr int TILE = tile_bytes<D>(KT);
    static constexpr int PG = KT / 16;
    static constexpr int QT = tile_bytes<D>(16);
    static constexpr int k = 0;                          // S K tiles
    static constexpr int few = k + S * TILE;             // S x 16 rows, fetched with a unit's first tile
    static constexpr int q = few + S * QT;               // QR rows
    static constexpr int w = q + tile_bytes<D>(QR);      // S x KT weights
    static constexpr int lse = w + S * KT * 4;           // S x 16, then QR
    static constexpr int scratch = lse + (S * 16 + QR) * 4;  // 32 long longs
    static constexpr int ring = scratch + 32 * 8;        // (S + 1) x PG pages
    static constexpr int pre = ring + (S + 1) * PG * 4;
    static constexpr int bytes(int n_req) { return pre + (n_req + 1) * 4; }
};

template <typename T, int D>
__global__ void __launch_bounds__(NT, D == 256 ? 1 : 2) k_accept(AcceptArgs a)
{
    using L = Smem<D>;
    constexpr int S = L::S, CH = D / 8, PG = L::PG, KW = KT / 4, NS = KW / 8;
    extern __shared__ __align__(128) char sm[];
    const uint32_t sm0 = smem_addr(sm);
    int* const pre = reinterpret_cast<int*>(sm + L::pre);
    int* const ring = reinterpret_cast<int*>(sm + L::ring);
    float* const lses = reinterpret_cast<float*>(sm + L::lse);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.kv.group, H = a.kv.kv_heads;
    const bool weigh = a.lse != nullptr;

    // a request whose offsets, length, kept tokens or pages make no sense keeps
    // nothing and is recorded
    const int total = plan_prefix<NT>(
        a.tok.n_req, pre, reinterpret_cast<long long*>(sm + L::scratch), [&](int r) -> long long {
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
            if (!ok) {
                if (blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
                return 0;
            }
            if (a1 == a0) return 0;
            const int t0 = weigh ? 0 : len / KT;
            return (long long)H * ((len + a1 - a0 + KT - 1) / KT - t0);
        });
    if (total <= 0) {
        if (total < 0 && blockIdx.x == 0 && tid == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        return;
    }
    const int begin = (int)((long long)total * blockIdx.x / gridDim.x),
              end = (int)((long long)total * (blockIdx.x + 1) / gridDim.x), n = end - begin;

    auto page_at = [&](const Cursor& u, int g) -> int {
        const int key = (u.t0 + u.tile) * KT + g * 16;
        if (key >= u.len + u.A) return -1;
        const int p = a.kv.table[(long long)u.r * a.kv.table_stride + (key >> a.kv.page_shift)];
        if ((unsigned)p >= (unsigned)a.kv.pages) {
            atomicOr(a.err, WORKER_BAD_INPUT);
            return -1;
        }
        return p;
    };
    if (n > 0) {
        if (tid < (S - 1) * PG && tid / PG < n) {
            Cursor u;
            locate(a, u, pre, begin + tid / PG);
            ring[tid] = page_at(u, tid % PG);
        }
        int page_next = -1;
        if (tid < PG && S - 1 < n) {
            Cursor u;
            locate(a, u, pre, begin + S - 1);
            page_next = page_at(u, tid);
        }
        Cursor C, F;
        locate(a, C, pre, begin);
        F = C;
        __syncthreads();

        int fu = -1;  // ordinal of the unit fetched
        auto fetch = [&](int j) {
            if (!weigh) return;  // the cached keys are not needed
            const int b = j % S, key0 = (F.t0 + F.tile) * KT;
            const uint32_t kd = sm0 + L::k + b * L::TILE;
            const int* pg = ring + (j % (S + 1)) * PG;
            const long long head = (long long)F.h * a.kv.head_stride;
            if (j == 0 || F.tile == 0) {
                ++fu;
                const int R = F.A * G;
                if (R <= 16) {
#pragma unroll
                    for (int i = 0; i < (16 * CH + NT - 1) / NT; ++i) {
                        const int x = tid + i * NT, row = x / CH, ch = x - row * CH;
                        if ((16 * CH) % NT && x >= 16 * CH) break;
                        const bool ok = row < R;
                        const int t = ok ? row / G : 0, g = ok ? row - t * G : 0;
                        cp16(sm0 + L::few + (fu % S) * L::QT + tile_at<D>(row, ch),
                             a.tok.q + (kept(a, F, t) * a.tok.q_stride + (long long)(F.h * G + g) * D + ch * 8) * 2,
                             ok);
                    }
                    if (tid < R) {
                        const int t = tid / G, g = tid - t * G;
                        cp4(sm0 + L::lse + ((fu % S) * 16 + tid) * 4,
                            a.lse + (long long)kept(a, F, t) * (H * G) + F.h * G + g, true);
                    }
                }
            }
            if (NT % CH == 0 && key0 + KT <= F.len) {
                // cached keys only: a thread copies one chunk of every NT / CH-th row
                constexpr int STEP = NT / CH;
                const int ch = tid % CH, r0 = tid / CH;
                long long e[KT / 16];
#pragma unroll
                for (int g = 0; g < KT / 16; ++g) {
                    const int at = (key0 + g * 16) & (a.kv.page - 1);
                    e[g] = pg[g] * a.kv.page_stride + head + (at + r0 % 16) * a.kv.token_stride + ch * 8;
                }
#pragma unroll
                for (int i = 0; i < KT / STEP; ++i) {
                    const bool ok = pg[i * STEP / 16] >= 0;
                    const long long x = ok ? (e[i * STEP / 16] + (i * STEP % 16) * a.kv.token_stride) * 2 : 0;
                    cp16(kd + tile_at<D>(r0 + i * STEP, ch), a.kv.k + x, ok);
                }
            } else {
#pragma unroll
                for (int i = 0; i < (KT * CH + NT - 1) / NT; ++i) {
                    const int x = tid + i * NT, row = x / CH, ch = x - row * CH, key = key0 + row;
                    if ((KT * CH) % NT && x >= KT * CH) break;
                    const char* src = a.kv.k;
                    bool ok = key < F.len + F.A;
                    if (key < F.len) {
                        const int p = pg[row >> 4];
                        ok = p >= 0;
                        if (ok)
                            src += (p * a.kv.page_stride + head + (key & (a.kv.page - 1)) * a.kv.token_stride +
                                    ch * 8) * 2;
                    } else if (ok) {
                        src = a.tok.k + (kept(a, F, key - F.len) * a.tok.k_stride + F.h * D + ch * 8) * 2;
                    }
                    cp16(kd + tile_at<D>(row, ch), src, ok);
                }
            }
            if (tid < KT) {
                const int key = key0 + tid, p = pg[tid >> 4];
                const bool ok = key < F.len && p >= 0;
                cp4(sm0 + L::w + (b * KT + tid) * 4,
                    a.kv.weight + (ok ? ((long long)p * H + F.h) * a.kv.page + (key & (a.kv.page - 1)) : 0), ok);
            }
        };
#pragma unroll
        for (int j = 0; j < S - 1; ++j) {
            if (j < n) {
                fetch(j);
                advance(a, F, pre);
            }
            cp_commit();
        }
        bool fresh = true;
        int cu = -1;  // ordinal of the unit weighed
        for (int j = 0; j < n; ++j) {
            cp_wait<S - 2>();
            if (tid < PG) ring[((j + S - 1) % (S + 1)) * PG + tid] = page_next;
            __syncthreads();
            if (j + S - 1 < n) {
                fetch(j + S - 1);
                if (j + S < n) {
                    advance(a, F, pre);
                    if (tid < PG) page_next = page_at(F, tid);
                }
            }
            cp_commit();

            const int key0 = (C.t0 + C.tile) * KT;
            const int* pg = ring + (j % (S + 1)) * PG;
            // new slots of this tile: keys, values and positions
            if (key0 + KT > C.len) {
                const int s0 = C.len > key0 ? C.len : key0,
                          s1 = C.len + C.A < key0 + KT ? C.len + C.A : key0 + KT;
                for (int x = tid; x < (s1 - s0) * CH; x += NT) {
                    const int i = x / CH, ch = x - i * CH, slot = s0 + i;
                    const int p = pg[(slot - key0) >> 4], at = slot & (a.kv.page - 1);
                    const long long t = kept(a, C, slot - C.len);
                    const long long d = p * a.kv.page_stride + C.h * a.kv.head_stride +
                                        at * a.kv.token_stride + ch * 8;
                    *reinterpret_cast<uint4*>(a.kv.k + d * 2) = *reinterpret_cast<const uint4*>(
                        a.tok.k + (t * a.tok.k_stride + C.h * D + ch * 8) * 2);
                    *reinterpret_cast<uint4*>(a.kv.v + d * 2) = *reinterpret_cast<const uint4*>(
                        a.tok.v + (t * a.tok.v_stride + C.h * D + ch * 8) * 2);
                    if (ch == 0) {
                        const long long m = ((long long)p * H + C.h) * a.kv.page + at;
                        if (a.kv.pos) a.kv.pos[m] = (a.kv.next ? a.kv.next[C.r] : C.len) + slot - C.len;
                        if (a.kv.weight && !weigh) a.kv.weight[m] = 0.0f;
                    }
                }
            }
            if (weigh) {
                const int R = C.A * G, b = j % S, k0 = warp * KW;
                const uint32_t kd = sm0 + L::k + b * L::TILE;
                const int id = lane >> 3, lr = lane & 7, gq = lane >> 2, tq = lane & 3;
                float sum[NS][2];
#pragma unroll
                for (int x = 0; x < NS; ++x) sum[x][0] = sum[x][1] = 0.0f;
                if (fresh) ++cu;
                const bool few = R <= 16;  // the rows came with the unit's first tile
                const uint32_t qs = sm0 + (few ? L::few + (cu % S) * L::QT : L::q);
                float* const ls = lses + (few ? (cu % S) * 16 : S * 16);
                for (int r0 = 0; r0 < R; r0 += QR) {
                    const int rows = R - r0 < QR ? R - r0 : QR;
                    if (!few && (fresh || R > QR)) {  // these rows are not staged yet
                        if (r0) __syncthreads();
                        for (int x = tid; x < QR * CH; x += NT) {
                            const int rr = x / CH, ch = x - rr * CH;
                            uint4 v = make_uint4(0, 0, 0, 0);
                            if (rr < rows) {
                                const int i = (r0 + rr) / G, g = r0 + rr - i * G;
                                v = *reinterpret_cast<const uint4*>(
                                    a.tok.q + (kept(a, C, i) * a.tok.q_stride +
                                               (long long)(C.h * G + g) * D + ch * 8) * 2);
                            }
                            *reinterpret_cast<uint4*>(sm + L::q + tile_at<D>(rr, ch)) = v;
                        }
                        if (tid < rows) {
                            const int i = (r0 + tid) / G, g = r0 + tid - i * G;
                            ls[tid] = a.lse[(long long)kept(a, C, i) * (H * G) + C.h * G + g];
                        }
                        __syncthreads();
                    }
                    for (int m0 = 0; m0 < rows; m0 += 16) {
                        float s[NS][4];
#pragma unroll
                        for (int x = 0; x < NS; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.0f;
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            uint32_t qf[4];
                            // a fragment's four parts: rows 0-7, rows 8-15, then the same 8 channels on
                            ldmatrix4(qf, qs + tile_at<D>(m0 + (id & 1) * 8 + lr, ks * 2 + (id >> 1)));
#pragma unroll
                            for (int x = 0; x < NS; x += 2) {
                                uint32_t f[4];
                                ldmatrix4(f, kd + tile_at<D>(k0 + x * 8 + (id >> 1) * 8 + lr, ks * 2 + (id & 1)));
                                Num<T>::mma(s[x], qf, f[0], f[1]);
                                Num<T>::mma(s[x + 1], qf, f[2], f[3]);
                            }
                        }
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const int rr = m0 + gq + y * 8;
                            // (a row without an attention, lse = -inf, has no weights to add)
                            const float lse = rr < rows ? ls[rr] : -INFINITY;
                            const float base = lse == -INFINITY ? INFINITY : lse * LOG2E;
                            const int sees = C.len + (r0 + rr) / G - key0;  // the last key that the row sees
#pragma unroll
                            for (int x = 0; x < NS; ++x) {
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    const float p = ex2(fmaf(s[x][y * 2 + e], a.scale_log2, -base));
                                    if (rr < rows && k0 + x * 8 + tq * 2 + e <= sees) sum[x][e] += p;
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int x = 0; x < NS; ++x) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = sum[x][e];
                        v += __shfl_xor_sync(0xffffffffu, v, 4);
                        v += __shfl_xor_sync(0xffffffffu, v, 8);
                        v += __shfl_xor_sync(0xffffffffu, v, 16);
                        const int row = k0 + x * 8 + tq * 2 + e, key = key0 + row, p = pg[row >> 4];
                        if (gq == x && key < C.len + C.A && p >= 0)
                            a.kv.weight[((long long)p * H + C.h) * a.kv.page + (key & (a.kv.page - 1))] =
                                reinterpret_cast<const float*>(sm + L::w)[b * KT + row] + v;
                    }
                }
            }
            fresh = C.tile + 1 == C.c;
            if (j + 1 < n) advance(a, C, pre);
        }
        cp_wait<0>();
    }

    // every CTA has read the lengths: the last one to come here advances them
    __shared__ int s_last;
    __threadfence();
    __syncthreads();
    if (tid == 0) s_last = atomicAdd(a.arrived, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (s_last) {
        if (tid == 0) *a.arrived = 0;
        for (int r = tid; r < a.tok.n_req; r += NT) {
            if (pre[r + 1] == pre[r]) continue;
            const int A = a.acc_off ? a.acc_off[r + 1] - a.acc_off[r] : a.tok.off[r + 1] - a.tok.off[r];
            a.kv.len[r] += A;
            if (a.kv.next) a.kv.next[r] += A;
        }
    }
}

template <typename T, int D>
cudaError_t launch(const AcceptArgs& a, int sms, cudaStream_t st)
{
    using L = Smem<D>;
    static_assert(L::bytes(ALADDIN_WORKER_MAX_REQUESTS) <= 227 * 1024 - 256, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_accept<T, D>>(L::bytes(ALADDIN_WORKER_MAX_REQUESTS));
    if (e != cudaSuccess) return e;
    const long long tiles = (long long)a.tok.n_req * a.kv.kv_heads * (a.lse ? a.kv.cap / KT + 2 : 2);
    const long long most = 2ll * sms;
    k_accept<T, D><<<(int)(tiles < most ? tiles : most), NT, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
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
