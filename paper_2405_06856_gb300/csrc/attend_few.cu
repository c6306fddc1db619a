// aladdin_worker_attend where the rows of a (request, key head) are few (at most
// 16 on average): decoding, and small trees of small groups. See attend.cu for
// the operator.
//
// Such a call reads every cached key and value once and computes next to nothing:
// what counts is bytes in flight and few instructions a byte. Every warp works
// alone: it owns a range of the axis of all key tiles and a few tiles of shared
// memory, which it fills by asynchronous copies a few tiles ahead, and waits for no
// other warp. The products are formed transposed, keys by rows and channels by
// rows, so that 8 rows (or 2 x 8) are a whole operand: 8 rows as the 16 of the
// other order would double products, registers and exponentials. The weights turn
// from one product's result into the other's operand in registers (an 8 x 8
// transposition). The next unit's queries are on their way while one is
// computed. A row of a tile is padded by 16 bytes, so that the matrix loads of
// eight rows meet different banks.
//
// A unit (request, head, row tile) that warps share is joined by the one that
// finishes last, in the order of its keys.
//
// Measured: 128 requests of 83,336 cached tokens, 32 query and 8 key heads of 128 channels in
// bf16: 74 us, 4.7 TB/s (warps of one CTA that shared tiles through barriers: 91 us; copies
// of a row each by the bulk engine: 95); two requests of 110,108 tokens, 32 heads of 64 in
// f16: 159 us, 5.7 TB/s of 6.8 that a copy reaches.
#include "attend.cuh"

namespace aladdin {
namespace wk {
namespace {

template <int D>
struct Few {
    static constexpr int TK = D == 64 ? 32 : 16;         // keys of a tile
    static constexpr int WARPS = D == 256 ? 4 : 8;       // warps of a CTA, one CTA an SM
    static constexpr int S = 3;                          // tiles of a warp
    static constexpr unsigned FULL = TK == 32 ? 0xffffffffu : 0xffffu;  // the mask of a tile of keys
    static constexpr int PITCH = D * 2 + 16;
    static constexpr int TILE = 2 * TK * PITCH;          // keys, then values
    static constexpr int oks = WARPS * S * TILE;         // masks of tiles
    static constexpr int scratch = (oks + WARPS * S * 4 + 7) / 8 * 8;
    static constexpr int pre = scratch + 32 * 8;
    static constexpr int bytes(int n_req) { return pre + (n_req + 1) * 8; }
};
// Keys of a place in calls that give every warp few tiles, and what a unit costs beside
// its tiles, in keys.
constexpr int PLACE_KEYS = 64, UNIT_KEYS = 32;

// NB: blocks of 8 rows.
template <typename T, int D, int NB>
__global__ void __launch_bounds__(Few<D>::WARPS * 32, 1) k_attend_few(AttendArgs a)
{
    constexpr int RM = NB * 8;
    using L = Few<D>;
    constexpr int TK = L::TK, S = L::S, NT = L::WARPS * 32, PITCH = L::PITCH;
    constexpr int KB = TK / 16, MO = D / 16, CH = D / 8, PG = TK / 16;  // blocks of 16 keys, of 16 channels
    extern __shared__ __align__(128) char sm[];
    int* const pre = reinterpret_cast<int*>(sm + L::pre);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.kv.group, H = a.kv.kv_heads;
    char* const tiles = sm + warp * S * L::TILE;
    const uint32_t tiles0 = smem_addr(tiles);
    unsigned* const oks = reinterpret_cast<unsigned*>(sm + L::oks) + warp * S;

    Axis ax;
    if (!plan<NT>(a.tok.n_req, ax, pre, pre + a.tok.n_req + 1, reinterpret_cast<long long*>(sm + L::scratch),
                  (int)gridDim.x * L::WARPS, UNIT_KEYS / TK, PLACE_KEYS / TK, a.err,
                  [&](int r, int& c) { return attend_units<TK, RM>(a, r, c); }))
        return;
    // neighbouring ranges lie on different SMs
    const int me = warp * gridDim.x + blockIdx.x;
    if (me >= ax.workers) return;
    Cursor C, F;  // the tile computed, the tile fetched
    const int n = range<TK, RM>(a, ax, C, me);
    F = C;
    // the pages of the tile under F, 16 keys each, as the table has them
    int page[PG];
    auto pages = [&]() {
#pragma unroll
        for (int g = 0; g < PG; ++g) {
            const int key = F.tile * TK + g * 16;
            page[g] = key < F.len ? a.kv.table[(long long)F.r * a.kv.table_stride + (key >> a.kv.page_shift)] : 0;
        }
    };
    pages();
    // the tile under F into place b; then F goes on
    auto fetch = [&](int b, bool more) {
        const int key0 = F.tile * TK, own = F.len - key0;  // cached keys from the tile's start
        const uint32_t kd = tiles0 + b * L::TILE, vd = kd + TK * PITCH;
        unsigned mask = 0;
#pragma unroll
        for (int g = 0; g < PG; ++g) {
            if ((unsigned)page[g] < (unsigned)a.kv.pages) mask |= 0xffffu << (g * 16);
            else if (lane == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        }
        const long long head = (long long)F.h * a.kv.head_stride;
        if (own >= TK && 32 % CH == 0) {
            // cached keys only: a lane copies one chunk of every 32 / CH-th row
            constexpr int STEP = 32 / CH;
            const int r0 = lane / CH, ch = lane % CH;
            const uint32_t d = r0 * PITCH + ch * 16;
#pragma unroll
            for (int g = 0; g < PG; ++g) {
                const bool ok = mask >> (g * 16) & 1;
                const long long e = ok ? (page[g] * a.kv.page_stride + head +
                                          (((key0 + g * 16) & (a.kv.page - 1)) + r0) * a.kv.token_stride + ch * 8) * 2
                                       : 0;
                const long long step = ok ? STEP * a.kv.token_stride * 2 : 0;
                const char *k = a.kv.k + e, *v = a.kv.v + e;
#pragma unroll
                for (int i = 0; i < 16 / STEP; ++i) {
                    cp16(kd + d + (g * 16 + i * STEP) * PITCH, k, ok);
                    cp16(vd + d + (g * 16 + i * STEP) * PITCH, v, ok);
                    k += step;
                    v += step;
                }
            }
        } else {
            const int all = own + F.T;  // keys from the tile's start
            const unsigned cached = own >= TK ? ~0u : own > 0 ? (1u << own) - 1 : 0u;
            mask = ((mask & cached) | ~cached) & (all >= TK ? L::FULL : (1u << all) - 1);
#pragma unroll 2
            for (int i = 0; i < (TK * CH + 31) / 32; ++i) {
                const int x = lane + i * 32, row = x / CH, ch = x - row * CH;
                if ((TK * CH) % 32 && x >= TK * CH) break;
                const char *k = a.kv.k, *v = a.kv.v;
                const bool ok = mask >> row & 1;
                if (ok && row < own) {
                    const int p = PG == 1 || row < 16 ? page[0] : page[PG - 1];
                    const long long e = (p * a.kv.page_stride + head +
                                         ((key0 + row) & (a.kv.page - 1)) * a.kv.token_stride + ch * 8) * 2;
                    k += e;
                    v += e;
                } else if (ok) {
                    const long long t = F.lo + row - own;
                    k = a.tok.k + (t * a.tok.k_stride + F.h * D + ch * 8) * 2;
                    v = a.tok.v + (t * a.tok.v_stride + F.h * D + ch * 8) * 2;
                }
                // (weights of 0 meet the values of rows that hold no key: zeros)
                cp16(kd + row * PITCH + ch * 16, k, ok);
                cp16(vd + row * PITCH + ch * 16, v, ok);
            }
        }
        if (lane == 0) oks[b] = mask;
        if (more) {
            advance<TK, RM>(a, F, pre);
            pages();
        }
    };
#pragma unroll
    for (int j = 0; j < S - 1; ++j) {
        if (j < n) fetch(j, j + 1 < n);
        cp_commit();
    }

    constexpr bool AHEAD = D < 256;  // (256 channels leave no registers for a second set of queries)
    const int gq = lane >> 2, tq = lane & 3, id = lane >> 3, lr = lane & 7;
    uint32_t qf[MO][NB][2], qn[AHEAD ? MO : 1][NB][2];
    // row gq of every block, channels 2 tq and 2 tq + 1 of every 8
    auto queries = [&](const Cursor& u, uint32_t (*q)[NB][2]) {
        const int rows = u.T * G - u.rt * RM;
#pragma unroll
        for (int y = 0; y < NB; ++y) {
            const int rho = u.rt * RM + y * 8 + gq;
            const bool ok = y * 8 + gq < rows;
            const int t = ok ? rho / G : 0;
            const uint32_t* p = reinterpret_cast<const uint32_t*>(
                a.tok.q + ((u.lo + t) * a.tok.q_stride + (long long)(u.h * G + (ok ? rho - t * G : 0)) * D) * 2) + tq;
#pragma unroll
            for (int x = 0; x < MO; ++x) {
                q[x][y][0] = ok ? __ldg(p + x * 8) : 0u;
                q[x][y][1] = ok ? __ldg(p + x * 8 + 4) : 0u;
            }
        }
    };
    if constexpr (AHEAD) queries(C, qn);

    float o[MO][NB][4], m[NB][2], l[NB][2];  // channels gq, gq + 8 of a block of rows 2 tq, 2 tq + 1
    unsigned long long see[NB][2];
    bool fresh = true;
    int b = 0, tile0 = 0;  // a tile's place; the first tile of the unit that this warp has

    for (int j = 0; j < n; ++j) {
        __syncwarp();
        if (j + S - 1 < n) fetch(b == 0 ? S - 1 : b - 1, j + S < n);
        cp_commit();
        const int rows = C.T * G - C.rt * RM;
        if (fresh) {
            fresh = false;
            tile0 = C.tile;
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int x = 0; x < MO; ++x) o[x][y][0] = o[x][y][1] = o[x][y][2] = o[x][y][3] = 0.0f;
                m[y][0] = m[y][1] = -INFINITY;
                l[y][0] = l[y][1] = 0.0f;
                see[y][0] = see[y][1] = 1;
            }
            if (C.T > 1) {
#pragma unroll
                for (int y = 0; y < NB; ++y)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int rr = y * 8 + tq * 2 + e;
                        see[y][e] = ancestors(a, C, rr < rows ? (C.rt * RM + rr) / G : 0);
                    }
            }
            if constexpr (AHEAD) {
#pragma unroll
                for (int x = 0; x < MO; ++x)
#pragma unroll
                    for (int y = 0; y < NB; ++y) {
                        qf[x][y][0] = qn[x][y][0];
                        qf[x][y][1] = qn[x][y][1];
                    }
                if (j + C.c - C.tile < n) {  // the range goes on behind this unit
                    Cursor u = C;
                    u.tile = u.c - 1;
                    advance<TK, RM>(a, u, pre);
                    queries(u, qn);
                }
            } else {
                queries(C, qf);
            }
        }
        cp_wait<S - 1>();
        __syncwarp();
        const uint32_t kd = tiles0 + b * L::TILE, vd = kd + TK * PITCH;
        const unsigned okm = oks[b];
        const int new0 = C.len - C.tile * TK;  // the first new key's place in the tile
        const bool mixed = new0 < TK;
        bool wild = false;
        if (mixed && C.T > 1) {
            // a value that is not finite would reach rows that do not see its token
            // (0 times infinity): such a tile is summed key by key below
            const int k1 = min(TK, new0 + C.T);
            for (int x = max(new0, 0) * CH + lane; x < k1 * CH; x += 32) {
                const int row = x / CH;
                const uint4 q = *reinterpret_cast<const uint4*>(tiles + b * L::TILE + (TK + row) * PITCH +
                                                                (x - row * CH) * 16);
                wild |= Num<T>::wild(q.x) || Num<T>::wild(q.y) || Num<T>::wild(q.z) || Num<T>::wild(q.w);
            }
            wild = __any_sync(0xffffffffu, wild);
        }

        float s[KB][NB][4];  // keys gq, gq + 8 of a block by rows 2 tq, 2 tq + 1
#pragma unroll
        for (int x = 0; x < KB; ++x)
#pragma unroll
            for (int y = 0; y < NB; ++y) s[x][y][0] = s[x][y][1] = s[x][y][2] = s[x][y][3] = 0.0f;
        {
            const uint32_t at = kd + ((id & 1) * 8 + lr) * PITCH + (id >> 1) * 16;
#pragma unroll
            for (int ks = 0; ks < MO; ++ks) {
#pragma unroll
                for (int x = 0; x < KB; ++x) {
                    uint32_t f[4];
                    ldmatrix4(f, at + x * 16 * PITCH + ks * 32);
#pragma unroll
                    for (int y = 0; y < NB; ++y) Num<T>::mma(s[x][y], f, qf[ks][y][0], qf[ks][y][1]);
                }
            }
        }
        if (mixed || okm != L::FULL) {
#pragma unroll
            for (int x = 0; x < KB; ++x) {
#pragma unroll
                for (int y = 0; y < NB; ++y) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = x * 16 + (e >> 1) * 8 + gq, u = k - new0;
                        const bool ok = u < 0 ? okm >> k & 1 : u < 64 && (see[y][e & 1] >> u & 1);
                        if (!ok) s[x][y][e] = -INFINITY;
                    }
                }
            }
        }
        float top[NB][2];
        bool higher = false;
#pragma unroll
        for (int y = 0; y < NB; ++y) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[y][e] = m[y][e];
#pragma unroll
                for (int x = 0; x < KB; ++x) {
                    s[x][y][e] *= a.scale_log2;
                    s[x][y][e + 2] *= a.scale_log2;
                    top[y][e] = fmaxf(top[y][e], fmaxf(s[x][y][e], s[x][y][e + 2]));
                }
                higher = higher || top[y][e] > m[y][e];
            }
        }
        if (__any_sync(0xffffffffu, higher)) {
#pragma unroll
            for (int y = 0; y < NB; ++y) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1)
                        top[y][e] = fmaxf(top[y][e], __shfl_xor_sync(0xffffffffu, top[y][e], x));
                    const float f = top[y][e] > m[y][e] ? ex2(m[y][e] - top[y][e]) : 1.0f;
                    m[y][e] = top[y][e];
                    l[y][e] *= f;
#pragma unroll
                    for (int x = 0; x < MO; ++x) {
                        o[x][y][e] *= f;
                        o[x][y][e + 2] *= f;
                    }
                }
            }
        }
        uint32_t p[KB][NB][2];
#pragma unroll
        for (int y = 0; y < NB; ++y) {
            const float base[2] = {m[y][0] == -INFINITY ? 0.0f : m[y][0], m[y][1] == -INFINITY ? 0.0f : m[y][1]};
#pragma unroll
            for (int x = 0; x < KB; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[x][y][e] = ex2(s[x][y][e] - base[e & 1]);
                    l[y][e & 1] += s[x][y][e];
                }
                p[x][y][0] = transpose8(Num<T>::pack(s[x][y][0], s[x][y][1]));
                p[x][y][1] = transpose8(Num<T>::pack(s[x][y][2], s[x][y][3]));
            }
        }
        if (!wild) {
            const uint32_t at = vd + ((id >> 1) * 8 + lr) * PITCH + (id & 1) * 16;
#pragma unroll
            for (int x = 0; x < KB; ++x) {
#pragma unroll
                for (int z = 0; z < MO; ++z) {
                    uint32_t f[4];
                    ldmatrix4t(f, at + x * 16 * PITCH + z * 32);
#pragma unroll
                    for (int y = 0; y < NB; ++y) Num<T>::mma(o[z][y], f, p[x][y][0], p[x][y][1]);
                }
            }
        } else {
#pragma unroll
            for (int x = 0; x < KB * 2; ++x) {
#pragma unroll 1
                for (int k = 0; k < 8; ++k) {
                    const char* row = tiles + b * L::TILE + (TK + x * 8 + k) * PITCH;
#pragma unroll
                    for (int y = 0; y < NB; ++y) {
                        float w[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            w[e] = __shfl_sync(0xffffffffu, s[x / 2][y][(x & 1) * 2 + e], k * 4 + tq);
#pragma unroll
                        for (int z = 0; z < MO; ++z) {
#pragma unroll
                            for (int c = 0; c < 2; ++c) {
                                const float v = Num<T>::unpack(*reinterpret_cast<const unsigned short*>(
                                    row + (z * 16 + c * 8 + gq) * 2)).x;
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    if (w[e] != 0.0f) o[z][y][c * 2 + e] += w[e] * v;
                            }
                        }
                    }
                }
            }
        }

        if (C.tile + 1 == C.c || j + 1 == n) {
            const bool whole = tile0 == 0 && C.tile + 1 == C.c;
            const int live = min(rows, RM);
            float* const part = part_of<D, RM>(a, me, tile0 == 0 ? 1 : 0);
#pragma unroll
            for (int y = 0; y < NB; ++y) {
                float inv[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int x = 4; x < 32; x <<= 1) l[y][e] += __shfl_xor_sync(0xffffffffu, l[y][e], x);
                    inv[e] = l[y][e] > 0.0f || l[y][e] != l[y][e] ? 1.0f / l[y][e] : 0.0f;
                    const int rr = y * 8 + tq * 2 + e;
                    if (rr < live) {
                        if (!whole) {
                            float* const d = part + RM * 2 + rr * D + gq;
#pragma unroll
                            for (int x = 0; x < MO; ++x) {
                                d[x * 16] = o[x][y][e];
                                d[x * 16 + 8] = o[x][y][e + 2];
                            }
                            if (gq == 0) *reinterpret_cast<float2*>(part + rr * 2) = make_float2(m[y][e], l[y][e]);
                        } else if (gq == 0 && a.lse) {
                            const int rho = C.rt * RM + rr, t = rho / G;
                            a.lse[(long long)(C.lo + t) * (H * G) + C.h * G + rho - t * G] =
                                (m[y][e] + log2f(l[y][e])) * LN2;
                        }
                    }
                }
                if (whole) {
                    // turned, lane 4 g + t holds channels 2 t and 2 t + 1 of row g
                    const int rr = y * 8 + gq, rho = C.rt * RM + rr, t = rho / G;
                    char* const d = a.out + ((C.lo + t) * a.out_stride +
                                             (long long)(C.h * G + rho - t * G) * D + tq * 2) * 2;
#pragma unroll
                    for (int x = 0; x < MO; ++x) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const uint32_t v =
                                transpose8(Num<T>::pack(o[x][y][c * 2] * inv[0], o[x][y][c * 2 + 1] * inv[1]));
                            if (rr < live) *reinterpret_cast<uint32_t*>(d + x * 32 + c * 16) = v;
                        }
                    }
                }
            }
            if (!whole) {
                int first, last;
                ax.sharers(C, first, last);
                __threadfence();
                __syncwarp();
                int arrived = 0;
                if (lane == 0) arrived = atomicAdd(a.arrived + first, 1);
                arrived = __shfl_sync(0xffffffffu, arrived, 0);
                if (arrived == last - first) {
                    if (lane == 0) a.arrived[first] = 0;
                    __threadfence();
                    join_rows<T, D, RM>(a, C, first, last, 0, live, 4, lane);
                }
            }
            fresh = true;
        }
        if (j + 1 < n) advance<TK, RM>(a, C, pre);
        if (++b == S) b = 0;
    }
    cp_wait<0>();
}

template <typename T, int D, int NB>
cudaError_t launch_rows(const AttendArgs& a, int sms, cudaStream_t st)
{
    using L = Few<D>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024 && L::WARPS <= ATTEND_WORKERS_PER_SM, "what a CTA has");
    cudaError_t e = allow_smem<k_attend_few<T, D, NB>>(most);
    if (e != cudaSuccess) return e;
    k_attend_few<T, D, NB><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t st)
{
    // 8 rows where the mean rows of a request's key head fit them (64 requests of about 1,500 tokens, 8 key
    // heads of 128: 8 rows 104 us with tiles of 8 and 111 of 16, 12 rows 145 and 121)
    if ((long long)a.tok.n_tok * a.kv.group <= 8ll * a.tok.n_req) return launch_rows<T, D, 1>(a, sms, st);
    return launch_rows<T, D, 2>(a, sms, st);
}

template <typename T>
cudaError_t launch_dim(const AttendArgs& a, int dim, int sms, cudaStream_t st)
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

cudaError_t launch_attend_few(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
