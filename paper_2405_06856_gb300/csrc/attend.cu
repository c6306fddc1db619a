// aladdin_worker_attend: attention of a step's new tokens over the paged cache.
//
// Request r has T new tokens, a tree (parent[t] < t or -1), and len cached
// tokens. Row (t, head g of key head h's group) has the scores
//     s_j = scale q . k_j,   j over the cached tokens, t's ancestors and t,
// and the results out = sum_j e^(s_j - lse) v_j, lse = log sum_j e^s_j.
//
// The rows of one (request, key head) share its keys, so they form the rows of
// a matrix product with K tiles and, after the softmax, with V tiles. The keys
// of a row tile, cached then new, are cut into tiles of KT; the tiles of all
// (request, head, row tile) units lie on one axis, which the CTAs share evenly:
// a CTA runs through a contiguous range, so that ragged requests and few long
// ones load every SM alike, and its copies run ahead across the units. A
// softmax goes over its tiles once with a running maximum and sum in 32 bits
// (base 2: the scores are multiplied by scale log2 e). A unit that CTAs share
// leaves a partial sum, maximum and accumulator from each; the one that
// arrives last adds them in the order of their keys, so that results do not
// depend on the order of arrival.
#include "worker_dev.cuh"

namespace aladdin {
namespace wk {
namespace {

template <int D>
struct Shape {
    static constexpr int KT = D == 64 ? 128 : 64;  // keys of a tile
    static constexpr int S = 3;                    // tiles in flight
};

// Where on the axis of all tiles a CTA is.
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

template <int KT, int RM>
__device__ __forceinline__ void locate(const AttendArgs& a, Cursor& u, const int* pre, int x)
{
    const int r = plan_find(pre, a.tok.n_req, x);
    enter<KT, RM>(a, u, r);
    const int y = x - pre[r], unit = y / u.c;
    u.tile = y - unit * u.c;
    u.h = unit / u.nrt;
    u.rt = unit - u.h * u.nrt;
}

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

// First tile of CTA i's range, and the CTA whose range holds tile x.
__device__ __forceinline__ int range_begin(int total, int ctas, int i)
{
    return (int)((long long)total * i / ctas);
}
__device__ __forceinline__ int range_of(int total, int ctas, int x)
{
    int i = (int)((long long)x * ctas / total);
    while (i + 1 < ctas && range_begin(total, ctas, i + 1) <= x) ++i;
    while (range_begin(total, ctas, i) > x) --i;
    return i;
}

// One partial: RM (maximum, sum) pairs, then RM x D accumulators.
template <int D, int RM>
__device__ __forceinline__ float* part_of(const AttendArgs& a, int cta, int slot)
{
    return a.part + ((size_t)cta * 2 + slot) * (size_t)(ATTEND_MAX_ROWS * (D + 2));
}

template <int D, int WR, int WK>
struct Smem {
    static constexpr int KT = Shape<D>::KT, S = Shape<D>::S, RM = WR * 16;
    static constexpr int TILE = tile_bytes<D>(KT);
    static_assert(WK == 1 || WK * RM * D * 4 <= 2 * TILE, "the warps' sums fit a tile's place");
    static constexpr bool QRING = RM == 16;               // the rows of a unit are fetched with its first tile
    static constexpr int QT = QRING ? tile_bytes<D>(RM) : 0;
    static constexpr int kv = 0;                          // S x (K tile, V tile)
    static constexpr int q = kv + S * 2 * TILE;           // S x RM rows
    static constexpr int ml = q + S * QT;                 // WK x RM (maximum, sum)
    static constexpr int anc = ml + WK * RM * 8;          // 64 masks
    static constexpr int scratch = anc + 64 * 8;          // 32 long longs
    static constexpr int par = scratch + 32 * 8;          // S x 64 parents
    static constexpr int ring = par + S * 64 * 4;         // (S + 1) x KT / 16 pages
    static constexpr int pre = ring + (S + 1) * (KT / 16) * 4 + 8;
    static constexpr int bytes(int n_req) { return pre + (n_req + 1) * 4; }
};

template <typename T, int D, int WR, int WK>
__global__ void __launch_bounds__(WR* WK * 32, D == 256 ? 1 : 2) k_attend(AttendArgs a)
{
    using L = Smem<D, WR, WK>;
    constexpr int KT = L::KT, S = L::S, RM = L::RM, NT = WR * WK * 32;
    constexpr int KW = KT / WK;      // keys of a warp in a tile
    constexpr int NS = KW / 8;       // score fragments
    constexpr int NO = D / 8;        // output fragments
    constexpr int CH = D / 8;        // 16-byte chunks of a row
    constexpr int PG = KT / 16;      // page look-ups of a tile
    extern __shared__ __align__(128) char sm[];
    const uint32_t sm0 = smem_addr(sm);
    int* const pre = reinterpret_cast<int*>(sm + L::pre);
    int* const ring = reinterpret_cast<int*>(sm + L::ring);
    int* const par = reinterpret_cast<int*>(sm + L::par);
    unsigned long long* const anc = reinterpret_cast<unsigned long long*>(sm + L::anc);
    float2* const ml = reinterpret_cast<float2*>(sm + L::ml);
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int wr = warp / WK, wk = warp - wr * WK;
    const int G = a.kv.group, H = a.kv.kv_heads;

    // the tiles of every request; a request whose offsets or length make no
    // sense has none and is recorded
    const int total = plan_prefix<NT>(
        a.tok.n_req, pre, reinterpret_cast<long long*>(sm + L::scratch), [&](int r) -> long long {
            const int lo = a.tok.off[r], hi = a.tok.off[r + 1], len = a.kv.len[r];
            if (lo < 0 || hi < lo || hi > a.tok.n_tok || hi - lo > ALADDIN_TREE_MAX || len < 0 ||
                len > a.kv.cap) {
                if (blockIdx.x == 0) atomicOr(a.err, WORKER_BAD_INPUT);
                return 0;
            }
            const int nt = hi - lo;
            return (long long)((nt * G + RM - 1) / RM) * H * ((len + nt + KT - 1) / KT);
        });
    if (total <= 0) {
        if (total < 0 && blockIdx.x == 0 && tid == 0) atomicOr(a.err, WORKER_BAD_INPUT);
        return;
    }
    // no more CTAs than tiles: every one of them has a part of the axis
    const int ctas = min((int)gridDim.x, total);
    if ((int)blockIdx.x >= ctas) return;
    const int begin = range_begin(total, ctas, blockIdx.x), end = range_begin(total, ctas, blockIdx.x + 1),
              n = end - begin;

    // the page of keys [16 g, 16 g + 16) of the tile under a cursor
    auto page_at = [&](const Cursor& u, int g) -> int {
        const int key = u.tile * KT + g * 16;
        if (key >= u.len) return -1;
        const int p = a.kv.table[(long long)u.r * a.kv.table_stride + (key >> a.kv.page_shift)];
        if ((unsigned)p >= (unsigned)a.kv.pages) {
            atomicOr(a.err, WORKER_BAD_INPUT);
            return -1;
        }
        return p;
    };
    // the pages of the first S tiles at once: one thread a look-up
    if (tid < (S - 1) * PG && tid / PG < n) {
        Cursor u;
        locate<KT, RM>(a, u, pre, begin + tid / PG);
        ring[tid] = page_at(u, tid % PG);
    }
    int page_next = -1;
    if (tid < PG && S - 1 < n) {
        Cursor u;
        locate<KT, RM>(a, u, pre, begin + S - 1);
        page_next = page_at(u, tid);
    }
    Cursor C, F;  // the tile computed, the tile fetched
    locate<KT, RM>(a, C, pre, begin);
    F = C;
    __syncthreads();

    // ordinal j of the CTA's tiles, under cursor F, into buffer j mod S, and with a
    // unit's first tile (ordinal fu of the units) its rows
    int fu = -1;
    auto fetch = [&](int j) {
        const int b = j % S, key0 = F.tile * KT;
        const uint32_t kd = sm0 + L::kv + b * 2 * L::TILE, vd = kd + L::TILE;
        const int* pg = ring + (j % (S + 1)) * PG;
        const long long head = (long long)F.h * a.kv.head_stride;
        constexpr int PER = (KT * CH + NT - 1) / NT;
        if (j == 0 || F.tile == 0) {
            ++fu;
            if constexpr (L::QRING) {
                const int rows = F.T * G - F.rt * RM;
#pragma unroll
                for (int i = 0; i < (RM * CH + NT - 1) / NT; ++i) {
                    const int x = tid + i * NT, row = x / CH, ch = x - row * CH;
                    if ((RM * CH) % NT && x >= RM * CH) break;
                    const bool ok = row < rows;
                    const int rho = F.rt * RM + row, t = ok ? rho / G : 0, g = ok ? rho - t * G : 0;
                    cp16(sm0 + L::q + (fu % S) * L::QT + tile_at<D>(row, ch),
                         a.tok.q + ((F.lo + t) * a.tok.q_stride + (long long)(F.h * G + g) * D + ch * 8) * 2, ok);
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
                const int row = r0 + i * STEP;
                const bool ok = pg[i * STEP / 16] >= 0;
                const long long x = ok ? (e[i * STEP / 16] + (i * STEP % 16) * a.kv.token_stride) * 2 : 0;
                const uint32_t d = tile_at<D>(row, ch);
                cp16(kd + d, a.kv.k + x, ok);
                cp16(vd + d, a.kv.v + x, ok);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int x = tid + i * NT, row = x / CH, ch = x - row * CH, key = key0 + row;
            if ((KT * CH) % NT && x >= KT * CH) break;
            const char *ks = a.kv.k, *vs = a.kv.v;
            bool ok = key < F.len + F.T;
            if (key < F.len) {
                const int p = pg[row >> 4];
                ok = p >= 0;
                const long long e = ok ? p * a.kv.page_stride + head +
                                             (key & (a.kv.page - 1)) * a.kv.token_stride + ch * 8
                                       : 0;
                ks += e * 2;
                vs += e * 2;
            } else if (ok) {
                const long long t = F.lo + key - F.len;
                ks = a.tok.k + (t * a.tok.k_stride + F.h * D + ch * 8) * 2;
                vs = a.tok.v + (t * a.tok.v_stride + F.h * D + ch * 8) * 2;
            }
            const uint32_t d = tile_at<D>(row, ch);
            cp16(kd + d, ks, ok);
            cp16(vd + d, vs, ok);
        }
        if (F.T > 1 && a.tok.parent && key0 + KT > F.len && tid < ALADDIN_TREE_MAX)
            cp4(smem_addr(par + b * ALADDIN_TREE_MAX + tid), a.tok.parent + F.lo + (tid < F.T ? tid : 0),
                tid < F.T);
    };
#pragma unroll
    for (int j = 0; j < S - 1; ++j) {
        if (j < n) {
            fetch(j);
            advance<KT, RM>(a, F, pre);
        }
        cp_commit();
    }

    uint32_t qf[D / 16][4];
    float o[NO][4], m[2], l[2];
    int row_tok[2];
    const int gq = lane >> 2, tq = lane & 3;
    bool fresh = true;
    int cu = -1;  // ordinal of the unit computed

    for (int j = 0; j < n; ++j) {
        cp_wait<S - 2>();
        if (tid < PG) ring[((j + S - 1) % (S + 1)) * PG + tid] = page_next;
        __syncthreads();
        if (j + S - 1 < n) {
            fetch(j + S - 1);
            if (j + S < n) {
                advance<KT, RM>(a, F, pre);
                if (tid < PG) page_next = page_at(F, tid);
            }
        }
        cp_commit();

        const int rows = C.T * G - C.rt * RM;  // rows of the tile that exist (may exceed RM)
        if (fresh) {
            fresh = false;
#pragma unroll
            for (int x = 0; x < NO; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.0f;
            m[0] = m[1] = -INFINITY;
            l[0] = l[1] = 0.0f;
            ++cu;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int rr = wr * 16 + gq + y * 8, rho = C.rt * RM + rr;
                const bool ok = rr < rows;
                const int t = ok ? rho / G : 0;
                row_tok[y] = t;
                if constexpr (!L::QRING) {
                    const char* p = a.tok.q + ((C.lo + t) * a.tok.q_stride +
                                               (long long)(C.h * G + (ok ? rho - t * G : 0)) * D) * 2;
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks) {
                        const uint32_t* w = reinterpret_cast<const uint32_t*>(p + ks * 32 + tq * 4);
                        qf[ks][y] = ok ? __ldg(w) : 0u;
                        qf[ks][y + 2] = ok ? __ldg(w + 4) : 0u;
                    }
                }
            }
            if constexpr (L::QRING) {
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                    ldmatrix4(qf[ks], sm0 + L::q + (cu % S) * L::QT +
                                          tile_at<D>((lane >> 3 & 1) * 8 + (lane & 7), ks * 2 + (lane >> 4)));
            }
        }

        const int b = j % S;
        const uint32_t kd = sm0 + L::kv + b * 2 * L::TILE, vd = kd + L::TILE;
        const int key0 = C.tile * KT, new0 = C.len - key0;  // the first new key's place in the tile
        const bool mixed = new0 < KT;                       // the tile holds new keys, or its last ones are none
        bool wild = false;
        if (mixed && C.T > 1) {
            if (tid < C.T) {
                unsigned long long see = 0;
                int u = tid;
                while (u >= 0) {
                    see |= 1ull << u;
                    int p = a.tok.parent ? par[b * ALADDIN_TREE_MAX + u] : u - 1;
                    if (p < -1 || p >= u) {
                        atomicOr(a.err, WORKER_BAD_INPUT);
                        p = -1;
                    }
                    u = p;
                }
                anc[tid] = see;
            }
            // a value that is not finite would reach rows that do not see its token
            // (0 times infinity): such a tile is summed key by key below
            bool w = false;
            const int k1 = min(KT, new0 + C.T);
            for (int x = max(new0, 0) * CH + tid; x < k1 * CH; x += NT) {
                const int row = x / CH;
                const uint4 q = *reinterpret_cast<const uint4*>(
                    sm + L::kv + (b * 2 + 1) * L::TILE + tile_at<D>(row, x - row * CH));
                w |= Num<T>::wild(q.x) || Num<T>::wild(q.y) || Num<T>::wild(q.z) || Num<T>::wild(q.w);
            }
            wild = __syncthreads_or(w);
        }

        if (wr * 16 < rows) {
            float s[NS][4];
            const int k0 = wk * KW;
#pragma unroll
            for (int x = 0; x < NS; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.0f;
            const int id = lane >> 3, lr = lane & 7;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
                for (int x = 0; x < NS; x += 2) {
                    uint32_t f[4];
                    ldmatrix4(f, kd + tile_at<D>(k0 + x * 8 + (id >> 1) * 8 + lr, ks * 2 + (id & 1)));
                    Num<T>::mma(s[x], qf[ks], f[0], f[1]);
                    Num<T>::mma(s[x + 1], qf[ks], f[2], f[3]);
                }
            }
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int x = 0; x < NS; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e) s[x][e] *= a.scale_log2;
            }
            // keys of a page outside the pool (-1, as are the pages behind the cached keys)
            const int* pg = ring + (j % (S + 1)) * PG + k0 / 16;
            if (!mixed) {
#pragma unroll
                for (int x = 0; x < NS; x += 2) {
                    if (pg[x / 2] < 0) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[x][e] = s[x + 1][e] = -INFINITY;
                    }
                }
            } else {
                const unsigned long long see[2] = {C.T > 1 ? anc[row_tok[0]] : 1, C.T > 1 ? anc[row_tok[1]] : 1};
#pragma unroll
                for (int x = 0; x < NS; ++x) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = k0 + x * 8 + tq * 2 + (e & 1), u = k - new0;
                        const bool ok = u < 0 ? pg[x / 2] >= 0 : u < 64 && (see[e >> 1] >> u & 1);
                        if (!ok) s[x][e] = -INFINITY;
                    }
                }
            }
#pragma unroll
            for (int x = 0; x < NS; ++x) {
                top[0] = fmaxf(top[0], fmaxf(s[x][0], s[x][1]));
                top[1] = fmaxf(top[1], fmaxf(s[x][2], s[x][3]));
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                top[y] = fmaxf(top[y], __shfl_xor_sync(0xffffffffu, top[y], 1));
                top[y] = fmaxf(top[y], __shfl_xor_sync(0xffffffffu, top[y], 2));
                top[y] = fmaxf(top[y], m[y]);
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const float f = top[y] > m[y] ? ex2(m[y] - top[y]) : 1.0f;
                    m[y] = top[y];
                    l[y] *= f;
#pragma unroll
                    for (int x = 0; x < NO; ++x) {
                        o[x][y * 2] *= f;
                        o[x][y * 2 + 1] *= f;
                    }
                }
            }
            const float base[2] = {m[0] == -INFINITY ? 0.0f : m[0], m[1] == -INFINITY ? 0.0f : m[1]};
#pragma unroll
            for (int x = 0; x < NS; ++x) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[x][e] = ex2(s[x][e] - base[e >> 1]);
                    l[e >> 1] += s[x][e];
                }
            }
            if (!wild) {
#pragma unroll
                for (int x = 0; x < NS; x += 2) {
                    const uint32_t p[4] = {Num<T>::pack(s[x][0], s[x][1]), Num<T>::pack(s[x][2], s[x][3]),
                                           Num<T>::pack(s[x + 1][0], s[x + 1][1]),
                                           Num<T>::pack(s[x + 1][2], s[x + 1][3])};
#pragma unroll
                    for (int y = 0; y < NO; y += 2) {
                        uint32_t f[4];
                        ldmatrix4t(f, vd + tile_at<D>(k0 + x * 8 + (id & 1) * 8 + lr, y + (id >> 1)));
                        Num<T>::mma(o[y], p, f[0], f[1]);
                        Num<T>::mma(o[y + 1], p, f[2], f[3]);
                    }
                }
            } else {
#pragma unroll
                for (int x = 0; x < NS; ++x) {
#pragma unroll 1
                    for (int k = 0; k < 8; ++k) {
                        const int src = (lane & 28) | (k >> 1);
                        const float pe0 = __shfl_sync(0xffffffffu, s[x][0], src),
                                    po0 = __shfl_sync(0xffffffffu, s[x][1], src),
                                    pe1 = __shfl_sync(0xffffffffu, s[x][2], src),
                                    po1 = __shfl_sync(0xffffffffu, s[x][3], src);
                        const float p0 = k & 1 ? po0 : pe0, p1 = k & 1 ? po1 : pe1;
#pragma unroll
                        for (int y = 0; y < NO; ++y) {
                            const float2 v = Num<T>::unpack(*reinterpret_cast<const uint32_t*>(
                                sm + L::kv + (b * 2 + 1) * L::TILE + tile_at<D>(k0 + x * 8 + k, y) + tq * 4));
                            if (p0 != 0.0f) {
                                o[y][0] += p0 * v.x;
                                o[y][1] += p0 * v.y;
                            }
                            if (p1 != 0.0f) {
                                o[y][2] += p1 * v.x;
                                o[y][3] += p1 * v.y;
                            }
                        }
                    }
                }
            }
        }

        const bool unit_ends = C.tile + 1 == C.c;
        if (unit_ends || j + 1 == n) {
            const int unit0 = begin + j - C.tile, unit1 = unit0 + C.c;  // the unit on the axis
            const bool whole = unit0 >= begin && unit1 <= end;
            const int live = rows < RM ? rows : RM;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                l[y] += __shfl_xor_sync(0xffffffffu, l[y], 1);
                l[y] += __shfl_xor_sync(0xffffffffu, l[y], 2);
            }
            float* const part = part_of<D, RM>(a, blockIdx.x, unit0 >= begin ? 1 : 0);
            // results of row rr: written where the unit is whole, else left for the join
            auto put2 = [&](int rr, int col, float x, float y, float sum) {
                if (whole) {
                    const int rho = C.rt * RM + rr, t = rho / G, head = C.h * G + rho - t * G;
                    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
                    *reinterpret_cast<uint32_t*>(
                        a.out + ((C.lo + t) * a.out_stride + (long long)head * D + col) * 2) =
                        Num<T>::pack(x * inv, y * inv);
                } else {
                    *reinterpret_cast<float2*>(part + RM * 2 + rr * D + col) = make_float2(x, y);
                }
            };
            auto put_ml = [&](int rr, float top, float sum) {
                if (whole) {
                    if (a.lse) {
                        const int rho = C.rt * RM + rr, t = rho / G, head = C.h * G + rho - t * G;
                        a.lse[(long long)(C.lo + t) * (H * G) + head] = (top + log2f(sum)) * LN2;
                    }
                } else {
                    *reinterpret_cast<float2*>(part + rr * 2) = make_float2(top, sum);
                }
            };
            if constexpr (WK > 1) {
                if (tq == 0) {
                    ml[wk * RM + wr * 16 + gq] = make_float2(m[0], l[0]);
                    ml[wk * RM + wr * 16 + gq + 8] = make_float2(m[1], l[1]);
                }
                // the tile's place takes every warp's sums (8 floats a group, the groups of a
                // row turned by the row, so that a warp's rows lie in different banks)
                __syncthreads();
                float* const sums = reinterpret_cast<float*>(sm + L::kv + b * 2 * L::TILE);
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    float* d = sums + (wk * RM + wr * 16 + gq + y * 8) * D + tq * 2;
#pragma unroll
                    for (int x = 0; x < NO; ++x) {
                        const int at = x + gq < NO ? x + gq : x + gq - NO;
                        *reinterpret_cast<float2*>(d + at * 8) = make_float2(o[x][y * 2], o[x][y * 2 + 1]);
                    }
                }
                __syncthreads();
                for (int x = tid; x < live * (D / 2); x += NT) {
                    const int rr = x / (D / 2), col = (x - rr * (D / 2)) * 2;
                    const int turned = (col >> 3) + (rr & 7), at = (turned < NO ? turned : turned - NO) * 8 + (col & 7);
                    float top = -INFINITY, sum = 0.0f;
                    float2 v = make_float2(0.0f, 0.0f);
#pragma unroll
                    for (int w = 0; w < WK; ++w) top = fmaxf(top, ml[w * RM + rr].x);
#pragma unroll
                    for (int w = 0; w < WK; ++w) {
                        const float2 q = ml[w * RM + rr];
                        const float f = q.x == -INFINITY ? 0.0f : ex2(q.x - top);
                        const float2 u = *reinterpret_cast<const float2*>(sums + (w * RM + rr) * D + at);
                        sum += q.y * f;
                        v.x += u.x * f;
                        v.y += u.y * f;
                    }
                    put2(rr, col, v.x, v.y, sum);
                    if (col == 0) put_ml(rr, top, sum);
                }
            } else {
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int rr = wr * 16 + gq + y * 8;
                    if (rr < live) {
#pragma unroll
                        for (int x = 0; x < NO; ++x) put2(rr, x * 8 + tq * 2, o[x][y * 2], o[x][y * 2 + 1], l[y]);
                        if (tq == 0) put_ml(rr, m[y], l[y]);
                    }
                }
            }
            if (!whole) {
                const int first = range_of(total, ctas, unit0), last = range_of(total, ctas, unit1 - 1);
                __threadfence();
                __syncthreads();
                if (tid == 0) s_last = atomicAdd(a.arrived + first, 1) == last - first;
                __syncthreads();
                if (s_last) {
                    if (tid == 0) a.arrived[first] = 0;
                    __threadfence();
                    // CTA `first` holds the unit's start in slot 1, the others theirs in slot 0
                    for (int rr = warp; rr < live; rr += NT / 32) {
                        float top = -INFINITY;
                        for (int i = first + lane; i <= last; i += 32)
                            top = fmaxf(top, __ldcg(part_of<D, RM>(a, i, i == first) + rr * 2));
#pragma unroll
                        for (int x = 16; x; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
                        const float ref = top == -INFINITY ? 0.0f : top;
                        float sum = 0.0f;
                        float2 acc[(D + 63) / 64];
#pragma unroll
                        for (int x = 0; x < (D + 63) / 64; ++x) acc[x] = make_float2(0.0f, 0.0f);
#pragma unroll 4
                        for (int i = first; i <= last; ++i) {
                            const float* p = part_of<D, RM>(a, i, i == first);
                            const float2 v = __ldcg(reinterpret_cast<const float2*>(p + rr * 2));
                            const float f = ex2(v.x - ref);
                            sum += v.y * f;
#pragma unroll
                            for (int x = 0; x < (D + 63) / 64; ++x) {
                                const int col = x * 64 + lane * 2;
                                if (D % 64 == 0 || col < D) {
                                    const float2 w =
                                        __ldcg(reinterpret_cast<const float2*>(p + RM * 2 + rr * D + col));
                                    acc[x].x += f * w.x;
                                    acc[x].y += f * w.y;
                                }
                            }
                        }
                        const int rho = C.rt * RM + rr, t = rho / G, head = C.h * G + rho - t * G;
                        const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
                        for (int x = 0; x < (D + 63) / 64; ++x) {
                            const int col = x * 64 + lane * 2;
                            if (D % 64 == 0 || col < D)
                                *reinterpret_cast<uint32_t*>(
                                    a.out + ((C.lo + t) * a.out_stride + (long long)head * D + col) * 2) =
                                    Num<T>::pack(acc[x].x * inv, acc[x].y * inv);
                        }
                        if (lane == 0 && a.lse)
                            a.lse[(long long)(C.lo + t) * (H * G) + head] = (ref + log2f(sum)) * LN2;
                    }
                }
            }
            fresh = true;
        }
        if (j + 1 < n) advance<KT, RM>(a, C, pre);
    }
    cp_wait<0>();
}

template <typename T, int D, int WR, int WK>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t st)
{
    using L = Smem<D, WR, WK>;
    const int smem = L::bytes(a.tok.n_req);
    static_assert(L::bytes(ALADDIN_WORKER_MAX_REQUESTS) <= 227 * 1024 - 256, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_attend<T, D, WR, WK>>(L::bytes(ALADDIN_WORKER_MAX_REQUESTS));
    if (e != cudaSuccess) return e;
    // at most one CTA a tile: the table's width bounds a request's cached tokens
    const long long units = (long long)a.tok.n_req * a.kv.kv_heads *
                            ((long long)(a.tok.n_tok < ALADDIN_TREE_MAX ? a.tok.n_tok : ALADDIN_TREE_MAX) *
                                 a.kv.group / L::RM + 1);
    const long long tiles = units * (a.kv.cap / L::KT + 2);
    const long long most = 2ll * sms;
    k_attend<T, D, WR, WK><<<(int)(tiles < most ? tiles : most), WR * WK * 32, smem, st>>>(a);
    return cudaGetLastError();
}

// Warps along the rows and along the keys by the mean rows of a request's
// key head: 16 rows leave the tile's keys to four warps, 64 rows its rows.
template <typename T, int D>
cudaError_t launch_rows(const AttendArgs& a, int sms, cudaStream_t st)
{
    const long long rows = ((long long)a.tok.n_tok * a.kv.group + a.tok.n_req - 1) / a.tok.n_req;
    if (rows <= 16) return launch<T, D, 1, 4>(a, sms, st);
    if constexpr (D < 256) {
        if (rows <= 32) return launch<T, D, 2, 2>(a, sms, st);
    }
    return launch<T, D, 4, 1>(a, sms, st);
}

template <typename T>
cudaError_t launch_dim(const AttendArgs& a, int dim, int sms, cudaStream_t st)
{
    switch (dim) {
        case 64: return launch_rows<T, 64>(a, sms, st);
        case 96: return launch_rows<T, 96>(a, sms, st);
        case 128: return launch_rows<T, 128>(a, sms, st);
        case 256: return launch_rows<T, 256>(a, sms, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace
}  // namespace wk

size_t attend_part_bytes(int ctas, int dim)
{
    return (size_t)ctas * 2 * ATTEND_MAX_ROWS * (dim + 2) * sizeof(float);
}

cudaError_t launch_attend(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
