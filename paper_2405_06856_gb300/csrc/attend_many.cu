// aladdin_worker_attend where the rows of a (request, key head) are many (trees of
// drafted tokens, large groups): the products run on the fifth-generation tensor
// cores (tcgen05). See attend.cuh for the operator.
//
// A CTA runs through a range of the axis of all key tiles, MT tiles of 128 rows at
// a time. Its warps have roles:
//   three warps copy keys and values (and at a unit's start its queries) into a ring
//   of shared memory, in the order K0 V0 K1 V1 ..., in the 128-byte-swizzled layout
//   of the matrix descriptors: tiles of cached tokens by tensor copies (TMA), a page
//   or a part of one each, that one thread starts; the queries and the tiles with new
//   tokens by asynchronous copies of 16 bytes, signalled a few copies later;
//   one thread issues the products: scores S = Q K' into tensor memory, and out +=
//   P V with the weights P, 16 bits each, from tensor memory in the place of S;
//   four warps for each row tile do the softmax, one thread a row: the maximum and
//   the exponentials need no exchange between threads.
// With two row tiles the tensor cores work on one while the softmax works on the
// other; with one, the scores of the next tile are formed ahead into a second
// place. The accumulator stays in tensor memory; it is rescaled only when a row's
// maximum has grown by more than 2^8 over the one that its weights refer to, which
// 32-bit sums and 16-bit weights hold without loss. The softmax's loops stay rolled
// (unrolled over a tile, with the scores read once and the weights held in registers,
// and with three exponentials of eight as polynomials, a call took 267 us for 205).
//
// Measured: 24 requests of 60,854 cached tokens with trees of up to 64 tokens, 64 query and 8
// key heads of 128 channels in f16: 184 us, 553 TFLOP/s of 1,932 that a large product
// reaches; a product of 128 x 128 x 16 takes 98 cycles of the 64 that it takes alone, as operands
// and copies share the shared memory. 37 requests of 57,837 tokens with chains of up to 5
// tokens, 28 and 4 heads of 96: 49 us, 1.9 TB/s.
//
// New tokens' values that are not finite would reach rows that do not see them
// (0 times infinity): they are replaced by 0 in shared memory, and rows that do
// see them get them added at the end.
#include <cuda.h>

#include "attend.cuh"
#include "tensor_dev.cuh"

namespace aladdin {
namespace wk {
namespace {

// A box of a tensor map (coordinates: channel, token of the page, head, page) into shared
// memory; its bytes count on bar. The channel is a multiple of 64.
__device__ __forceinline__ void box_copy(uint32_t dst, const CUtensorMap* map, int channel, int token, int head,
                                         int page, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, "
        "%5}], [%6];" ::"r"(dst),
        "l"(map), "r"(channel), "r"(token), "r"(head), "r"(page), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, int bytes)
{
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

// Boxes of 64 channels by `rows` tokens of the cache's keys and values.
struct Maps {
    CUtensorMap k, v;
    int rows;  // a power of two, at most a page and a tile
};

template <int D, int MT>
struct Many {
    // (two CTAs an SM with tiles of 64 keys, for one row tile, were slower: 56 us for 50, as units
    // were split and joined more often)
    static constexpr int KT = D == 256 ? 64 : 128;       // keys of a tile
    static constexpr int RM = 128 * MT;                  // rows of a unit
    static constexpr int HALVES = (D + 63) / 64;         // blocks of 64 channels
    static constexpr int TILE = HALVES * KT * 128;       // a tile of keys or values
    static constexpr int QT = HALVES * 128 * 128;        // 128 rows of queries
    static constexpr int NQ = MT == 1 && D < 256 ? 2 : 1;  // sets of queries
    static constexpr int ROOM = 220 * 1024 - NQ * MT * QT;
    static constexpr int NB = ROOM / TILE < 8 ? ROOM / TILE : 8;  // tiles of the ring
    static_assert(NB >= 4, "keys and values of two tiles");
    static constexpr int q = NB * TILE;
    static constexpr int bars = q + NQ * MT * QT;        // full NB, empty NB, the queries' 2 NQ, then 2 x 4, 1
    static constexpr int full = bars, empty = full + NB * 8, qfull = empty + NB * 8, qempty = qfull + NQ * 8,
                         sready = qempty + NQ * 8, pready = sready + 16, odone = pready + 16, ofree = odone + 16,
                         over = ofree + 16, tmem = over + 16;
    static constexpr int okm = tmem + 16;                // 8 masks of valid pages, a tile each
    static constexpr int wild = okm + 8 * 4;             // 8 flags of units
    static constexpr int late = wild + 8 * 4;            // whether a wait ran out
    static constexpr int scratch = late + 8;
    static constexpr int pre = scratch + 32 * 8;
    static constexpr int bytes(int n_req) { return pre + (n_req + 1) * 8; }
    static constexpr int COPIES = 3;                     // warps that copy
    static constexpr int WARPS = 4 * MT + 1 + COPIES;    // softmax, products, copies
    // columns of tensor memory: the scores' two places, the accumulators
    static constexpr int s0 = 0, o0 = 2 * KT;
    static_assert(o0 + MT * HALVES * 64 <= 512, "tensor memory");
    static constexpr int LAG = 3;                        // copies in flight behind the one signalled
};

// What a unit costs beside its tiles, in keys.
constexpr int UNIT_KEYS = 512;

template <typename T, int D, int MT>
__global__ void __launch_bounds__(Many<D, MT>::WARPS * 32, 1) k_attend_many(AttendArgs a, const __grid_constant__ Maps maps)
{
    using L = Many<D, MT>;
    constexpr int KT = L::KT, RM = L::RM, NB = L::NB, NQ = L::NQ, NT = L::WARPS * 32, CH = D / 8, PG = KT / 16;
    extern __shared__ __align__(1024) char sm[];
    const uint32_t sm0 = smem_addr(sm);
    int* const pre = reinterpret_cast<int*>(sm + L::pre);
    volatile int* const okm = reinterpret_cast<volatile int*>(sm + L::okm);
    // (a tile's mask, a unit's flag: the copies run fewer than 8 tiles ahead of the softmax)
    volatile int* const wilds = reinterpret_cast<volatile int*>(sm + L::wild);
    volatile int* const late = reinterpret_cast<volatile int*>(sm + L::late);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int G = a.kv.group, H = a.kv.kv_heads;

    if (sm0 & 1023) {  // the operands' layout wants it
        if (tid == 0) atomicOr(a.err, WORKER_TIMEOUT);
        return;
    }
    Axis ax;
    if (!plan<NT>(a.tok.n_req, ax, pre, pre + a.tok.n_req + 1, reinterpret_cast<long long*>(sm + L::scratch),
                  (int)gridDim.x, UNIT_KEYS / KT, 1, a.err,
                  [&](int r, int& c) { return attend_units<KT, RM>(a, r, c); }))
        return;
    const int me = blockIdx.x;
    if (me >= ax.workers) return;
    Cursor C;
    const int n = range<KT, RM>(a, ax, C, me);
    if (n == 0) return;

    if (warp == 0) tmem_alloc(sm0 + L::tmem, 512);
    if (tid == 0) {
        for (int b = 0; b < NB; ++b) {
            mbar_init(sm0 + L::full + b * 8, L::COPIES);
            mbar_init(sm0 + L::empty + b * 8, 1);
        }
        for (int b = 0; b < NQ; ++b) {
            mbar_init(sm0 + L::qfull + b * 8, L::COPIES);
            mbar_init(sm0 + L::qempty + b * 8, 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(sm0 + L::sready + w * 8, 1);
            mbar_init(sm0 + L::pready + w * 8, 4);
            mbar_init(sm0 + L::odone + w * 8, 1);
            mbar_init(sm0 + L::ofree + w * 8, 4);
        }
        mbar_init(sm0 + L::over, 1);
        for (int u = 0; u < 8; ++u) wilds[u] = 0;
        *late = 0;
        mbar_init_fence();
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tm = *reinterpret_cast<volatile uint32_t*>(sm + L::tmem);

    // A wait that runs out is recorded and ends its warp's part; the others' waits run
    // out after it (no warps meet at a barrier without a limit before the end), and all meet at
    // the end, where what is in flight is waited for and tensor memory is freed.
    auto wait = [&](uint32_t bar, int phase) -> bool {
        if (mbar_wait(bar, phase & 1)) return true;
        atomicOr(a.err, WORKER_TIMEOUT);
        return false;
    };
    int filled = 0;  // places of the ring that a copying warp has filled
    bool ok = true;  // no wait of this warp ran out

    if (warp >= 4 * MT + 1) {
        // ------------------------------------------------------------ copies
        constexpr int CT = L::COPIES * 32, STEP = CT / CH;  // rows that the threads copy at a time
        static_assert(CT % CH == 0, "a thread copies one chunk of every STEP-th row");
        const int ct = tid - (4 * MT + 1) * 32, cw = ct >> 5, r0 = ct / CH, ch = ct % CH;
        // the page of keys [16 lane, 16 lane + 16) of the tile under u, as the table has it
        auto pages = [&](const Cursor& u) -> int {
            const int key = u.tile * KT + lane * 16;
            return lane < PG && key < u.len
                       ? a.kv.table[(long long)u.r * a.kv.table_stride + (key >> a.kv.page_shift)]
                       : 0;
        };
        // byte of this thread's chunk of row `row` in a block of `rows` rows
        auto at = [&](int row, int rows) {
            return (uint32_t)((ch >> 3) * rows * 128 + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
        };
        int units = -1, waiting = 0;   // copies of 16 bytes a time that are not signalled yet: the oldest first,
        uint32_t slots = 0;            // 8 bits each, the slot + 1 or (queries) 128 + their set
        auto landed = [&]() {
            fence_async();
            __syncwarp();
            const uint32_t x = slots & 255;
            if (lane == 0) mbar_arrive(sm0 + (x & 128 ? L::qfull + (x & 127) * 8 : L::full + (x - 1) * 8));
            slots >>= 8;
            --waiting;
        };
        auto copied = [&](uint32_t x) {  // the copies since the last call are one
            cp_commit();
            slots |= x << (8 * waiting);
            if (++waiting > L::LAG) {
                cp_wait<L::LAG>();
                landed();
            }
        };
        auto drain = [&]() {
            if (waiting) cp_wait<0>();
            while (waiting) landed();
        };
        // waits for a place; what is in flight is signalled first where it is not free yet
        auto room = [&](uint32_t bar, int phase) {
            if (__all_sync(0xffffffffu, mbar_test(bar, phase & 1))) return;
            drain();
            ok = __all_sync(0xffffffffu, wait(bar, phase));
        };
        int page = pages(C);
        for (int j = 0; j < n && ok; ++j) {
            const bool start = j == 0 || C.tile == 0;
            const bool have = (unsigned)page < (unsigned)a.kv.pages;
            if (lane < PG && !have && cw == 0) atomicOr(a.err, WORKER_BAD_INPUT);
            const unsigned mask = __ballot_sync(0xffffffffu, have) & ((1u << PG) - 1);
            Cursor N = C;  // the next tile, its pages on their way
            int page_next = 0;
            if (j + 1 < n) {
                advance<KT, RM>(a, N, pre);
                page_next = pages(N);
            }
            const int key0 = C.tile * KT, own = C.len - key0, all = own + C.T;
            // boxes of cached keys, in turn to the warps, one a lane
            const int boxes = maps.rows ? min(max(own, 0), KT) / maps.rows : 0, rest = boxes * maps.rows;
            const int box = lane * L::COPIES + cw, box_half = box % L::HALVES, box_row = box / L::HALVES * maps.rows;
            const int box_page = __shfl_sync(0xffffffffu, have ? page : a.kv.pages, box_row >> 4 & 31);
            const int my_boxes = (boxes * L::HALVES - cw + L::COPIES - 1) / L::COPIES;
#pragma unroll 1
            for (int part = 0; part < 2 && ok; ++part) {  // keys, values
                const int i = 2 * j + part, slot = i % NB;
                if (i >= NB) room(sm0 + L::empty + slot * 8, i / NB - 1);
                if (!ok) break;
                const uint32_t d = sm0 + slot * L::TILE, bar = sm0 + L::full + slot * 8;
                if (part == 0 && start) {
                    ++units;
                    if (units >= NQ) room(sm0 + L::qempty + units % NQ * 8, units / NQ - 1);
                    if (!ok) break;
                }
                if (boxes) {
                    if (lane == 0) mbar_expect(bar, my_boxes * maps.rows * 128);
                    __syncwarp();
                    // (a page outside the pool, whatever its index: the one behind the pool, which
                    // gives zeros, and the tile's mask hides them)
                    if (lane < my_boxes)
                        box_copy(d + box_half * KT * 128 + box_row * 128, part ? &maps.v : &maps.k, box_half * 64,
                                 (key0 + box_row) & (a.kv.page - 1), C.h, box_page, bar);
                    __syncwarp();
                }
                if (part == 0 && ct == 0) okm[j & 7] = (int)mask;
                if (rest == KT) {
                    if (lane == 0) mbar_arrive(bar);
                } else {
                    bool w = false;
                    // cached rows behind the boxes
                    const char* const pool = part ? a.kv.v : a.kv.k;
                    const long long head = (long long)C.h * a.kv.head_stride + ch * 8;
                    for (int row0 = rest; row0 < min(own, KT); row0 += STEP) {
                        const int row = row0 + r0, p = __shfl_sync(0xffffffffu, page, row >> 4 & 31);
                        if (row < min(own, KT)) {
                            const bool ok1 = mask >> (row >> 4) & 1;
                            const long long e = ok1 ? p * a.kv.page_stride + head +
                                                          ((key0 + row) & (a.kv.page - 1)) * a.kv.token_stride
                                                    : 0;
                            cp16(d + at(row, KT), pool + e * 2, ok1);
                        }
                    }
                    // new tokens
                    const int lo = max(own, 0), hi = min(all, KT);
                    if (part == 0) {
                        const char* src = a.tok.k + ((long long)(C.lo + lo + r0 - own) * a.tok.k_stride + C.h * D + ch * 8) * 2;
                        for (int row = lo + r0; row < hi; row += STEP, src += STEP * a.tok.k_stride * 2)
                            cp16(d + at(row, KT), src, true);
                        // (keys of rows that hold no token are masked, whatever they are)
                    } else {
                        // values that are not finite become 0
                        const char* src = a.tok.v + ((long long)(C.lo + lo + r0 - own) * a.tok.v_stride + C.h * D + ch * 8) * 2;
                        for (int row = lo + r0; row < hi; row += 4 * STEP) {
                            uint4 v[4];
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                v[x] = make_uint4(0, 0, 0, 0);
                                if (row + x * STEP < hi) v[x] = *reinterpret_cast<const uint4*>(src);
                                src += STEP * a.tok.v_stride * 2;
                            }
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                if (Num<T>::wild(v[x].x) || Num<T>::wild(v[x].y) || Num<T>::wild(v[x].z) ||
                                    Num<T>::wild(v[x].w)) {
                                    w = true;
                                    v[x].x = Num<T>::tame(v[x].x), v[x].y = Num<T>::tame(v[x].y);
                                    v[x].z = Num<T>::tame(v[x].z), v[x].w = Num<T>::tame(v[x].w);
                                }
                                if (row + x * STEP < hi)
                                    *reinterpret_cast<uint4*>(sm + slot * L::TILE + at(row + x * STEP, KT)) = v[x];
                            }
                        }
                        // weights of 0 meet the values of rows that hold no token: zeros
                        for (int row = hi + r0; row < KT; row += STEP)
                            *reinterpret_cast<uint4*>(sm + slot * L::TILE + at(row, KT)) = make_uint4(0, 0, 0, 0);
                        if (w) wilds[units & 7] = units + 1;
                    }
                    copied(slot + 1);
                }
                if (part == 0 && start) {
                    // the unit's queries, behind its first keys
                    const int rows = min(C.T * G - C.rt * RM, RM);
                    const uint32_t qd = sm0 + L::q + units % NQ * (MT * L::QT);
                    int t = (C.rt * RM + r0) / G, g = C.rt * RM + r0 - t * G;
                    const char* const base = a.tok.q + ((long long)C.lo * a.tok.q_stride + (long long)C.h * G * D + ch * 8) * 2;
#pragma unroll 4
                    for (int row = r0; row < rows; row += STEP) {
                        cp16(qd + (row >> 7) * L::QT + at(row & 127, 128), base + (t * a.tok.q_stride + g * D) * 2, true);
                        g += STEP;
                        while (g >= G) g -= G, ++t;
                    }
                    copied(128 | units % NQ);
                    drain();
                }
                ++filled;
            }
            C = N;
            page = page_next;
        }
        drain();
    } else if (warp == 4 * MT) {
        // ------------------------------------------------------------ products
        {
            constexpr uint32_t qk = product<T>(KT, false), pv = product<T>(D, true);
            const bool leader = elected();
            Cursor N = C;  // the tile whose scores are formed next
            int scored = 0, units = -1, run0 = 0, run1 = 0, start0 = 0, start1 = 0;
            // scores of tile `scored` for row tile w, into place s
            auto scores = [&](int w, int s) {
                const uint32_t k0 = operand_lo(sm0 + 2 * scored % NB * L::TILE, 0),
                               q0 = operand_lo(sm0 + L::q + (units % NQ * MT + w) * L::QT, 0);
                if (leader) {
#pragma unroll
                    for (int x = 0; x < D / 16; ++x)
                        tc_mma_ss(tm + L::s0 + s * KT, whole(q0 + ((x >> 2) * 128 * 128 + (x & 3) * 32) / 16, OPERAND_HI),
                                  whole(k0 + ((x >> 2) * KT * 128 + (x & 3) * 32) / 16, OPERAND_HI), qk, x > 0);
                    tc_commit(sm0 + L::sready + s * 8);
                }
                __syncwarp();
            };
            // waits for the keys (and queries) of the tile under N
            auto enter_tile = [&]() {
                if (scored == 0 || N.tile == 0) {
                    ++units;
                    ok = ok && wait(sm0 + L::qfull + units % NQ * 8, units / NQ);
                }
                ok = __all_sync(0xffffffffu, ok && wait(sm0 + L::full + 2 * scored % NB * 8, 2 * scored / NB));
                tc_after();
            };
            // the tile under N has its scores on the way
            auto leave_tile = [&]() {
                if (leader) {
                    tc_commit(sm0 + L::empty + 2 * scored % NB * 8);
                    if (N.tile + 1 == N.c) tc_commit(sm0 + L::qempty + units % NQ * 8);
                }
                __syncwarp();
                if (++scored < n) advance<KT, RM>(a, N, pre);
            };
            auto active = [&](const Cursor& u, int w) { return u.T * G - u.rt * RM > w * 128; };
            enter_tile();
            if (ok) {
                for (int w = 0; w < MT; ++w)
                    if (active(N, w)) scores(w, w);
                leave_tile();
            }
            for (int j = 0; j < n && ok; ++j) {
                const bool more = j + 1 < n;
                if (MT == 1 && more) {
                    enter_tile();
                    if (!ok) break;
                    scores(0, (j + 1) & 1);
                    leave_tile();
                }
                const int v = 2 * j + 1;
                // (the next unit's queries may not be there yet: this unit's values come first)
                const bool turns = C.tile + 1 == C.c;
#pragma unroll
                for (int w = 0; w < MT; ++w) {
                    if (active(C, w)) {
                        const bool start = j == 0 || C.tile == 0;
                        ok = ok && wait(sm0 + L::pready + w * 8, (w ? run1 : run0)++);
                        ok = ok && wait(sm0 + L::full + v % NB * 8, v / NB);
                        if (start && (w ? start1 : start0)++ > 0)
                            ok = ok && wait(sm0 + L::ofree + w * 8, (w ? start1 : start0) - 2);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        tc_after();
                        const uint32_t v0 = operand_lo(sm0 + v % NB * L::TILE, KT * 128),
                                       p = tm + L::s0 + (MT == 1 ? j & 1 : w) * KT;
                        if (leader) {
#pragma unroll
                            for (int x = 0; x < KT / 16; ++x)
                                tc_mma_ts(tm + L::o0 + w * (L::HALVES * 64), p + x * 8,
                                          whole(v0 + x * 2048 / 16, OPERAND_HI), pv, !start || x > 0);
                            tc_commit(sm0 + L::odone + w * 8);
                        }
                        __syncwarp();
                    }
                    if (MT == 2 && more && !turns) {
                        if (w == 0) {
                            enter_tile();
                            if (!ok) break;
                        }
                        if (active(N, w)) scores(w, w);
                    }
                }
                if (!ok) break;
                if (leader) tc_commit(sm0 + L::empty + v % NB * 8);
                __syncwarp();
                if (MT == 2 && more && turns) {
                    enter_tile();
                    if (!ok) break;
#pragma unroll
                    for (int w = 0; w < MT; ++w)
                        if (active(N, w)) scores(w, w);
                }
                if (MT == 2 && more) leave_tile();
                if (more) advance<KT, RM>(a, C, pre);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax
        const int w = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16, om = tm + lanes + L::o0 + w * (L::HALVES * 64);
        float m = -INFINITY, l = 0.0f;
        unsigned long long see = 0;
        int token = 0, units = -1, tile0 = 0, used[2] = {0, 0}, done = 0;
        for (int j = 0; j < n && ok; ++j) {
            const bool start = j == 0 || C.tile == 0, unit_ends = C.tile + 1 == C.c;
            const int rows = C.T * G - C.rt * RM - w * 128;
            if (start) {
                ++units;
                tile0 = C.tile;
            }
            if (rows > 0) {
                if (start) {
                    m = -INFINITY;
                    l = 0.0f;
                    const int rho = C.rt * RM + w * 128 + row;
                    token = row < rows ? rho / G : 0;
                    see = ancestors(a, C, token);
                }
                const int s = MT == 1 ? j & 1 : w;
                ok = __all_sync(0xffffffffu, wait(sm0 + L::sready + s * 8, used[MT == 1 ? s : 0]++));
                if (!ok) break;
                tc_after();
                const uint32_t st = tm + lanes + L::s0 + s * KT;
                const int new0 = C.len - C.tile * KT;  // the first new key's place in the tile
                const unsigned valid = (unsigned)okm[j & 7];
                const bool masked = new0 < KT || valid != (1u << PG) - 1;
                // what this row sees of keys 32 c ..: cached ones of valid pages, then new ones
                auto mask = [&](uint32_t(&v)[32], int c) {
                    const int at = new0 - c * 32;  // the first new key's place in the 32
                    const uint32_t pages = (valid >> (c * 2) & 1 ? 0xffffu : 0u) | (valid >> (c * 2) & 2 ? 0xffff0000u : 0u);
                    const uint32_t old = at >= 32 ? 0xffffffffu : at > 0 ? (1u << at) - 1 : 0u;
                    const uint32_t fresh =
                        at >= 32 || at <= -64 ? 0u : at >= 0 ? (uint32_t)see << at : (uint32_t)(see >> -at);
                    const uint32_t vis = (pages & old) | fresh;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!(vis >> i & 1)) v[i] = 0xff800000u;
                };
                // 32 scores at a time, the next ones on their way
                uint32_t va[32], vb[32];
                float t0 = -INFINITY, t1 = -INFINITY;
                auto highest = [&](uint32_t(&v)[32], int c) {
                    if (masked) mask(v, c);
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        t0 = fmaxf(fmaxf(t0, __uint_as_float(v[i])), __uint_as_float(v[i + 1]));
                        t1 = fmaxf(fmaxf(t1, __uint_as_float(v[i + 2])), __uint_as_float(v[i + 3]));
                    }
                };
                tmem_start(va, st);
#pragma unroll 1
                for (int c = 0; c < KT / 32; c += 2) {
                    tmem_loaded(va);
                    tmem_start(vb, st + c * 32 + 32);
                    highest(va, c);
                    tmem_loaded(vb);
                    tmem_start(va, st + (c + 2 < KT / 32 ? c * 32 + 64 : 0));  // in the end the first ones again
                    highest(vb, c + 1);
                }
                const float top = fmaxf(t0, t1) * a.scale_log2;
                // the weights of the tile before are in the accumulator
                if (done) ok = __all_sync(0xffffffffu, wait(sm0 + L::odone + w * 8, done - 1));
                if (!ok) break;
                if (start) {
                    m = top;
                } else {
                    const bool grown = top > m + 8.0f;  // (always where m is -inf and top is not)
                    if (__any_sync(0xffffffffu, grown)) {
                        tc_after();
                        const float f = grown ? ex2(m - top) : 1.0f;
                        if (grown) m = top;
                        l *= f;
                        tmem_loaded(va);
#pragma unroll 1
                        for (int c = 0; c < (D + 31) / 32; ++c) {
                            tmem_load(vb, om + c * 32);
#pragma unroll
                            for (int i = 0; i < 32; ++i) vb[i] = __float_as_uint(__uint_as_float(vb[i]) * f);
                            tmem_store32(om + c * 32, vb);
                        }
                    }
                }
                const float base = m == -INFINITY ? 0.0f : m;
                float l0 = 0.0f, l1 = 0.0f;
                auto weights = [&](uint32_t(&v)[32], int c) {
                    if (masked) mask(v, c);
                    uint32_t p[16];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float e0 = ex2(fmaf(__uint_as_float(v[i]), a.scale_log2, -base)),
                                    e1 = ex2(fmaf(__uint_as_float(v[i + 1]), a.scale_log2, -base));
                        l0 += e0;
                        l1 += e1;
                        p[i / 2] = Num<T>::pack(e0, e1);
                    }
                    // weights of these 32 keys lie where scores were that are read already
                    tmem_store16(st + c * 16, p);
                };
                tmem_loaded(va);
#pragma unroll 1
                for (int c = 0; c < KT / 32; c += 2) {
                    tmem_start(vb, st + c * 32 + 32);
                    weights(va, c);
                    tmem_loaded(vb);
                    if (c + 2 < KT / 32) tmem_start(va, st + c * 32 + 64);
                    weights(vb, c + 1);
                    if (c + 2 < KT / 32) tmem_loaded(va);
                }
                l += l0 + l1;
                tmem_stored();
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sm0 + L::pready + w * 8);
                ++done;

                if (unit_ends || j + 1 == n) {
                    ok = __all_sync(0xffffffffu, wait(sm0 + L::odone + w * 8, done - 1));
                    if (!ok) break;
                    tc_after();
                    const bool whole = tile0 == 0 && unit_ends;
                    const int rr = w * 128 + row, rho = C.rt * RM + rr, t = rho / G, hd = C.h * G + rho - t * G;
                    float* const part = part_of<D, RM>(a, me, tile0 == 0 ? 1 : 0);
                    const float scale = whole ? (l > 0.0f || l != l ? 1.0f / l : 0.0f) : 1.0f;
                    const bool wild = wilds[units & 7] == units + 1;
                    // the new tokens of the tiles that this CTA had of the unit
                    const int x0 = max(0, tile0 * KT - C.len), x1 = min(C.T, (C.tile + 1) * KT - C.len);
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t v[32];
                        tmem_load(v, om + c * 32);
                        if (row < rows) {
                            if (wild) {
                                // values that are not finite, of the tokens that this row sees
                                for (int x = x0; x < x1; ++x) {
                                    if (!(see >> x & 1)) continue;
                                    const unsigned short* p = reinterpret_cast<const unsigned short*>(
                                        a.tok.v + ((long long)(C.lo + x) * a.tok.v_stride + C.h * D + c * 32) * 2);
#pragma unroll
                                    for (int i = 0; i < 32; ++i) {
                                        const float y = Num<T>::unpack(p[i]).x;
                                        if (y - y != 0.0f) v[i] = __float_as_uint(__uint_as_float(v[i]) + y);
                                    }
                                }
                            }
                            if (whole) {
                                uint4* const d = reinterpret_cast<uint4*>(
                                    a.out + ((C.lo + t) * a.out_stride + (long long)hd * D + c * 32) * 2);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    uint32_t q[4];
#pragma unroll
                                    for (int k = 0; k < 4; ++k)
                                        q[k] = Num<T>::pack(__uint_as_float(v[i * 8 + k * 2]) * scale,
                                                            __uint_as_float(v[i * 8 + k * 2 + 1]) * scale);
                                    d[i] = make_uint4(q[0], q[1], q[2], q[3]);
                                }
                            } else {
                                // four columns of all rows together: neighbouring threads' stores meet
                                uint4* const d = reinterpret_cast<uint4*>(part + RM * 2) + c * 8 * RM + rr;
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    d[i * RM] = make_uint4(v[i * 4], v[i * 4 + 1], v[i * 4 + 2], v[i * 4 + 3]);
                            }
                        }
                    }
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sm0 + L::ofree + w * 8);
                    if (row < rows) {
                        if (!whole) *reinterpret_cast<float2*>(part + rr * 2) = make_float2(m, l);
                        else if (a.lse) a.lse[(long long)(C.lo + t) * (H * G) + hd] = (m + log2f(l)) * LN2;
                    }
                    if (!whole) {
                        int first, last;
                        ax.sharers(C, first, last);
                        // (a row's parts come from warps of one number in their CTAs: no other warp is
                        // waited for)
                        int* const arrived = a.arrived + first * ATTEND_WORKERS_PER_SM + warp;
                        __threadfence();
                        __syncwarp();
                        int count = 0;
                        if (lane == 0) count = atomicAdd(arrived, 1);
                        count = __shfl_sync(0xffffffffu, count, 0);
                        if (count == last - first && lane == 0) *arrived = 0;
                        if (count == last - first && row < rows) {
                            __threadfence();
                            join_row<T, D, RM>(a, C, first, last, rr, t, hd);
                        }
                    }
                }
            }
            if (j + 1 < n) advance<KT, RM>(a, C, pre);
        }
    }
    if (!ok) *late = 1;
    tc_before();
    __syncthreads();
    tc_after();
    if (*late) {
        // products, boxes, loads and stores of tensor memory may be in flight
        if (warp == 4 * MT) {
            if (elected()) tc_commit(sm0 + L::over);
            __syncwarp();
            wait(sm0 + L::over, 0);
        } else if (warp > 4 * MT) {
            for (int i = max(0, filled - NB); i < filled; ++i) wait(sm0 + L::full + i % NB * 8, i / NB);
        } else {
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tmem_stored();
        }
        __syncthreads();
    }
    if (warp == 0) tmem_free(tm, 512);
}

// The driver's function that encodes tensor maps, looked up once.
typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                           const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                           CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder()
{
    static const Encode f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) !=
                cudaSuccess ||
            r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return (Encode)p;
    }();
    return f;
}

// Maps of the cache; rows 0 where its strides are more than a map holds (2^40 bytes): every
// tile is copied 16 bytes at a time then.
template <typename T, int D>
cudaError_t make_maps(const AttendArgs& a, int keys, Maps* m)
{
    m->rows = 0;
    const long long limit = 1ll << 39;
    if (a.kv.token_stride >= limit || a.kv.head_stride >= limit || a.kv.page_stride >= limit) return cudaSuccess;
    const Encode f = encoder();
    if (!f) return cudaErrorNotSupported;
    const int rows = a.kv.page < keys ? a.kv.page : keys;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)a.kv.page, (cuuint64_t)a.kv.kv_heads,
                                (cuuint64_t)a.kv.pages};
    const cuuint64_t strides[3] = {(cuuint64_t)a.kv.token_stride * 2, (cuuint64_t)a.kv.head_stride * 2,
                                   (cuuint64_t)a.kv.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
    const CUtensorMapDataType type =
        std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    for (int v = 0; v < 2; ++v)
        if (f(v ? &m->v : &m->k, type, 4, v ? a.kv.v : a.kv.k, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return cudaErrorInvalidValue;
    m->rows = rows;
    return cudaSuccess;
}

template <typename T, int D, int MT>
cudaError_t launch_tiles(const AttendArgs& a, int sms, cudaStream_t st)
{
    using L = Many<D, MT>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_attend_many<T, D, MT>>(most);
    if (e != cudaSuccess) return e;
    Maps maps;
    if ((e = make_maps<T, D>(a, L::KT, &maps)) != cudaSuccess) return e;
    k_attend_many<T, D, MT><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a, maps);
    return cudaGetLastError();
}

// One tile of 128 rows, or two, by the mean rows of a request's key head (64 requests of about 1,500
// tokens, 8 key heads of 128: 128 rows 143 us with one and 150 with two, 192 rows 262 and 180).
template <typename T, int D>
cudaError_t launch(const AttendArgs& a, int sms, cudaStream_t st)
{
    if constexpr (D < 256) {
        if ((long long)a.tok.n_tok * a.kv.group > 128ll * a.tok.n_req) return launch_tiles<T, D, 2>(a, sms, st);
    }
    return launch_tiles<T, D, 1>(a, sms, st);
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

cudaError_t launch_attend_many(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
