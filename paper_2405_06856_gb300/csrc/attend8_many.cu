// aladdin_worker_attend8 where the rows of a (request, key head) are many (trees of drafted tokens, large groups): the
// products run on the fifth-generation tensor cores (tcgen05). See attend8.cuh for the operator.
//
// A CTA runs through a range of the axis of all key tiles, up to MT tiles of 128 rows at a time. Its warps have roles:
//   four warps for each row tile do the softmax, one thread a row. A thread brings its row of queries into shared memory
//   (256 channels: tensor memory), in half precision and scaled for it, reads a tile's scores once, and leaves the weights
//   in the place of the scores;
//   one thread issues the products: scores S = Q K' and out += P V, P from tensor memory;
//   seven warps convert, 16 keys or values at a time in turn: codes come by asynchronous copies a few of those ahead, each
//   lane's own, and go as half precision into a ring of shared memory, K0 V0 K1 V1 ..., in the 128-byte-swizzled layout of
//   the matrix descriptors. New tokens have a tile of their own; their values, and keys of bfloat16, are scaled by a power of
//   two for each.
// A row tile's scores have two places: the next ones are formed while the softmax works on those before. (Even and odd tiles of a
// single row tile by the two sets of softmax warps, with an accumulator each, took 5 to 10% longer: 64 requests of 1,500 tokens,
// 64 rows of 128 channels, 137 us for 124.) The accumulators stay in tensor memory; they are rescaled only when a row's
// maximum has grown by more than 2^8 over the one that its weights refer to.
//
// What bounds it: latency of a few warps a role. 16 warps share four schedulers, an instruction takes a warp 4 to 6 cycles,
// and each role has some 200 of them for a tile, so code is kept small as well: with products, tiles and units
// unrolled into the roles' loops (145 KB of code) a quarter of the warps' time went into fetching instructions. Measured,
// 24 requests of 60,854 cached tokens with trees of up to 64 tokens, 64 query and 8 key heads of 128 channels: 324 us so,
// 219 with a loop over units and one over tiles in each role, 205 with queries in shared memory and two places of
// scores, 195 with weights that refer to one maximum for each row, 521 TFLOP/s of 1,888 that a large product reaches; 37
// requests of 57,837 tokens with trees of up to 5, 28 and 4 heads of 96: 63 us, and 48 since seven warps convert in turn.
//
// New tokens' values that are not finite would reach rows that do not see them (0 times infinity): they are replaced by
// 0 in shared memory, and rows that do see them get them added at the end.
#include "attend8.cuh"
#include "tensor_dev.cuh"

namespace aladdin {
namespace wk {
namespace {

template <int D, int MT>
struct Many8 {
    static constexpr int KT = 64;                        // keys of a tile
    static constexpr int RM = 128 * MT;                  // rows of a unit
    static constexpr int HALVES = (D + 63) / 64;         // blocks of 64 channels
    static constexpr int TILE = HALVES * KT * 128;       // keys or values of a tile, half precision
    // the queries: 128 rows a row tile in shared memory, in tensor memory where 256 channels leave no room for that
    static constexpr bool QS = D < 256;
    static constexpr int QT = QS ? HALVES * 128 * 128 : 0;
    static constexpr int PLACES = MT == 2 ? 4 : 2;       // of scores: two for each row tile
    static constexpr int NB = D == 256 ? 4 : D == 64 ? 8 : 6;  // tiles of the ring (128 channels: 5, and 4 in flight, 213 us for 205)
    static constexpr int CONV = 7;                       // warps that convert, 16 keys or values at a time
    static constexpr int CPL = D / 32;                   // 16 codes each: what a lane has of those
    static constexpr int NF = D == 64 ? 4 : D == 96 ? 3 : 2;  // of them in flight, a warp
    static constexpr int RAW = CPL * 512 + 16;           // their codes, scales, whether their page is one of the pool
    static constexpr int q = NB * TILE;
    static constexpr int raw = q + MT * QT;
    static constexpr int bars = (raw + CONV * NF * RAW + 15) / 16 * 16;
    static constexpr int full = bars, empty = full + NB * 8, qready = empty + NB * 8, sready = qready + 16,
                         pready = sready + 32, odone = pready + 32, ofree = odone + 32, over = ofree + 16,
                         tmem = over + 8;
    static constexpr int wild = tmem + 8;                // 8 flags of units
    static constexpr int late = wild + 8 * 4;            // whether a wait ran out
    static constexpr int info = (late + 8 + 15) / 16 * 16;  // 8 tiles' Info
    static constexpr int scratch = info + 8 * (64 * 8 + 16);
    static constexpr int pre = scratch + 96 * 8;
    static constexpr int bytes(int n_req) { return pre + Axis8::ints(n_req) * 4; }
    static constexpr int WARPS = 4 * MT + 1 + CONV;      // softmax, products, conversions
    // columns of tensor memory: the scores' places, the accumulators, queries
    static constexpr int s0 = 0, o0 = PLACES * KT, q0 = o0 + MT * HALVES * 64;
    static_assert(q0 + (QS ? 0 : MT * (D / 2)) <= 512, "tensor memory");
    static_assert(info % 16 == 0 && scratch % 8 == 0 && TILE % 1024 == 0, "alignment");
};

// A tile's scales for the softmax: of blocks of 16 keys, or of each key where they are new.
struct Info {
    float k[64];    // factors of scores
    float lv[64];   // logarithms of the values' scales
    int valid[4];   // blocks of 16 keys on pages of the pool
};

// What a unit costs beside its tiles, in keys.
constexpr int UNIT_KEYS = 512;

// Room of the weights in half precision (attend8.cuh): a row's maxima may be 2^LAG behind.
constexpr float UP = 7.0f, LAG = 8.0f;

__device__ __forceinline__ uint64_t pair2(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float low2(uint64_t a) { return __uint_as_float((uint32_t)a); }
__device__ __forceinline__ float high2(uint64_t a) { return __uint_as_float((uint32_t)(a >> 32)); }

template <typename T, int D, int MT>
__global__ void __launch_bounds__(Many8<D, MT>::WARPS * 32, 1) k_attend8_many(Attend8Args a)
{
    using L = Many8<D, MT>;
    constexpr int KT = L::KT, RM = L::RM, NB = L::NB, NT = L::WARPS * 32;
    constexpr bool BF16 = !std::is_same<T, __half>::value;
    extern __shared__ __align__(1024) char sm[];
    const uint32_t sm0 = smem_addr(sm);
    // (tiles' scales, units' flags: the conversions run fewer than 8 tiles ahead of the softmax)
    Info* const infos = reinterpret_cast<Info*>(sm + L::info);
    volatile int* const wilds = reinterpret_cast<volatile int*>(sm + L::wild);
    volatile int* const late = reinterpret_cast<volatile int*>(sm + L::late);
    // (the warp's number by one lane: what follows from it is the same for all lanes, and the compiler sees it)
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int G = a.kv.group, H = a.kv.kv_heads;

    if (sm0 & 1023) {  // the operands' layout wants it
        if (tid == 0) atomicOr(a.err, WORKER_TIMEOUT);
        return;
    }
    Axis8 ax;
    if (!plan8<NT, KT, KT, RM>(a, ax, reinterpret_cast<int*>(sm + L::pre), reinterpret_cast<long long*>(sm + L::scratch),
                               (int)gridDim.x, UNIT_KEYS / KT, 1))
        return;
    const int me = blockIdx.x;
    if (me >= ax.workers) return;
    Cursor C;
    const int n = __shfl_sync(0xffffffffu, range8<KT, KT, RM>(a, ax, C, me), 0);
    if (n == 0) return;

    if (warp == 0) tmem_alloc(sm0 + L::tmem, 512);
    if (tid == 0) {
        for (int b = 0; b < NB; ++b) {
            mbar_init(sm0 + L::full + b * 8, 4);
            mbar_init(sm0 + L::empty + b * 8, 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(sm0 + L::qready + w * 8, 4);
            mbar_init(sm0 + L::pready + w * 16, 4);
            mbar_init(sm0 + L::pready + w * 16 + 8, 4);
            mbar_init(sm0 + L::odone + w * 16, 1);
            mbar_init(sm0 + L::odone + w * 16 + 8, 1);
            mbar_init(sm0 + L::ofree + w * 8, 4);
        }
        for (int w = 0; w < 4; ++w) mbar_init(sm0 + L::sready + w * 8, 1);
        mbar_init(sm0 + L::over, 1);
        for (int u = 0; u < 8; ++u) wilds[u] = 0;
        *late = 0;
        mbar_init_fence();
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tm = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t*>(sm + L::tmem), 0);

    // A wait that runs out is recorded and ends its warp's part; the others' waits run
    // out after it (no warps meet at a barrier without a limit before the end), and all meet at
    // the end, where what is in flight is waited for and tensor memory is freed. Whoever waits for a
    // barrier waits for all of its phases, or knows that the one before is over: a wait tells two apart, not three.
    auto wait = [&](uint32_t bar, int phase) -> bool {
        if (mbar_wait(bar, phase & 1)) return true;
        atomicOr(a.err, WORKER_TIMEOUT);
        return false;
    };
    // row tiles of the unit under u, of MT at most
    auto active = [&](const Cursor& u) { return MT == 2 && u.T * G - u.rt * RM > 128 ? 2 : 1; };
    // to the next unit
    auto next_unit = [&](Cursor& u) { next_unit8<KT, KT, RM>(a, ax, u); };
    // where the scores of row tile w and a unit's tile y lie
    auto place = [&](int w, int y) { return MT == 2 ? (y & 1) * 2 + w : y & 1; };
    bool ok = true;  // no wait of this warp ran out

    // Every role goes over the units of the range, and in each over its tiles; tile `done` + t of the range has places
    // 2 (done + t) % NB and the one behind it of the ring.
    if (warp >= 4 * MT + 1) {
        // ------------------------------------------------------------ conversions
        // Jobs of 16 keys or values of a tile, in turn to the warps: job 8 t + 4 part + g of tile t.
        const int cw = warp - (4 * MT + 1), rr = lane >> 2, cc = lane & 3;
        const int jobs = 8 * n;
        char* const raws = sm + L::raw + cw * (L::NF * L::RAW);
        // this lane's i-th chunk of 16 codes: its row of the 16, its first channel
        auto row_of = [&](int i) { return D == 96 && i == 2 ? lane >> 1 : i / (D == 96 ? 1 : L::HALVES) * 8 + rr; };
        auto channel_of = [&](int i) { return D == 96 ? (i == 2 ? 64 + (lane & 1) * 16 : cc * 16) : i % L::HALVES * 64 + cc * 16; };
        const long long row0 = row_of(0) * a.kv.token_stride + channel_of(0), eight = 8 * a.kv.token_stride;
        Cursor F = C;  // of the job that is fetched
        int fq = cw, ft = 0, fslot = 0, page = -1;
        // the page of job fq's keys, as the table has it
        auto find = [&]() {
            for (; ft < fq >> 3; ++ft) advance8<KT, KT, RM>(a, ax, F);
            const int key = F.tile * KT + (fq & 3) * 16;
            page = key < F.len ? a.kv.table[(long long)F.r * a.kv.table_stride + (key >> a.kv.page_shift)] : -1;
        };
        if (fq < jobs) find();
        // the codes of job fq, and with keys the scales of keys and values; then on to the next
        auto fetch = [&]() {
            if (fq < jobs) {
                const int key = F.tile * KT + (fq & 3) * 16, own = F.len - key;
                const bool values = fq & 4, valid = (unsigned)page < (unsigned)a.kv.pages;
                const uint32_t d = smem_addr(raws) + fslot * L::RAW;
                const int at = key & (a.kv.page - 1);
                const char* const src = (values ? a.kv.v : a.kv.k) +
                                        (valid ? page * a.kv.page_stride + F.h * a.kv.head_stride + at * a.kv.token_stride : 0);
                // (weights of 0 meet the codes of rows that hold no key: zeros)
                if (D != 96 && valid && own >= 16) {
                    const char* p = src + row0;
#pragma unroll
                    for (int i = 0; i < L::CPL; ++i) {
                        cp16(d + i * 512 + lane * 16, p + (i % L::HALVES) * 64, true);
                        if (i % L::HALVES == L::HALVES - 1) p += eight;
                    }
                } else {
#pragma unroll(D == 96 ? 3 : 1)  // (96 channels have no other way: rolled, 37 requests of trees up to 5 take 54 us for 48)
                    for (int i = 0; i < L::CPL; ++i) {
                        const bool in = valid && row_of(i) < own;
                        cp16(d + i * 512 + lane * 16, src + (in ? row_of(i) * a.kv.token_stride + channel_of(i) : 0), in);
                    }
                }
                if (!values && lane < 2) {
                    const long long e = valid ? ((long long)page * H + F.h) * a.scales.per_page + (at >> a.scales.block_shift) : 0;
                    cp4(d + L::CPL * 512 + lane * 4, (lane ? a.scales.v : a.scales.k) + e, valid);
                    if (lane == 0) *reinterpret_cast<int*>(raws + fslot * L::RAW + L::CPL * 512 + 8) = valid;
                    if (!valid && own > 0) atomicOr(a.err, WORKER_BAD_INPUT);
                }
                fq += L::CONV;
                if (fq < jobs) find();
                if (++fslot == L::NF) fslot = 0;
            }
            cp_commit();
        };
#pragma unroll 1
        for (int i = 0; i < L::NF - 1; ++i) fetch();
        Cursor u = C;
        int ut = 0, slot = 0, units = 0;
#pragma unroll 1
        for (int q = cw; q < jobs; q += L::CONV) {
            fetch();
            for (; ut < q >> 3; ++ut) {
                if (u.tile + 1 == u.c) ++units;
                advance8<KT, KT, RM>(a, ax, u);
            }
            const int part = q >> 2 & 1, g = q & 3;
            // A place is free when the half that lay there, NB halves before, has been read. That the phase before is over too (a
            // wait tells two phases apart, not three) follows from this warp's last job, at most two halves back: the half
            // NB before that one had been read then. Keys are read in their order, values in theirs, and the keys of
            // a tile not before the values `ahead` tiles back (below); in all cases the half 2 NB before this one is among
            // them. And no phase goes by before this warp's job is done.
            const int half = q >> 2;
            if (half >= NB) ok = wait(sm0 + L::empty + half % NB * 8, half / NB - 1);
            cp_wait<L::NF - 1>();
            __syncwarp();
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            char* const d = sm + half % NB * L::TILE + g * (16 * 128);
            Info& info = infos[ut & 7];
            if (u.tile * KT < u.len) {
                const char* const src = raws + slot * L::RAW;
                if (part == 0 && lane == 0) {
                    const float k = *reinterpret_cast<const float*>(src + L::CPL * 512), v = *reinterpret_cast<const float*>(src + L::CPL * 512 + 4);
                    const int valid = *reinterpret_cast<const int*>(src + L::CPL * 512 + 8);
                    // (0 too as it is: the products that it meets are finite, and -inf only where it is not used)
                    info.k[g] = finite_scale(k);
                    info.lv[g] = valid && u.tile * KT + g * 16 < u.len ? log_scale(v) : LOG_ZERO;
                    info.valid[g] = valid;
                }
#pragma unroll
                for (int i = 0; i < L::CPL; ++i) {
                    const uint4 c = *reinterpret_cast<const uint4*>(src + i * 512 + lane * 16);
                    const int row = row_of(i), p = channel_of(i) >> 3, e = row * 128 + (p >> 3) * (KT * 128);
                    *reinterpret_cast<uint4*>(d + e + (((p & 7) ^ (row & 7)) << 4)) =
                        make_uint4(half2_lo(c.x), half2_hi(c.x), half2_lo(c.y), half2_hi(c.y));
                    *reinterpret_cast<uint4*>(d + e + ((((p & 7) + 1) ^ (row & 7)) << 4)) =
                        make_uint4(half2_lo(c.z), half2_hi(c.z), half2_lo(c.w), half2_hi(c.w));
                }
            } else {
                // new tokens g * 16 ..
                constexpr int CH = D / 8;
                const char* const base = part ? a.tok.v : a.tok.k;
                const long long stride = (part ? a.tok.v_stride : a.tok.k_stride) * 2;
                int mine = 0;  // the largest exponent of this lane's row of the part
                {
                    // of two halves of a row a lane, of keys (bfloat16, if they are this job's) and values, not of infinities and NaN
                    const int row = g * 16 + (lane >> 1);
                    int most = 0;
#pragma unroll 1
                    for (int e = part; e < 2; ++e) {
                        if (!BF16 && e == 0) continue;
                        const uint4* const q = reinterpret_cast<const uint4*>(
                            (e ? a.tok.v + (u.lo + row) * a.tok.v_stride * 2 : a.tok.k + (u.lo + row) * a.tok.k_stride * 2) +
                            (u.h * D + (lane & 1) * (D / 2)) * 2);
                        most = 0;
                        if (row < u.T) {
#pragma unroll 4
                            for (int c = 0; c < D / 16; ++c) {
                                const uint4 v = q[c];
                                most = finite_exponent<T>(v.x, finite_exponent<T>(v.y, finite_exponent<T>(v.z, finite_exponent<T>(v.w, most))));
                            }
                        }
                        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                        if (e == part) mine = most;
                    }
                    if (part == 0 && (lane & 1) == 0) {  // (the softmax has the values' scales with the keys)
                        info.k[row] = BF16 ? half_back(mine) : 1.0f;
                        info.lv[row] = (float)(min(max(most, 15), 254) - 141);
                    }
                }
                bool w = false;
#pragma unroll 1
                for (int x = lane; x < 16 * CH; x += 32) {
                    const int row = x / CH, c = x - row * CH, t = g * 16 + row;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (t < u.T) v = *reinterpret_cast<const uint4*>(base + (u.lo + t) * stride + (u.h * D + c * 8) * 2);
                    if (part && (Num<T>::wild(v.x) || Num<T>::wild(v.y) || Num<T>::wild(v.z) || Num<T>::wild(v.w))) {
                        w = true;
                        v.x = Num<T>::tame(v.x), v.y = Num<T>::tame(v.y), v.z = Num<T>::tame(v.z), v.w = Num<T>::tame(v.w);
                    }
                    static_assert(16 * CH % 32 == 0, "all lanes take part");
                    const float f = half_factor(__shfl_sync(0xffffffffu, mine, row * 2));
                    if (BF16 || part) v = make_uint4(to_half<T>(v.x, f), to_half<T>(v.y, f), to_half<T>(v.z, f), to_half<T>(v.w, f));
                    *reinterpret_cast<uint4*>(d + (c >> 3) * (KT * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = v;
                }
                if (w) wilds[units & 7] = units + 1;
            }
            if (++slot == L::NF) slot = 0;
            fence_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm0 + L::full + half % NB * 8);
        }
        cp_wait<0>();
    } else if (warp == 4 * MT) {
        // ------------------------------------------------------------ products
        // Steps of a tile and a row tile each. A row tile's scores have two places in turn (place 2 (y % 2) + w of tile y and row
        // tile w; 256 channels: y % 2), and are formed when the products with values of the step two tiles before have been
        // started: a step's scores are formed while the softmax works on those before.
        constexpr uint32_t qk = product<__half>(KT, false), pv = product<__half>(D, true);
        if (elected()) {  // (one thread waits and issues)
            Cursor u = C;
            int asked[2] = {0, 0}, run[4] = {0, 0, 0, 0}, started[2] = {0, 0};
#pragma unroll 1
            for (int done = 0; done < n && ok;) {
                const int count = min(u.c - u.tile, n - done), two = active(u) == 2;
                const int steps = two ? 2 * count : count, ahead = two ? 4 : 2;
                if (two) ok = wait(sm0 + L::qready + 8, asked[1]++);
                ok = ok && wait(sm0 + L::qready, asked[0]++);
#pragma unroll 1
                for (int k = -ahead; k < steps; ++k) {
                    if (k >= 0) {
                        // out += P V of step k
                        const int w = two ? k & 1 : 0, y = two ? k >> 1 : k, v = 2 * (done + y) + 1, x2 = w * 2 + (y & 1);
                        ok = ok && wait(sm0 + L::pready + x2 * 8, x2 == 0 ? run[0]++ : x2 == 1 ? run[1]++ : x2 == 2 ? run[2]++ : run[3]++);
                        if (w == 0) ok = ok && wait(sm0 + L::full + v % NB * 8, v / NB);
                        if (y == 0) {
                            const int before = w ? started[1]++ : started[0]++;
                            if (before > 0) ok = ok && wait(sm0 + L::ofree + w * 8, before - 1);
                        }
                        if (!ok) break;
                        tc_after();
                        const uint32_t v0 = operand_lo(sm0 + v % NB * L::TILE, KT * 128), at = tm + L::s0 + place(w, y) * KT,
                                       o = tm + L::o0 + w * (L::HALVES * 64);
#pragma unroll
                        for (int x = 0; x < KT / 16; ++x)
                            tc_mma_ts(o, at + x * 8, whole(v0 + x * 2048 / 16, OPERAND_HI), pv, y > 0 || x > 0);
                        tc_commit(sm0 + L::odone + x2 * 8);
                        if (w == 1 || !two) tc_commit(sm0 + L::empty + v % NB * 8);
                    }
                    const int z = k + ahead;
                    if (z < steps) {
                        // S = Q K' of step z
                        const int w = two ? z & 1 : 0, y = two ? z >> 1 : z, i = 2 * (done + y);
                        if (w == 0) ok = ok && wait(sm0 + L::full + i % NB * 8, i / NB);
                        if (!ok) break;
                        tc_after();
                        const uint32_t k0 = operand_lo(sm0 + i % NB * L::TILE, 0), at = tm + L::s0 + place(w, y) * KT;
                        if constexpr (L::QS) {
                            const uint32_t q0 = operand_lo(sm0 + L::q + w * L::QT, 0);
#pragma unroll
                            for (int x = 0; x < D / 16; ++x)
                                tc_mma_ss(at, whole(q0 + ((x >> 2) * 128 * 128 + (x & 3) * 32) / 16, OPERAND_HI),
                                          whole(k0 + ((x >> 2) * KT * 128 + (x & 3) * 32) / 16, OPERAND_HI), qk, x > 0);
                        } else {
                            const uint32_t q0 = tm + L::q0;
#pragma unroll
                            for (int x = 0; x < D / 16; ++x)
                                tc_mma_ts(at, q0 + x * 8, whole(k0 + ((x >> 2) * KT * 128 + (x & 3) * 32) / 16, OPERAND_HI), qk, x > 0);
                        }
                        tc_commit(sm0 + L::sready + place(w, y) * 8);
                        if (w == 1 || !two) tc_commit(sm0 + L::empty + i % NB * 8);
                    }
                }
                done += count;
                if (done < n) next_unit(u);
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------ softmax
        const int w = warp >> 2, row = tid & 127, first_row = warp * 32;
        const uint32_t lanes = (uint32_t)(warp & 3) * 32u << 16, om = tm + lanes + L::o0 + w * (L::HALVES * 64);
        float factor = 0.0f;  // of this row's scores
        int weighed[2] = {0, 0};  // this row tile's steps so far, of even and odd tiles
        // this row's queries of the unit under u, 32 channels a time, into shared (tensor) memory
        auto queries = [&](const Cursor& u) {
            if (u.T * G - u.rt * RM <= w * 128) return;
            if (u.T * G - u.rt * RM <= first_row) {  // (none of this warp's rows: whatever lies there meets no other row)
                if (lane == 0) mbar_arrive(sm0 + L::qready + w * 8);
                return;
            }
            const int rho = u.rt * RM + w * 128 + row, t = rho / G;
            const bool live = rho < u.T * G;
            const uint4* const src = reinterpret_cast<const uint4*>(
                a.tok.q + ((u.lo + (live ? t : 0)) * a.tok.q_stride + (long long)(u.h * G + (live ? rho - t * G : 0)) * D) * 2);
            const uint4 none = make_uint4(0, 0, 0, 0);
            int top = 0;
            if constexpr (BF16) {
                uint32_t most = 0;
#pragma unroll 8
                for (int c = 0; c < D / 8; ++c) {
                    const uint4 v = live ? __ldg(src + c) : none;
                    most = largest2(largest2(largest2(largest2(most, v.x), v.y), v.z), v.w);
                }
                top = exponent<T>(most);
            }
            const float f = half_factor(top);
            factor = (BF16 ? half_back(top) : 1.0f) * a.scale_log2;
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
                uint32_t x[16];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 v = live ? __ldg(src + c * 4 + i) : none;
                    x[i * 4] = v.x, x[i * 4 + 1] = v.y, x[i * 4 + 2] = v.z, x[i * 4 + 3] = v.w;
                }
                if constexpr (BF16) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = to_half<T>(x[i], f);
                }
                if constexpr (L::QS) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int p = c * 4 + i;
                        *reinterpret_cast<uint4*>(sm + L::q + w * L::QT + (p >> 3) * (128 * 128) + row * 128 + (((p & 7) ^ (row & 7)) << 4)) =
                            make_uint4(x[i * 4], x[i * 4 + 1], x[i * 4 + 2], x[i * 4 + 3]);
                    }
                } else {
                    tmem_store16(tm + lanes + L::q0 + w * (D / 2) + c * 16, x);
                }
            }
            if constexpr (L::QS) {
                fence_async();
            } else {
                tmem_stored();
                tc_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(sm0 + L::qready + w * 8);
        };
        Cursor u = C;
        queries(u);
        int units = 0;
#pragma unroll 1
        for (int done = 0; done < n && ok;) {
            const int count = min(u.c - u.tile, n - done);
            const bool more = done + count < n;
            const int rows = u.T * G - u.rt * RM - w * 128;  // of the row tile
            const bool idle = rows <= (warp & 3) * 32;
            Cursor next = u;
            if (rows <= 0) {
                if (more) {
                    next_unit(next);
                    queries(next);
                }
            } else {
                const unsigned long long see = Ancestors(a, u, lane).of(row < rows ? (u.rt * RM + w * 128 + row) / G : 0);
                float M = -INFINITY, l = 0.0f, d = 0.0f;  // (attend8.cuh)
#pragma unroll 1
                for (int y = 0; y < count; ++y) {
                    const int s = place(w, y);
                    ok = __all_sync(0xffffffffu, wait(sm0 + L::sready + s * 8, y & 1 ? weighed[1] : weighed[0]));
                    if (!ok) break;
                    if (y & 1) ++weighed[1];
                    else ++weighed[0];
                    if (idle) {
                        if (lane == 0) mbar_arrive(sm0 + L::pready + (w * 2 + (y & 1)) * 8);
                        continue;
                    }
                    tc_after();
                    const uint32_t st = tm + lanes + L::s0 + s * KT;
                    uint32_t v[2][32];
                    tmem_start(v[0], st);
                    tmem_start(v[1], st + 32);
                    const Info& info = infos[(done + y) & 7];
                    const int own = u.len - (u.tile + y) * KT;  // cached keys from the tile's start
                    const float4 kf = *reinterpret_cast<const float4*>(info.k), lf = *reinterpret_cast<const float4*>(info.lv);
                    const int4 valid = *reinterpret_cast<const int4*>(info.valid);
                    const float lv[4] = {lf.x, lf.y, lf.z, lf.w}, hi = fmaxf(fmaxf(lf.x, lf.y), fmaxf(lf.z, lf.w)),
                                lo = fminf(fminf(lf.x, lf.y), fminf(lf.z, lf.w));
                    const bool all = own >= KT && (valid.x & valid.y & valid.z & valid.w);
                    if (y == 0 && all) d = hi;
                    const bool near = __all_sync(0xffffffffu, all && !(hi > d + FAR) && !(lo < d - FAR));
                    tmem_loaded(v[0]);
                    tmem_loaded(v[1]);
                    float grow = 1.0f;  // what the accumulator is multiplied by: the row's maximum grew by more than LAG
                    bool grown;
                    if (near) {
                        const float f[4] = {kf.x * factor, kf.y * factor, kf.z * factor, kf.w * factor};
                        float top = -INFINITY;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                            for (int i = 0; i < 16; i += 4) {
                                const uint32_t* const e = &v[x / 2][x % 2 * 16 + i];
                                t0 = fmaxf(fmaxf(t0, __uint_as_float(e[0])), __uint_as_float(e[1]));
                                t1 = fmaxf(fmaxf(t1, __uint_as_float(e[2])), __uint_as_float(e[3]));
                            }
                            top = fmaxf(top, __fmaf_ru(fmaxf(t0, t1), f[x], lv[x]));
                        }
                        grown = y == 0 || top - M > LAG;
                        if (grown) {
                            grow = ex2(M - top);
                            M = top;
                        }
                        const float base = M == -INFINITY ? 0.0f : M;
                        float sums = 0.0f;
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const float shift = __fadd_rd(lv[x] + UP, -base);
                            const uint64_t ff = pair2(__float_as_uint(f[x]), __float_as_uint(f[x])),
                                           bb = pair2(__float_as_uint(shift), __float_as_uint(shift));
                            uint64_t sum = 0;
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                const uint32_t* const e = &v[x / 2][x % 2 * 16 + i];
                                const uint64_t z = fma2(pair2(e[0], e[1]), ff, bb);
                                const float e0 = ex2(low2(z)), e1 = ex2(high2(z));
                                sum = add2(sum, pair2(__float_as_uint(e0), __float_as_uint(e1)));
                                v[x / 2][x % 2 * 8 + i / 2] = Num<__half>::pack(e0, e1);
                            }
                            sums += (low2(sum) + high2(sum)) * ex2(d - UP - lv[x]);
                        }
                        l = l * grow + sums;
                        // (the scores of all 64 keys have been read)
                        tmem_store16(st, *reinterpret_cast<const uint32_t(*)[16]>(&v[0][0]));
                        tmem_store16(st + 16, *reinterpret_cast<const uint32_t(*)[16]>(&v[1][0]));
                    } else {
                        // keys that are not seen or have scales of their own, or scales of very different size: scores are scaled in
                        // their place, those of a block whose scale is none NaN
                        const int step = own > 0 ? 0 : 1;
                        float m = M - d, most = -INFINITY, with = -INFINITY;
                        const float m0 = m == -INFINITY ? 0.0f : m;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t z[16];
                            tmem_load16(z, st + c * 16);
                            const int left = own - c * 16, at = step ? c * 16 : c;
                            const uint32_t vis = own <= 0 ? (uint32_t)(see >> (c * 16))
                                                 : !info.valid[c] ? 0u : left >= 16 ? 0xffffu : left > 0 ? (1u << left) - 1 : 0u;
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const float k = info.k[at + i * step] * factor, b = info.lv[at + i * step];
                                const float t = vis >> i & 1 ? fmaf(__uint_as_float(z[i]), k, b - b) : -INFINITY;
                                most = fmaxf(most, t);
                                with = fmaxf(with, (t - m0) + b);
                                z[i] = __float_as_uint(t);
                            }
                            tmem_store16(st + c * 16, z);
                        }
                        tmem_stored();
                        const float to = fmaxf(m, most), from = to == -INFINITY ? 0.0f : to;
                        with -= from - m0;
                        if (__any_sync(0xffffffffu, fabsf(from - m0) > 16384.0f)) {
                            // (next to such differences logarithms are lost: from the new maximum on)
                            with = -INFINITY;
#pragma unroll 1
                            for (int c = 0; c < 4; ++c) {
                                uint32_t z[16];
                                tmem_load16(z, st + c * 16);
                                const int at = step ? c * 16 : c;
#pragma unroll
                                for (int i = 0; i < 16; ++i) with = fmaxf(with, (__uint_as_float(z[i]) - from) + info.lv[at + i * step]);
                            }
                        }
                        grown = y == 0 || most - m > LAG || with - (M - from) > LAG;  // (always where M is -inf and top is not)
                        if (grown) {
                            const float by = m - from, next = fmaxf(fmaxf(d + by, with), 2 * LOG_ZERO);
                            grow = ex2(by + (d - next));
                            l *= ex2(by);
                            M = to == -INFINITY ? to : __fadd_ru(to, next);
                            d = next;
                            m = to;
                        }
                        const float base = m == -INFINITY ? 0.0f : m;
                        // weights lie where scores were that have been read
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t z[16], p[8];
                            tmem_load16(z, st + c * 16);
                            const int at = step ? c * 16 : c;
#pragma unroll
                            for (int i = 0; i < 16; i += 2) {
                                float e[2];
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const float t = __uint_as_float(z[i + k]) - base;
                                    l += ex2(t);
                                    e[k] = ex2(t + (info.lv[at + (i + k) * step] - d + UP));
                                }
                                p[i / 2] = Num<__half>::pack(e[0], e[1]);
                            }
                            tmem_store8(st + c * 8, p);
                        }
                    }
                    if (y > 0 && __any_sync(0xffffffffu, grown)) {
                        // the weights of the tile before are in the accumulator (those of the one before it were when
                        // these scores were formed)
                        ok = __all_sync(0xffffffffu, wait(sm0 + L::odone + (w * 2 + (y + 1 & 1)) * 8, (y & 1 ? weighed[0] : weighed[1]) - 1));
                        if (!ok) break;
                        tc_after();
#pragma unroll 1
                        for (int c = 0; c < D / 16; ++c) {
                            uint32_t o[16];
                            tmem_load16(o, om + c * 16);
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * grow);
                            tmem_store16(om + c * 16, o);
                        }
                    }
                    tmem_stored();
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(sm0 + L::pready + (w * 2 + (y & 1)) * 8);
                }
                if (!ok) break;
                // the next unit's queries, while the last products run: this unit's scores are done
                if (more) {
                    next_unit(next);
                    queries(next);
                }
                ok = __all_sync(0xffffffffu, wait(sm0 + L::odone + (w * 2 + (count - 1 & 1)) * 8, (count & 1 ? weighed[0] : weighed[1]) - 1));
                if (!ok) break;
                if (idle) {
                    if (lane == 0) mbar_arrive(sm0 + L::ofree + w * 8);
                    done += count;
                    ++units;
                    u = next;
                    continue;
                }
                tc_after();
                const float m = M - d;
                const bool whole = u.tile == 0 && count == u.c;
                const int rr = w * 128 + row, rho = u.rt * RM + rr, t = rho / G, hd = u.h * G + rho - t * G;
                float* const part = part_of<D, RM>(a, me, u.tile == 0 ? 1 : 0);
                float2 unit = unit_of(d);
                unit.y *= (whole ? (l > 0.0f || l != l ? 1.0f / l : 0.0f) : 1.0f) * ex2(-UP);
                const bool wild = wilds[units & 7] == units + 1;
#pragma unroll 1
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t o[32];
                    tmem_load(o, om + c * 32);
#pragma unroll
                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * unit.y * unit.x);
                    if (row < rows) {
                        if (wild && !(whole && l == 0.0f)) {
                            // values that are not finite, of the tokens that this row sees, whatever their weight
                            for (int x = 0; x < u.T; ++x) {
                                if (!(see >> x & 1)) continue;
                                const unsigned short* p = reinterpret_cast<const unsigned short*>(
                                    a.tok.v + ((long long)(u.lo + x) * a.tok.v_stride + u.h * D + c * 32) * 2);
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const float y = Num<T>::unpack(p[i]).x;
                                    if (y - y != 0.0f) o[i] = __float_as_uint(__uint_as_float(o[i]) + y);
                                }
                            }
                        }
                        if (whole) {
                            uint4* const d = reinterpret_cast<uint4*>(
                                a.out + ((u.lo + t) * a.out_stride + (long long)hd * D + c * 32) * 2);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                uint32_t q[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    q[k] = Num<T>::pack(__uint_as_float(o[i * 8 + k * 2]), __uint_as_float(o[i * 8 + k * 2 + 1]));
                                d[i] = make_uint4(q[0], q[1], q[2], q[3]);
                            }
                        } else {
                            // four columns of all rows together: neighbouring threads' stores meet
                            uint4* const d = reinterpret_cast<uint4*>(part + RM * 2) + c * 8 * RM + rr;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                d[i * RM] = make_uint4(o[i * 4], o[i * 4 + 1], o[i * 4 + 2], o[i * 4 + 3]);
                        }
                    }
                }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sm0 + L::ofree + w * 8);
                if (row < rows) {
                    if (!whole) *reinterpret_cast<float2*>(part + rr * 2) = make_float2(m, wild ? -l : l);
                    else if (a.lse) a.lse[(long long)(u.lo + t) * (H * G) + hd] = (m + log2f(l)) * LN2;
                }
                if (!whole) {
                    int first, last;
                    ax.sharers(u, first, last);
                    // (a row's parts come from warps of one number in their CTAs: no other warp is
                    // waited for)
                    int* const arrived = a.arrived + first * ATTEND_WORKERS_PER_SM + warp;
                    __threadfence();
                    __syncwarp();
                    int seen = 0;
                    if (lane == 0) seen = atomicAdd(arrived, 1);
                    seen = __shfl_sync(0xffffffffu, seen, 0);
                    if (seen == last - first && lane == 0) *arrived = 0;
                    if (seen == last - first && row < rows) {
                        __threadfence();
                        join_row<T, D, RM>(a, u, first, last, rr, t, hd);
                    }
                }
            }
            done += count;
            ++units;
            u = next;
        }
    }
    if (!ok) *late = 1;
    tc_before();
    __syncthreads();
    tc_after();
    if (*late) {
        // products, loads and stores of tensor memory may be in flight
        if (warp == 4 * MT) {
            if (elected()) tc_commit(sm0 + L::over);
            __syncwarp();
            wait(sm0 + L::over, 0);
        } else if (warp < 4 * MT) {
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            tmem_stored();
        }
        __syncthreads();
    }
    if (warp == 0) tmem_free(tm, 512);
}

template <typename T, int D>
cudaError_t launch(const Attend8Args& a, int sms, cudaStream_t st)
{
    constexpr int MT = D < 256 ? 2 : 1;
    using L = Many8<D, MT>;
    constexpr int most = L::bytes(ALADDIN_WORKER_MAX_REQUESTS);
    static_assert(most <= 227 * 1024, "shared memory of a CTA");
    cudaError_t e = allow_smem<k_attend8_many<T, D, MT>>(most);
    if (e != cudaSuccess) return e;
    k_attend8_many<T, D, MT><<<sms, L::WARPS * 32, L::bytes(a.tok.n_req), st>>>(a);
    return cudaGetLastError();
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

cudaError_t launch_attend8_many(const Attend8Args& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
