// aladdin_worker_rotate: rotary positions on the queries and keys of a step's new tokens.
//
// A pass over the data, 16 bytes a lane: what counts is bytes in flight. A warp takes one token
// and some of its heads' rows, forms the angles of its lanes' channels once and keeps several rows'
// loads in flight. A lane holds 8 channels of a row; the partners of the half layout come from the
// row's other half, which the same warp has just brought in. All loads of a row come
// before the first store to it, so that the outputs may be the inputs.
//
// Measured: pieces of prompts of 18,275 tokens, 32 heads of 96 channels: 41 us, 5.4 TB/s of 6.75 that a copy reaches; trees of
// 1,185 tokens, 72 heads of 128: 11 us, 3.9 TB/s, of it 3 until positions are known, which the rows' loads wait for although they
// need not (a token's rows in four times as many parts: 16, as each forms its
// angles).
#include "rope.cuh"

namespace aladdin {
namespace wk {
namespace {

constexpr int WARPS = 8, ROWS = 4;  // warps of a CTA, rows in flight of a lane

// The request of token t: the last one whose tokens begin at t or before, by all lanes together.
__device__ __forceinline__ int request_of(const int32_t* off, int n, int t, int lane)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, i = lo + lane * step;
        const int c = __popc(__ballot_sync(0xffffffffu, i < hi && off[i] <= t));
        if (c == 0) break;
        lo += (c - 1) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

template <typename T, int D, bool INTERLEAVED>
__global__ void __launch_bounds__(WARPS * 32) k_rotate(RotateArgs a, int parts)
{
    constexpr int CH = D / 8, RPW = 32 / CH;  // chunks of a row, rows of a warp at a time
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
    if (blockIdx.x == 0 && !a.pos) {
        // requests whose offsets make no sense, or that are trees of too many tokens
        for (int r = threadIdx.x; r < a.tok.n_req; r += WARPS * 32) {
            const int lo = a.tok.off[r], hi = a.tok.off[r + 1];
            if (lo < 0 || hi < lo || hi > a.tok.n_tok || (a.tok.parent && hi - lo > ALADDIN_TREE_MAX))
                atomicOr(a.err, WORKER_BAD_INPUT);
        }
    }
    const int t = (int)(unit / parts), part = (int)(unit - (long long)t * parts);
    if (t >= a.tok.n_tok) return;

    int p;
    if (a.pos) {
        p = a.pos[t];
    } else {
        const int r = request_of(a.tok.off, a.tok.n_req, t, lane);
        const int lo = a.tok.off[r], hi = a.tok.off[r + 1];
        if (lo < 0 || t < lo || t >= hi || hi > a.tok.n_tok) return;
        int depth = t - lo;
        if (a.tok.parent) {
            if (hi - lo > ALADDIN_TREE_MAX) return;
            // two tokens' parents a lane; one that is not an earlier token counts as none
            int up[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = e * 32 + lane;
                up[e] = i < hi - lo ? a.tok.parent[lo + i] : -1;
                if (up[e] < -1 || up[e] >= i) {
                    if (up[e] != -1) atomicOr(a.err, WORKER_BAD_INPUT);
                    up[e] = -1;
                }
            }
            int at = depth;
            depth = -1;
            while (at >= 0) {
                ++depth;
                const int x = __shfl_sync(0xffffffffu, up[0], at & 31), y = __shfl_sync(0xffffffffu, up[1], at & 31);
                at = at < 32 ? x : y;
            }
        }
        p = (int)((unsigned)(a.next ? a.next[r] : 0) + (unsigned)depth);
    }

    const int sub = lane / CH, ch = lane - sub * CH;
    Rotor<INTERLEAVED> rotor;
    rotor.load(a.rope, ch);
    rotor.at(p);
    const int nq = a.q_out ? a.q_heads : 0, rows = nq + (a.k_out ? a.kv_heads : 0);
    const int per = ((rows + parts - 1) / parts + RPW - 1) / RPW * RPW;
    const int row0 = part * per, row1 = min(rows, row0 + per);
    const char* const q = a.tok.q + (long long)t * a.tok.q_stride * 2;
    const char* const k = a.tok.k + (long long)t * a.tok.k_stride * 2;
    char* const qo = a.q_out + (long long)t * a.q_out_stride * 2;
    char* const ko = a.k_out + (long long)t * a.k_out_stride * 2;
    for (int row = row0; row < row1; row += RPW * ROWS) {
        uint4 x[ROWS], y[ROWS];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int h = row + i * RPW + sub;
            if (sub < RPW && h < row1) {
                const char* const src = h < nq ? q + (long long)h * D * 2 : k + (long long)(h - nq) * D * 2;
                x[i] = *reinterpret_cast<const uint4*>(src + ch * 16);
                if (!INTERLEAVED) y[i] = partners<T>(a.rope, src, ch);
            }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int h = row + i * RPW + sub;
            if (sub < RPW && h < row1) {
                float u[8], v[8];
                widen<T>(x[i], u);
                if (!INTERLEAVED) widen<T>(y[i], v);
                rotor.turn(u, v);
                char* const dst = h < nq ? qo + (long long)h * D * 2 : ko + (long long)(h - nq) * D * 2;
                *reinterpret_cast<uint4*>(dst + ch * 16) = narrow<T>(u);
            }
        }
    }
}

template <typename T, int D>
cudaError_t launch(const RotateArgs& a, int sms, cudaStream_t st)
{
    constexpr int RPW = 32 / (D / 8);
    const int rows = (a.q_out ? a.q_heads : 0) + (a.k_out ? a.kv_heads : 0);
    // a token's rows in as many parts as give every SM 8 warps, of ROWS loads a lane at least
    const long long want = ((long long)sms * 8 + a.tok.n_tok - 1) / a.tok.n_tok;
    const int most = (rows + RPW * ROWS - 1) / (RPW * ROWS), parts = (int)(want < most ? want : most);
    const long long ctas = ((long long)a.tok.n_tok * parts + WARPS - 1) / WARPS;
    if (ctas > 0x7fffffffll) return cudaErrorInvalidValue;
    if (a.rope.interleaved) k_rotate<T, D, true><<<(int)ctas, WARPS * 32, 0, st>>>(a, parts);
    else k_rotate<T, D, false><<<(int)ctas, WARPS * 32, 0, st>>>(a, parts);
    return cudaGetLastError();
}

template <typename T>
cudaError_t launch_dim(const RotateArgs& a, int dim, int sms, cudaStream_t st)
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

cudaError_t launch_rotate(const RotateArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    return dtype == ALADDIN_BF16 ? wk::launch_dim<__nv_bfloat16>(a, dim, sms, st)
                                 : wk::launch_dim<__half>(a, dim, sms, st);
}

}  // namespace aladdin
