// Internals of the worker step's operators, shared by their translation units
// (worker.cu: the C ABI; attend.cu, accept.cu, evict.cu, logprobs.cu: kernels).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/aladdin.h"

namespace aladdin {

// Raises Kern's dynamic shared-memory limit to `bytes` (the same on every call
// for one kernel), once per device ordinal < 64.
template <auto Kern>
cudaError_t allow_smem(int bytes)
{
    static std::atomic<unsigned long long> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
    if (bit && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(Kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && bit) done.fetch_or(bit, std::memory_order_acq_rel);
    return e;
}

// Key heads, group size and page of a worker, and its paged cache as the
// kernels see it (aladdin_kv, checked).
struct KvDev {
    char* k;
    char* v;
    long long page_stride, head_stride, token_stride;  // elements
    const int32_t* table;
    int32_t* len;
    float* weight;
    int32_t* pos;
    int32_t* next;
    long long table_stride; // entries from a table row to the next
    int pages;              // pages of the pool
    int page, page_shift;   // tokens of a page
    int kv_heads, group;
    long long cap;          // table width * page: tokens that a request can hold
};

struct TokDev {
    int n_req, n_tok;
    const int32_t* off;
    const int32_t* parent;
    const char* q;
    const char* k;
    const char* v;
    long long q_stride, k_stride, v_stride;  // elements from token to token
};

// Bits of a worker's error word.
constexpr unsigned WORKER_BAD_INPUT = 1u;
constexpr unsigned WORKER_TIMEOUT = 4u;  // a wait for a copy ran out

struct AttendArgs {
    KvDev kv;
    TokDev tok;
    float scale_log2;       // scale * log2(e)
    char* out;
    long long out_stride;
    float* lse;
    float* part;            // split units' partial results, 2 slots a worker
    int* arrived;           // split units' arrivals, one a worker, zero between calls
    unsigned* err;
};

struct AcceptArgs {
    KvDev kv;
    TokDev tok;
    float scale_log2;
    const float* lse;
    const int32_t* acc_off;
    const int32_t* acc;
    int n_acc;
    int* arrived;           // finished CTAs, zero between calls
    unsigned* err;
};

struct EvictArgs {
    KvDev kv;
    int dim;
    int n_req;
    const int32_t* budget;
    int recent;
    int* moves;             // of the (request, head) pairs, where clusters serve them,
    long long* bases;       // and where their lists start
    int32_t* lists;         // holes, then movers of each pair in a place of its own
    unsigned long long lists_n;  // entries: as many as the pool has slots
    unsigned long long* cursor;  // entries that are taken, zero between calls
    int* arrived;
    unsigned* err;
};

struct LogprobArgs {
    int n, vocab, top;
    const char* x;
    long long stride;       // elements from row to row
    const int32_t* token;
    float* logprob;
    float* entropy;
    int32_t* rank;
    int32_t* top_id;
    float* top_logprob;
    unsigned* err;
};

// Workers of an attention launch on one SM, at most (warps, or a CTA's row tiles), and
// the bytes of AttendArgs::part: two units of each SM's CTA of at most 256 rows (128
// of 256 channels), or of at most 8 warps of 16 rows.
constexpr int ATTEND_WORKERS_PER_SM = 8;
inline size_t attend_part_bytes(int sms, int dim)
{
    return (size_t)sms * 2 * (dim < 256 ? 256 : 128) * (dim + 2) * sizeof(float);
}
cudaError_t launch_attend_few(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st);
cudaError_t launch_attend_many(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st);
cudaError_t launch_attend(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st);
cudaError_t launch_accept(const AcceptArgs& a, int dtype, int dim, int sms, cudaStream_t st);
cudaError_t launch_evict(const EvictArgs& a, int sms, cudaStream_t st);
cudaError_t launch_logprobs(const LogprobArgs& a, int dtype, int sms, cudaStream_t st);

}  // namespace aladdin
