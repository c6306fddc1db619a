// C ABI of a worker's decode step (include/aladdin.h): the worker object, the
// checks of its arguments and its workspaces. The kernels are in attend.cu,
// accept.cu, evict.cu and logprobs.cu.
#include <cmath>
#include <new>

#include "aladdin_host.h"
#include "worker.h"

using namespace aladdin;

struct aladdin_worker {
    int device = 0;
    int sms = 0;
    cudaStream_t st = nullptr;
    aladdin_worker_shape shape = {};
    int page_shift = 0;
    // one allocation: the error word and the counters (zero between calls), then
    // the partial results of attention units that CTAs share
    char* fixed = nullptr;
    unsigned* err = nullptr;
    int* done = nullptr;     // CTAs of an accept or evict call that have finished
    int* arrived = nullptr;  // [ATTEND_WORKERS_PER_SM * sms]
    int* moves = nullptr;    // [1024] evict: moves of (request, head) pairs,
    long long* bases = nullptr;            // [1024] where their lists start,
    unsigned long long* cursor = nullptr;  // and what is taken of the lists
    size_t ints = 0;         // bytes of the word and the counters
    float* part = nullptr;
    int32_t* lists = nullptr;  // evict (grow-only)
    size_t lists_n = 0;

    ~aladdin_worker()
    {
        if (fixed) cudaFree(fixed);
        if (lists) cudaFree(lists);
    }
};

namespace {

#define CK(x)                        \
    do {                             \
        cudaError_t e_ = (x);        \
        if (e_ != cudaSuccess) {     \
            cudaGetLastError();      \
            return ALADDIN_ERR_CUDA; \
        }                            \
    } while (0)

constexpr long long MAX_SLOTS = 0x7fffffffll - 65536;  // slots of a request; tile ends stay in an int

int check_shape(const aladdin_worker_shape* s)
{
    if (!s) return ALADDIN_ERR_ARG;
    if (s->dtype != ALADDIN_BF16 && s->dtype != ALADDIN_F16) return ALADDIN_ERR_ARG;
    if (s->kv_heads < 1 || s->q_heads < 1 || s->q_heads > 1024 || s->q_heads % s->kv_heads)
        return ALADDIN_ERR_ARG;
    const int d = s->head_dim, p = s->page_tokens;
    if (!(d == 64 || d == 96 || d == 128 || d == 256)) return ALADDIN_ERR_ARG;
    if (!(p == 16 || p == 32 || p == 64 || p == 128 || p == 256)) return ALADDIN_ERR_ARG;
    return ALADDIN_OK;
}

// Device memory of the worker's GPU, or managed memory, aligned to `align`.
bool on_device(const aladdin_worker* wk, const void* p, size_t align)
{
    if (reinterpret_cast<uintptr_t>(p) % align) return false;
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeDevice && a.device == wk->device);
}
bool all_on_device(const aladdin_worker* wk, std::initializer_list<const void*> ptrs, size_t align)
{
    for (const void* p : ptrs)
        if (p && !on_device(wk, p, align)) return false;
    return true;
}

bool stride_ok(int64_t s, int64_t least) { return s >= least && s % 8 == 0; }

int check_kv(const aladdin_worker* wk, const aladdin_kv* kv, KvDev* d)
{
    if (!kv || !kv->k || !kv->v || !kv->table || !kv->len) return ALADDIN_ERR_ARG;
    const aladdin_worker_shape& s = wk->shape;
    if (kv->pages < 1 || kv->table_width < 1 || kv->table_stride < kv->table_width ||
        (long long)kv->table_width * s.page_tokens > MAX_SLOTS)
        return ALADDIN_ERR_ARG;
    if (!stride_ok(kv->page_stride, 8) || !stride_ok(kv->head_stride, 8) ||
        !stride_ok(kv->token_stride, s.head_dim))
        return ALADDIN_ERR_ARG;
    if (!all_on_device(wk, {kv->k, kv->v}, 16) ||
        !all_on_device(wk, {kv->table, kv->len, kv->weight, kv->pos, kv->next}, 4))
        return ALADDIN_ERR_ARG;
    d->k = static_cast<char*>(kv->k);
    d->v = static_cast<char*>(kv->v);
    d->page_stride = kv->page_stride;
    d->head_stride = kv->head_stride;
    d->token_stride = kv->token_stride;
    d->table = kv->table;
    d->table_stride = kv->table_stride;
    d->len = kv->len;
    d->weight = kv->weight;
    d->pos = kv->pos;
    d->next = kv->next;
    d->pages = kv->pages;
    d->page = s.page_tokens;
    d->page_shift = wk->page_shift;
    d->kv_heads = s.kv_heads;
    d->group = s.q_heads / s.kv_heads;
    d->cap = (long long)kv->table_width * s.page_tokens;
    return ALADDIN_OK;
}

int check_tokens(const aladdin_worker* wk, const aladdin_tokens* t, bool need_q, TokDev* d)
{
    if (!t || t->n_req < 0 || t->n_req > ALADDIN_WORKER_MAX_REQUESTS || t->n_tok < 0) return ALADDIN_ERR_ARG;
    d->n_req = t->n_req;
    d->n_tok = t->n_tok;
    if (t->n_req == 0 || t->n_tok == 0) return ALADDIN_OK;  // nothing is read
    const aladdin_worker_shape& s = wk->shape;
    const int64_t kv = (int64_t)s.kv_heads * s.head_dim;
    if (!t->off || !t->k || !t->v || (need_q && !t->q)) return ALADDIN_ERR_ARG;
    if (!stride_ok(t->k_stride, kv) || !stride_ok(t->v_stride, kv) ||
        (t->q && !stride_ok(t->q_stride, (int64_t)s.q_heads * s.head_dim)))
        return ALADDIN_ERR_ARG;
    if (!all_on_device(wk, {t->off, t->parent}, 4) || !all_on_device(wk, {t->q, t->k, t->v}, 16))
        return ALADDIN_ERR_ARG;
    d->off = t->off;
    d->parent = t->parent;
    d->q = static_cast<const char*>(t->q);
    d->k = static_cast<const char*>(t->k);
    d->v = static_cast<const char*>(t->v);
    d->q_stride = t->q_stride;
    d->k_stride = t->k_stride;
    d->v_stride = t->v_stride;
    return ALADDIN_OK;
}

bool scale_ok(float s) { return std::isfinite(s) && s > 0.0f; }

constexpr double LOG2E_D = 1.4426950408889634;

}  // namespace

extern "C" {

int aladdin_worker_create(const aladdin_worker_shape* shape, void* cuda_stream, aladdin_worker** out)
try {
    if (!out) return ALADDIN_ERR_ARG;
    *out = nullptr;
    const int rc = check_shape(shape);
    if (rc) return rc;
    DevInfo d;
    CK(device_info(&d));
    aladdin_worker* wk = new (std::nothrow) aladdin_worker();
    if (!wk) return ALADDIN_ERR_NOMEM;
    wk->device = d.device;
    wk->sms = d.sms;
    wk->st = (cudaStream_t)cuda_stream;
    wk->shape = *shape;
    while ((1 << wk->page_shift) < shape->page_tokens) ++wk->page_shift;
    const size_t words = (size_t)(2 + ATTEND_WORKERS_PER_SM * d.sms + 1024);  // an even number
    const size_t ints = (words * 4 + (1024 + 1) * 8 + 255) / 256 * 256;
    wk->ints = ints;
    const size_t bytes = ints + attend_part_bytes(d.sms, shape->head_dim);
    cudaError_t e = cudaMalloc((void**)&wk->fixed, bytes);
    if (e == cudaSuccess) e = cudaMemsetAsync(wk->fixed, 0, ints, wk->st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(wk->st);
    if (e != cudaSuccess) {
        cudaGetLastError();
        delete wk;
        return e == cudaErrorMemoryAllocation ? ALADDIN_ERR_NOMEM : ALADDIN_ERR_CUDA;
    }
    wk->err = reinterpret_cast<unsigned*>(wk->fixed);
    wk->done = reinterpret_cast<int*>(wk->fixed) + 1;
    wk->arrived = wk->done + 1;
    wk->moves = wk->arrived + ATTEND_WORKERS_PER_SM * d.sms;
    wk->cursor = reinterpret_cast<unsigned long long*>(wk->fixed + words * 4);
    wk->bases = reinterpret_cast<long long*>(wk->cursor + 1);
    wk->part = reinterpret_cast<float*>(wk->fixed + ints);
    *out = wk;
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_destroy(aladdin_worker* wk)
try {
    if (!wk) return ALADDIN_ERR_ARG;
    cudaSetDevice(wk->device);
    cudaStreamSynchronize(wk->st);
    delete wk;
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_status(aladdin_worker* wk)
try {
    if (!wk) return ALADDIN_ERR_ARG;
    CK(cudaSetDevice(wk->device));
    unsigned err = 0;
    CK(cudaMemcpyAsync(&err, wk->err, sizeof(err), cudaMemcpyDeviceToHost, wk->st));
    CK(cudaStreamSynchronize(wk->st));
    if (err) CK(cudaMemsetAsync(wk->fixed, 0, wk->ints, wk->st));  // counters of a call that gave up, too
    if (err & WORKER_TIMEOUT) return ALADDIN_ERR_TIMEOUT;
    return err ? ALADDIN_ERR_STATE : ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_attend(aladdin_worker* wk, const aladdin_kv* kv, const aladdin_tokens* tok, float scale,
                          void* out, int64_t out_stride, float* lse)
try {
    if (!wk || !scale_ok(scale)) return ALADDIN_ERR_ARG;
    AttendArgs a = {};
    int rc = check_tokens(wk, tok, true, &a.tok);
    if (rc) return rc;
    if (a.tok.n_req == 0 || a.tok.n_tok == 0) return ALADDIN_OK;
    if ((rc = check_kv(wk, kv, &a.kv))) return rc;
    if (!out || !stride_ok(out_stride, (int64_t)wk->shape.q_heads * wk->shape.head_dim) ||
        !all_on_device(wk, {out}, 16) || !all_on_device(wk, {lse}, 4))
        return ALADDIN_ERR_ARG;
    CK(cudaSetDevice(wk->device));
    a.scale_log2 = (float)(scale * LOG2E_D);
    a.out = static_cast<char*>(out);
    a.out_stride = out_stride;
    a.lse = lse;
    a.part = wk->part;
    a.arrived = wk->arrived;
    a.err = wk->err;
    CK(launch_attend(a, wk->shape.dtype, wk->shape.head_dim, wk->sms, wk->st));
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_accept(aladdin_worker* wk, const aladdin_kv* kv, const aladdin_tokens* tok, float scale,
                          const float* lse, const int32_t* acc_off, const int32_t* acc, int32_t n_acc)
try {
    if (!wk || !kv) return ALADDIN_ERR_ARG;
    const bool weigh = lse != nullptr;
    if (weigh && !kv->weight) return ALADDIN_ERR_ARG;
    if (weigh && !scale_ok(scale)) return ALADDIN_ERR_ARG;
    AcceptArgs a = {};
    int rc = check_tokens(wk, tok, weigh, &a.tok);
    if (rc) return rc;
    if (a.tok.n_req == 0 || a.tok.n_tok == 0) return ALADDIN_OK;
    if ((rc = check_kv(wk, kv, &a.kv))) return rc;
    if (acc_off && n_acc < 0) return ALADDIN_ERR_ARG;
    if (acc_off && n_acc == 0) return ALADDIN_OK;
    if ((acc_off && !acc) || (!acc_off && acc) || !all_on_device(wk, {lse, acc_off, acc}, 4))
        return ALADDIN_ERR_ARG;
    CK(cudaSetDevice(wk->device));
    a.scale_log2 = (float)(scale * LOG2E_D);
    a.lse = lse;
    a.acc_off = acc_off;
    a.acc = acc;
    a.n_acc = acc_off ? n_acc : a.tok.n_tok;
    a.arrived = wk->done;
    a.err = wk->err;
    CK(launch_accept(a, wk->shape.dtype, wk->shape.head_dim, wk->sms, wk->st));
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_evict(aladdin_worker* wk, const aladdin_kv* kv, int32_t n_req, const int32_t* budget,
                         int32_t recent)
try {
    if (!wk || n_req < 0 || n_req > ALADDIN_WORKER_MAX_REQUESTS || recent < 0) return ALADDIN_ERR_ARG;
    if (n_req == 0) return ALADDIN_OK;
    EvictArgs a = {};
    const int rc = check_kv(wk, kv, &a.kv);
    if (rc) return rc;
    if (!kv->weight || !kv->pos || !kv->next || !budget || !all_on_device(wk, {budget}, 4))
        return ALADDIN_ERR_ARG;
    CK(cudaSetDevice(wk->device));
    const size_t slots = (size_t)kv->pages * wk->shape.kv_heads * wk->shape.page_tokens;
    if (slots > wk->lists_n) {
        CK(cudaStreamSynchronize(wk->st));
        if (wk->lists) cudaFree(wk->lists);
        wk->lists = nullptr;
        wk->lists_n = 0;
        const cudaError_t e = cudaMalloc((void**)&wk->lists, slots * sizeof(int32_t));
        if (e != cudaSuccess) {
            cudaGetLastError();
            return e == cudaErrorMemoryAllocation ? ALADDIN_ERR_NOMEM : ALADDIN_ERR_CUDA;
        }
        wk->lists_n = slots;
    }
    a.dim = wk->shape.head_dim;
    a.n_req = n_req;
    a.budget = budget;
    a.recent = recent;
    a.moves = wk->moves;
    a.bases = wk->bases;
    a.lists = wk->lists;
    a.lists_n = wk->lists_n;
    a.cursor = wk->cursor;
    a.arrived = wk->done;
    a.err = wk->err;
    CK(launch_evict(a, wk->sms, wk->st));
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

int aladdin_worker_logprobs(aladdin_worker* wk, int32_t logits_dtype, int32_t n, int32_t vocab,
                            const void* logits, int64_t stride, const int32_t* token, int32_t top,
                            float* logprob, float* entropy, int32_t* rank, int32_t* top_id,
                            float* top_logprob)
try {
    if (!wk || n < 0 || vocab < 1) return ALADDIN_ERR_ARG;
    if (logits_dtype != ALADDIN_BF16 && logits_dtype != ALADDIN_F16 && logits_dtype != ALADDIN_F32)
        return ALADDIN_ERR_ARG;
    if (top < 0 || top > ALADDIN_TOP_MAX || top > vocab) return ALADDIN_ERR_ARG;
    if (n == 0) return ALADDIN_OK;
    if (!logits || stride < vocab || ((logprob || rank) && !token)) return ALADDIN_ERR_ARG;
    if (n > 0x7fffffff / 8) return ALADDIN_ERR_ARG;  // CTAs of a launch
    if (!all_on_device(wk, {logits}, logits_dtype == ALADDIN_F32 ? 4 : 2) ||
        !all_on_device(wk, {token, logprob, entropy, rank, top_id, top_logprob}, 4))
        return ALADDIN_ERR_ARG;
    CK(cudaSetDevice(wk->device));
    LogprobArgs a = {};
    a.n = n;
    a.vocab = vocab;
    a.top = top_id || top_logprob ? top : 0;
    a.x = static_cast<const char*>(logits);
    a.stride = stride;
    a.token = token;
    a.logprob = logprob;
    a.entropy = entropy;
    a.rank = rank;
    a.top_id = top_id;
    a.top_logprob = top_logprob;
    a.err = wk->err;
    CK(launch_logprobs(a, logits_dtype, wk->sms, wk->st));
    return ALADDIN_OK;
} catch (...) {
    return ALADDIN_ERR_NOMEM;
}

}  // extern "C"
