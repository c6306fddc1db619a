// aladdin_worker_attend: attention of a step's new tokens over the paged cache.
// Which kernel serves a call.
#include "worker.h"

namespace aladdin {

cudaError_t launch_attend(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    // By the mean rows of a request's key head: what one warp holds, or the tensor cores' tiles. (With
    // 4 rows the few-row kernel takes 74 us for 83,336 cached tokens; with 28 rows a warp-level kernel
    // of 32 rows a CTA took 82 us where the tensor cores' takes 48. Many-row tiles of 128 rows
    // with 4 of them in use leave most of the softmax's lanes idle.)
    if ((long long)a.tok.n_tok * a.kv.group <= 16ll * a.tok.n_req) return launch_attend_few(a, dtype, dim, sms, st);
    return launch_attend_many(a, dtype, dim, sms, st);
}

}  // namespace aladdin
