// aladdin_worker_attend: attention of a step's new tokens over the paged cache.
// Which kernel serves a call.
#include "worker.h"

namespace aladdin {

cudaError_t launch_attend(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    // by the mean rows of a request's key head: what one warp holds, or the tensor cores' tiles
    if ((long long)a.tok.n_tok * a.kv.group <= 16ll * a.tok.n_req) return launch_attend_few(a, dtype, dim, sms, st);
    return launch_attend_many(a, dtype, dim, sms, st);
}

}  // namespace aladdin
