// aladdin_worker_attend8: attention of a step's new tokens over the paged cache of 8 bits.
// Which kernel serves a call.
#include "worker.h"

namespace aladdin {

cudaError_t launch_attend8(const Attend8Args& a, int dtype, int dim, int sms, cudaStream_t st)
{
    // By the mean rows of a request's key head.
    if ((long long)a.tok.n_tok * a.kv.group <= 16ll * a.tok.n_req) return launch_attend8_few(a, dtype, dim, sms, st);
    return launch_attend8_many(a, dtype, dim, sms, st);
}

}  // namespace aladdin
