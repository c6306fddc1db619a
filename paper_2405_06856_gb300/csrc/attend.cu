// aladdin_worker_attend: attention of a step's new tokens over the paged cache.
// Which kernel serves a call.
#include "worker.h"

namespace aladdin {

cudaError_t launch_attend(const AttendArgs& a, int dtype, int dim, int sms, cudaStream_t st)
{
    // By the mean rows of a request's key head: what one warp holds, or the tensor cores' tiles. Measured, few
    // rows' kernel then the many rows', 64 requests of about 1,500 tokens, 8 key heads of 128 channels: 8 rows
    // 104 and 113 us, 12 rows 121 and 113, 16 rows 125 and 115, 20 rows 162 and 115; of about 2,500 tokens,
    // 64 channels: 8 rows 94 and 137, 16 rows 113 and 150, 24 rows 137 and 150, 48 rows 170 and 154. A few
    // large requests among many small ones take the small ones' kernel, which goes over their cache
    // once for each of their row tiles, and the other way round: 127 decodes with a chain of 64 tokens over 6,000
    // take 141 us, 90 and 53 apart; 100 decodes with 24 trees of 40 tokens 250 us, the trees alone 117. And
    // the kernel that a request meets, and so the rounding, depends on the others of its call.
    if ((long long)a.tok.n_tok * a.kv.group <= 16ll * a.tok.n_req) return launch_attend_few(a, dtype, dim, sms, st);
    return launch_attend_many(a, dtype, dim, sms, st);
}

}  // namespace aladdin
