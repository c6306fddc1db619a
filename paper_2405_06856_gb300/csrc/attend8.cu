// aladdin_worker_attend8: attention of a step's new tokens over the paged cache of 8 bits.
// Which kernel serves a call.
#include "worker.h"

namespace aladdin {

cudaError_t launch_attend8(const Attend8Args& a, int dtype, int dim, int sms, cudaStream_t st)
{
    // By the mean rows of a request's key head: the few rows' kernel has 8 or 16 of them in a warp and goes over the keys
    // once for each; the many rows' kernel takes about as long for any number up to 128. Measured, few rows' kernel then the
    // many rows': 64 requests of about 1,500 tokens, 8 key heads of 128 channels: 8 rows 52 and 114 us, 16 rows 84 and 114,
    // 24 rows 112 and 116, 32 rows 123 and 116; of about 2,500 tokens, 64 channels: 16 rows 71 and 144, 32 rows 127 and 144;
    // 37 of 1,500, 4 heads of 96: 7 rows 26 and 42, 14 rows 57 and 40, 28 rows 50 and 40; 64 of 1,000, 256 channels:
    // 8 rows 77 and 129, 16 rows 125 and 137, 20 rows 190 and 141. As in the attention over 16 bits, the kernel that a
    // request meets depends on the others of its call.
    const int most = dim == 64 ? 32 : dim == 96 ? 12 : dim == 128 ? 24 : 16;
    if ((long long)a.tok.n_tok * a.kv.group <= (long long)most * a.tok.n_req) return launch_attend8_few(a, dtype, dim, sms, st);
    return launch_attend8_many(a, dtype, dim, sms, st);
}

}  // namespace aladdin
