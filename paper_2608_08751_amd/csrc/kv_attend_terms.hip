// The single-token attention kernel with terms in its scores (kv_terms.h).
#include "kv_attend_kernel.h"

namespace ivf {

hipError_t launch_kv_tokens_terms(const KvAttend &a, const KvTerms &x, int64_t groups, hipStream_t s)
{
    return a.c.bf16 ? launch_tokens_dim<KvBf16>(a, x, groups, s) : launch_tokens_dim<KvF16>(a, x, groups, s);
}

}  // namespace ivf
