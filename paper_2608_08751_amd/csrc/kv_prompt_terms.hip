// The prompts' attention kernel with terms in its scores (kv_terms.h).
#include "kv_prompt_kernel.h"

namespace ivf {

hipError_t launch_kv_prompt_terms(const KvAttend &a, const KvTerms &x, hipStream_t s)
{
    return a.c.bf16 ? launch_prompt_dim<KvBf16>(a, x, s) : launch_prompt_dim<KvF16>(a, x, s);
}

}  // namespace ivf
