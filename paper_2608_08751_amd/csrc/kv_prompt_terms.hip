// The prompts' attention kernel with terms in its scores (kv_terms.h).
#include "kv_prompt_kernel.h"

namespace ivf {

namespace {

template <bool CAP, bool BIAS> hipError_t launch_terms(const KvAttend &a, const KvTerms &x, hipStream_t s)
{
    const KvTermsOf<CAP, BIAS> terms = {x};
    return a.c.bf16 ? launch_prompt_dim<KvBf16>(a, terms, s) : launch_prompt_dim<KvF16>(a, terms, s);
}

}  // namespace

hipError_t launch_kv_prompt_terms(const KvAttend &a, const KvTerms &x, hipStream_t s)
{
    if (x.cap != 0.f) return x.slopes ? launch_terms<true, true>(a, x, s) : launch_terms<true, false>(a, x, s);
    return x.slopes ? launch_terms<false, true>(a, x, s) : launch_terms<false, false>(a, x, s);
}

}  // namespace ivf
