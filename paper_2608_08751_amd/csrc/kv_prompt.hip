// Attention of many query rows per request over the 4-bit cache (kv_prompt_kernel.h).
#include "kv_prompt_kernel.h"

namespace ivf {

int kv_prompt_rows(int dim) { return dim <= 128 ? PromptShape<128>::rows : PromptShape<256>::rows; }

int kv_prompt_resident(int dim) { return dim <= 128 ? 8 / PromptShape<128>::waves : 1; }

hipError_t launch_kv_prompt(const KvAttend &a, hipStream_t s)
{
    return a.c.bf16 ? launch_prompt_dim<KvBf16>(a, KvNoTerms(), s) : launch_prompt_dim<KvF16>(a, KvNoTerms(), s);
}

}  // namespace ivf
