// Sampling a token for each row of logits (sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ivf {

constexpr int64_t kSampleMaxVocab = 1 << 20;  // weights of 2^43 at most: their sums stay below 2^63
constexpr int kSampleMaxParts = 8;               // workgroups that share a row
constexpr int kSampleList = 2048;

struct Sample {
    const void *logits;
    int dt;          // an ivf_dtype: fp32, f16 or bf16
    int64_t stride;  // of rows, in elements
    int64_t T;
    int V;
    // [T] each; all but uniform may be null
    const float *uniform, *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p;
    int32_t *token;
    float *logprob;  // may be null
    int parts, per;  // workgroups a row; groups of eight logits a wave
};

// What the launches of a call that shares rows out hand on (workspace), for T rows of `parts` parts.
struct SampleShare {
    float2 *ends;                // [T][parts] largest and least logit
    int *first;                  // [T][parts] where the largest stands
    unsigned long long *range;   // [T][parts * 16] sums of weights
    uint32_t *cursor;            // [T][2]
    // with top_k or top_p
    void *decision;              // [T]
    unsigned long long *list;    // [T][kSampleList]
    uint32_t *count;             // [T][parts][bins]
    unsigned long long *sum;
};

// Workgroups that share a row; 0: one a row, in one launch. Bytes of the workspace (0 with it), and with a base what lies where.
int sample_parts(int64_t T, int64_t V, int num_cus);
size_t sample_workspace(int64_t T, int parts, bool cuts, char *base, SampleShare *x);
hipError_t launch_sample(Sample a, int parts, const SampleShare &x, hipStream_t s);

}  // namespace ivf
