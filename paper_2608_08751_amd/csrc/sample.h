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

hipError_t launch_sample(Sample a, hipStream_t s);

}  // namespace ivf
