// The paged 4-bit key/value cache: its layout and the launch parameters of the
// kernels that build its tables (kv_plan.hip), write and read it
// (kv_cache.hip), select blocks (kv_select.hip) and attend (kv_attend.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ivf {

constexpr int kKvMaxRequests = 16384;  // of one plan: their prefix sums lie in LDS
constexpr int kKvMaxSelectCols = 32768;  // block scores of a row lie in LDS
constexpr int kKvMaxCount = 4096;
constexpr int kKvMaxUnits = 1024;  // whose key ranges are shared out evenly (prefix sums in LDS)

struct KvCache {
    uint8_t *rec;
    int8_t *summary;
    float *weight;
    int64_t blocks;
    int bs;        // tokens per block, 1 << shift
    int shift;
    int heads;
    int dim;
    bool bf16;     // else f16
    __host__ __device__ size_t rec_bytes() const { return (size_t)bs * dim / 16 * 17; }
    // offsets inside a record
    __host__ __device__ int v_codes() const { return bs * (dim / 2); }
    __host__ __device__ int k_scales() const { return bs * dim; }
    __host__ __device__ int v_scales() const { return bs * dim + bs * (dim / 32); }
};

// Query rows by strides, in elements.
struct KvRows {
    const void *p;
    int64_t ts, hs;
};

hipError_t launch_kv_plan(const int32_t *cached, const int32_t *added, int B, int shift, int32_t *table, int cols,
                          const int32_t *free_blocks, int64_t n_free, int64_t T, int32_t *start, int64_t *slots,
                          int32_t *request, int32_t *position, int64_t *info, int num_cus, hipStream_t s);

// Threads of the launch that writes or reads T tokens and sums or reads n blocks (at most: 2048 / dim
// tokens or blocks take 256 threads a head).
inline int64_t kv_cache_threads(const KvCache &c, int64_t T, int64_t n)
{
    const int64_t at_once = 2048 / c.dim;
    return ((T + at_once - 1) / at_once + (n + at_once - 1) / at_once) * c.heads * 256;
}
// Appending up to this many tokens takes one launch (kv_cache.hip).
constexpr int64_t kKvFewTokens = 512;

hipError_t launch_kv_append(const KvCache &c, KvRows k, KvRows v, const int64_t *slots, int64_t T, hipStream_t s);
hipError_t launch_kv_read(const KvCache &c, const int64_t *slots, int64_t T, void *k, void *v, const int32_t *blocks,
                          int64_t n, float *mean, hipStream_t s);

struct KvSelect {
    KvCache c;
    KvRows q;
    int group;  // query heads per key/value head
    int64_t T;
    const int32_t *request, *position, *table;
    int64_t B;
    int cols;
    int first, last, count;
    int32_t *out;
};
hipError_t launch_kv_select(const KvSelect &a, hipStream_t s);

struct KvAttend {
    KvCache c;
    KvRows q;
    int group;
    int64_t T;
    const int32_t *start, *request, *position, *table;
    int64_t B;
    int cols;
    const int32_t *blocks;  // selected blocks, or null
    int count;
    float scale;      // |scale| log2(e), above 0
    uint32_t q_flip;  // flips the signs of two query channels where the scale is negative
    void *out;
    float *lse;
    // a request with at most small_rows rows (tokens * group) is the single-token
    // kernel's, any other the prompt kernel's
    int64_t small_rows;
    // Long key ranges are cut into parts, whose results lie here: sums
    // [row][dim] and (reference, sum of exponentials) [row]. With blocks, and of the
    // prompt kernel, every row has `splits` parts, [token][query head][split]. Of the
    // single-token kernel without blocks `splits` workgroups a head share all units'
    // keys; rows are [head][slot][unit_rows], and unit_parts holds each unit's first
    // slot and number of parts (1: written to `out` at once). splits 1: no parts.
    int splits;
    int unit_size;  // rows of a unit: 8 or 16
    int team;       // waves that share a unit: 8, 4 or 1
    int unit_rows;  // rows that a unit has room for in part[]
    int per_unit;   // units of a request, or of a token with `blocks`
    int units;
    int slots;
    float *part;
    float2 *part_ml;
    int2 *unit_parts;
};

// Which kernels take a call, in how many parts, and what those need.
struct KvAttendPlan {
    bool tokens, prompt;
    int64_t small_rows;
    int per_unit, unit_size, unit_rows, team;
    int64_t units, slots;
    int token_splits, prompt_splits;
    int64_t token_groups;  // workgroups of the single-token kernel per head
    // workspace, and where part_ml and unit_parts begin in it
    size_t token_bytes, token_ml, token_parts, prompt_bytes, prompt_ml;
};
KvAttendPlan kv_attend_plan(const KvCache &c, int group, int64_t T, int64_t B, int64_t cols, int64_t count,
                            int64_t longest, int num_cus);
hipError_t launch_kv_tokens(const KvAttend &a, int64_t groups, hipStream_t s);
// joins the parts of prompts and of the single-token kernel's calls; either may be null
hipError_t launch_kv_combine(const KvAttend *prompts, const KvAttend *units, hipStream_t s);

int kv_prompt_rows(int dim);      // rows of a workgroup
int kv_prompt_resident(int dim);  // workgroups that a CU holds
hipError_t launch_kv_prompt(const KvAttend &a, hipStream_t s);

}  // namespace ivf
