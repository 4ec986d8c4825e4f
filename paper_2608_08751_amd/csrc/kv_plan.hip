// Block tables and slots of a paged cache from request lengths.
//
// Request b holds cached[b] tokens and brings added[b]: with o = ceil(cached /
// bs) and n = ceil((cached + added) / bs) it takes n - o blocks, the ones of
// rank before(b) ... in the list of free blocks, before(b) the exclusive sum of
// n - o. Token i of it stands at position cached + i in block (position / bs) of
// its table row. One launch: every workgroup forms both prefix sums in LDS (8
// bytes a request to read, from L2) and then takes its share of the tokens,
// each of which finds its request by bisection, and of the table rows. What it
// writes, 16 bytes a token and the tables, bounds a large call; a small one is
// one launch long: 16 requests of one token 4.8 us, 2,000 requests with 300
// prompts of up to 700 tokens (149,000 tokens, 4.5 MB) 11.7 us.
// Up to 2,048 requests 256 threads hold 8 each; with 1,024 threads of 16, which
// 16,384 requests need, these two calls take 8.2 and 13.0 us.
#include "kv.h"

#include <algorithm>

namespace ivf {
namespace {

__device__ __forceinline__ int64_t blocks_of(int64_t tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }

// THREADS threads hold PER requests each.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void kv_plan_kernel(
    const int32_t *__restrict__ cached, const int32_t *__restrict__ added, int B, int shift, int32_t *table, int cols,
    const int32_t *__restrict__ free_blocks, int64_t n_free, int64_t T, int32_t *__restrict__ start,
    int64_t *__restrict__ slots, int32_t *__restrict__ request, int32_t *__restrict__ position,
    int64_t *__restrict__ info)
{
    // sums are 64-bit and stored clamped: tokens at T (< 2^31), ranks at INT32_MAX (none that far is free)
    __shared__ int32_t first[THREADS * PER];   // token prefix
    __shared__ int32_t before[THREADS * PER];  // block prefix
    __shared__ int64_t wave_sum[2][THREADS / 64];
    __shared__ int beyond;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t bs_cols = (int64_t)cols << shift;
    if (tid == 0) beyond = 0;

    int64_t tok = 0, blk = 0;
    int over = 0;
    int64_t tk[PER], bk[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = tid * PER + i;
        const int64_t c = b < B ? max(cached[b], 0) : 0, a = b < B ? max(added[b], 0) : 0;
        tk[i] = tok;
        bk[i] = blk;
        tok += a;
        blk += min(blocks_of(c + a, shift), (int64_t)cols) - min(blocks_of(c, shift), (int64_t)cols);
        over += c + a > bs_cols;
    }
    int64_t ti = tok, bi = blk;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t t = __shfl_up(ti, d), u = __shfl_up(bi, d);
        if (lane >= d) ti += t, bi += u;
    }
    if (lane == 63) wave_sum[0][wave] = ti, wave_sum[1][wave] = bi;
    __syncthreads();
    if (over) atomicAdd(&beyond, over);
    int64_t tb = ti - tok, bb = bi - blk, tall = 0, ball = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) tb += wave_sum[0][w], bb += wave_sum[1][w];
        tall += wave_sum[0][w], ball += wave_sum[1][w];
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        first[tid * PER + i] = (int32_t)min(tb + tk[i], T);
        before[tid * PER + i] = (int32_t)min(bb + bk[i], (int64_t)INT32_MAX);
    }
    __syncthreads();
    const int64_t total = min(tall, T);
    if (blockIdx.x == 0) {
        for (int b = tid; b < B; b += THREADS) start[b] = first[b];
        if (tid == 0) {
            if (start) start[B] = (int32_t)total;
            if (info) {
                info[0] = tall;
                info[1] = ball;
                info[2] = min(ball, n_free);
                info[3] = beyond;
            }
        }
    }

    // tokens
    for (int64_t t = (int64_t)blockIdx.x * THREADS + tid; t < T; t += (int64_t)gridDim.x * THREADS) {
        int b = -1;
        int64_t slot = -1, pos = -1;
        if (t < total) {
            int lo = 0, hi = B;  // the last request with first <= t (later ones of the same start are not empty)
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first[mid] <= t) lo = mid;
                else hi = mid;
            }
            b = lo;
            const int64_t c = max(cached[b], 0);
            pos = c + (t - first[b]);
            if (pos < bs_cols) {
                const int64_t j = pos >> shift, o = blocks_of(c, shift);
                int32_t id = -1;
                if (j < o) {
                    id = table[(int64_t)b * cols + j];
                } else {
                    const int64_t r = before[b] + (j - o);
                    if (r < n_free) id = free_blocks[r];
                }
                if (id >= 0) slot = ((int64_t)id << shift) + (pos & ((1 << shift) - 1));
            }
            pos = min(pos, (int64_t)INT32_MAX);
        }
        if (slots) slots[t] = slot;  // null in an empty batch only
        if (request) request[t] = b;
        if (position) position[t] = (int32_t)pos;
    }

    // table rows, a wave each: columns from the first new block on
    for (int b = blockIdx.x * (THREADS / 64) + wave; b < B; b += gridDim.x * (THREADS / 64)) {
        const int64_t c = max(cached[b], 0), a = max(added[b], 0);
        const int64_t o = blocks_of(c, shift), n = blocks_of(c + a, shift);
        for (int64_t j = o + lane; j < cols; j += 64) {
            const int64_t r = before[b] + (j - o);
            table[(int64_t)b * cols + j] = j < n && r < n_free ? free_blocks[r] : -1;
        }
    }
}

}  // namespace

hipError_t launch_kv_plan(const int32_t *cached, const int32_t *added, int B, int shift, int32_t *table, int cols,
                          const int32_t *free_blocks, int64_t n_free, int64_t T, int32_t *start, int64_t *slots,
                          int32_t *request, int32_t *position, int64_t *info, int num_cus, hipStream_t s)
{
    const int threads = B <= 2048 ? 256 : 1024;
    int64_t grid = (T + threads - 1) / threads;
    grid = std::max<int64_t>(grid, (B + threads / 64 - 1) / (threads / 64));
    grid = std::max<int64_t>(1, std::min<int64_t>(grid, (int64_t)num_cus * (B <= 2048 ? 2 : 1)));
    if (B <= 2048)
        hipLaunchKernelGGL((kv_plan_kernel<256, 8>), dim3((unsigned)grid), dim3(256), 0, s, cached, added, B, shift,
                           table, cols, free_blocks, n_free, T, start, slots, request, position, info);
    else
        hipLaunchKernelGGL((kv_plan_kernel<1024, 16>), dim3((unsigned)grid), dim3(1024), 0, s, cached, added, B, shift,
                           table, cols, free_blocks, n_free, T, start, slots, request, position, info);
    return hipGetLastError();
}

}  // namespace ivf
