// Blocks of the paged cache that requests share, give back and move: forks,
// the list of free blocks, compaction, and the copies that these ask for.
//
// The tables are the only state. A block is in use where a table row names it within
// its request's length, so that a fork shares blocks by naming them, a request ends
// by its length becoming 0, and no count of uses has to be kept right. What a fork copies is the
// last block alone, where that is partly filled: full blocks never change.
#include "kv.h"

#include <algorithm>

namespace ivf {
namespace {

__device__ __forceinline__ int64_t blocks_of(int64_t tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }
// Entries of a row that a request of n tokens holds.
__device__ __forceinline__ int held(int32_t n, int shift, int cols)
{
    return (int)min(blocks_of(max(n, 0), shift), (int64_t)cols);
}

// The sum of x over a workgroup's threads before this one; *all: over all of them.
template <int THREADS> __device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t *all)
{
    __shared__ uint32_t sums[THREADS / 64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t up = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(up, d);
        if (lane >= d) up += y;
    }
    __syncthreads();  // sums may still be read
    if (lane == 63) sums[wave] = up;
    __syncthreads();
    uint32_t before = up - x, total = 0;
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += sums[w];
        total += sums[w];
    }
    *all = total;
    return before;
}

// Columns of a table row that a wave takes at a time.
constexpr int kChunk = 256;

// Fork i makes row child[i] a copy of row parent[i]. It counts where both rows exist and
// differ, no later fork names the child, and no such fork has the child as its
// parent: rows that are read are then not written. Every workgroup works the whole
// list out in LDS (12 bytes a fork from L2) and takes its share of the rows.
template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void kv_fork_kernel(const int32_t *__restrict__ parent,
                                                          const int32_t *__restrict__ child, int n, int32_t *cached,
                                                          int B, int shift, int32_t *table, int cols,
                                                          const int32_t *__restrict__ free_blocks, int64_t n_free,
                                                          int32_t *__restrict__ source, int32_t *__restrict__ to,
                                                          int64_t *__restrict__ info)
{
    __shared__ int32_t last[THREADS * PER];  // the last fork that names a row as its child
    __shared__ uint32_t read[THREADS * PER / 32];  // rows that are parents
    __shared__ int32_t rank[THREADS * PER];  // of the block that a fork takes; -1: none, -2: the fork does not count
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // with info the last workgroup counts the blocks that are taken, entries of -1 are none; the others take the rows
    const unsigned groups = gridDim.x - (info != nullptr);
    int32_t id[PER];
    if (blockIdx.x == groups) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = tid + k * THREADS;
            id[k] = i < n && i < n_free ? free_blocks[i] : -1;
        }
    }
    for (int b = tid; b < B; b += THREADS) last[b] = -1;
    for (int b = tid; b * 32 < B; b += THREADS) read[b] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
        const int p = parent[i], c = child[i];
        if (p >= 0 && p < B && c >= 0 && c < B && p != c) {
            atomicMax(&last[c], i);
            atomicOr(&read[p >> 5], 1u << (p & 31));
        }
    }
    __syncthreads();
    const int per = (n + THREADS - 1) / THREADS;
    uint32_t takes = 0;
#pragma unroll 1
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i >= n) break;
        const int p = parent[i], c = child[i];
        int r = -2;
        if (p >= 0 && p < B && c >= 0 && c < B && p != c && last[c] == i && !(read[c >> 5] >> (c & 31) & 1)) {
            r = -1;
            const int32_t m = max(cached[p], 0);
            const int64_t used = blocks_of(m, shift);
            if ((m & ((1 << shift) - 1)) && used <= cols && table[(int64_t)p * cols + used - 1] >= 0) r = (int)takes++;
        }
        rank[i] = r;
    }
    uint32_t all;
    const uint32_t before = sum_before<THREADS>(takes, &all);
    for (int k = 0; k < per; ++k) {
        const int i = tid * per + k;
        if (i < n && rank[i] >= 0) rank[i] += (int)before;
    }
    __syncthreads();
    if (blockIdx.x == groups) {
        uint32_t got = 0, taken;
#pragma unroll
        for (int k = 0; k < PER; ++k) got += tid + k * THREADS < (int)all && id[k] >= 0;
        sum_before<THREADS>(got, &taken);
        if (tid == 0) {
            info[0] = all;
            info[1] = taken;
        }
        return;
    }
    const uint32_t chunks = (uint32_t)(cols + kChunk - 1) / kChunk;
    const int64_t units = (int64_t)n * chunks;
    for (int64_t u = (int64_t)blockIdx.x * (THREADS / 64) + wave; u < units; u += (int64_t)groups * (THREADS / 64)) {
        const int i = (int)((uint64_t)u / chunks), r = rank[i];
        const int j0 = (int)((uint64_t)u % chunks) * kChunk;
        if (r == -2) {
            if (j0 == 0 && lane == 0) source[i] = to[i] = -1;
            continue;
        }
        const int p = parent[i], c = child[i];
        const int32_t m = cached[p];
        const int used = held(m, shift, cols);
        const int32_t *from = table + (int64_t)p * cols;
        int32_t *row = table + (int64_t)c * cols;
        const int32_t fresh = r >= 0 && r < n_free ? free_blocks[r] : -1;
#pragma unroll
        for (int k = 0; k < kChunk / 64; ++k) {
            const int j = j0 + 64 * k + lane;
            if (j < cols) row[j] = j >= used ? -1 : r >= 0 && j == used - 1 ? fresh : from[j];
        }
        if (j0 == 0 && lane == 0) {
            cached[c] = m;
            source[i] = fresh >= 0 ? from[used - 1] : -1;
            to[i] = fresh >= 0 ? fresh : -1;
        }
    }
}

// Copies pairs of blocks, kPiece bytes of records a workgroup at a time (the last
// of a pair with the summaries). Bound by memory, read + written: 139 MB 26 us, 276 MB 56 us, 5.3 and 4.9 TB/s.
constexpr int kPiece = 16384;
__global__ __launch_bounds__(256) void kv_copy_kernel(KvCache dst, KvCache src, const int32_t *__restrict__ to,
                                                      const int32_t *__restrict__ source, int64_t units, uint32_t pieces)
{
    const size_t bytes = src.rec_bytes() * src.heads;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t i = (int64_t)((uint64_t)u / pieces);
        const uint32_t piece = (uint32_t)((uint64_t)u % pieces);
        const int a = source[i], b = to[i];
        if (a < 0 || a >= src.blocks || b < 0 || b >= dst.blocks) continue;
        const uint8_t *from = src.rec + (size_t)a * bytes;
        uint8_t *at = dst.rec + (size_t)b * bytes;
        const size_t begin = (size_t)piece * kPiece + 16 * threadIdx.x;
        uint4 x[kPiece / 4096];
#pragma unroll
        for (int k = 0; k < kPiece / 4096; ++k)
            if (begin + 4096 * k < bytes) x[k] = *(const uint4 *)(from + begin + 4096 * k);
#pragma unroll
        for (int k = 0; k < kPiece / 4096; ++k)
            if (begin + 4096 * k < bytes) *(uint4 *)(at + begin + 4096 * k) = x[k];
        if (piece == pieces - 1) {
            const size_t means = (size_t)src.heads * src.dim;
            for (size_t o = 16 * threadIdx.x; o < means; o += 4096)
                *(uint4 *)(dst.summary + b * means + o) = *(const uint4 *)(src.summary + a * means + o);
            for (int h = threadIdx.x; h < src.heads; h += 256)
                dst.weight[(size_t)b * src.heads + h] = src.weight[(size_t)a * src.heads + h];
        }
    }
}

// Calls f(row, column) for the entries that requests hold: waves take chunks of rows.
template <int THREADS, typename F> __device__ __forceinline__ void for_entries(const KvReclaim &a, F f)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t chunks = (uint32_t)(a.cols + kChunk - 1) / kChunk;
    const int64_t units = a.B * chunks;
    for (int64_t u = (int64_t)blockIdx.x * (THREADS / 64) + wave; u < units; u += (int64_t)gridDim.x * (THREADS / 64)) {
        const int64_t b = (int64_t)((uint64_t)u / chunks);
        const int j0 = (int)((uint64_t)u % chunks) * kChunk, n = held(a.cached[b], a.shift, a.cols);
#pragma unroll
        for (int k = 0; k < kChunk / 64; ++k) {
            const int j = j0 + 64 * k + lane;
            if (j < n) f(b * a.cols + j);
        }
    }
}

// The same in one workgroup for few entries (kKvFewBlocks at most): a thread an entry, eight loads each at a time, none
// of which waits for another.
template <int THREADS, typename F> __device__ __forceinline__ void for_few_entries(const KvReclaim &a, F f)
{
    constexpr int U = 8;
    const uint32_t all = (uint32_t)(a.B * a.cols), cols = (uint32_t)a.cols;
    for (uint32_t e0 = threadIdx.x; e0 < all; e0 += U * THREADS) {
        int32_t id[U], n[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t e = min(e0 + k * THREADS, all - 1);
            id[k] = a.table[e];
            n[k] = a.cached[e / cols];
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const uint32_t e = e0 + k * THREADS;
            if (e < all && (int)(e % cols) < held(n[k], a.shift, a.cols)) f(e, id[k]);
        }
    }
}

// With U blocks in use, the used ones at U and beyond (as many as there are holes below U)
// move into the holes, both in ascending order, the first `made` of them.
struct Moves {
    int64_t used;   // U
    int64_t below;  // of these, below U
    int64_t made;
    // Block id, in use or not, with `before` used ones below it.
    template <typename Source, typename To, typename Free>
    __device__ __forceinline__ void place(int64_t id, bool in_use, int64_t before, Source source, To to, Free free) const
    {
        const bool low = id < used;
        const int64_t hole = low ? id - before : used - below;  // holes before it
        const int64_t high = low ? 0 : before - below;          // blocks that would move, before it
        if (low && !in_use && hole < made) to(hole, id);
        if (!low && in_use && high < made) source(high, id);
        const bool stays = in_use ? low || high >= made : low && hole < made;
        if (!stays) free(id - (before + min(hole, made) - min(high, made)), id);
    }
};

// A set of blocks as bits, in LDS with the counts of the words before each.
struct Bits {
    const uint32_t *word, *before;
    __device__ __forceinline__ bool has(int64_t id) const { return word[id >> 5] >> (id & 31) & 1; }
    __device__ __forceinline__ int64_t below(int64_t id) const
    {
        return (int64_t)before[id >> 5] + __popc(word[id >> 5] & ((1u << (id & 31)) - 1));
    }
};

// The whole call in one workgroup: up to kKvFewBlocks blocks.
constexpr int kOne = 1024;
__global__ __launch_bounds__(kOne) void kv_reclaim_one_kernel(KvReclaim a)
{
    constexpr int kWords = kKvFewBlocks / 32;
    __shared__ uint32_t word[kWords + 1], before[kWords + 1];
    const int tid = threadIdx.x;
    const int words = (int)(a.blocks + 31) / 32;
    for (int w = tid; w <= words; w += kOne) word[w] = 0;
    __syncthreads();
    for_few_entries<kOne>(a, [&](uint32_t, int id) {
        if (id >= 0 && id < a.blocks) atomicOr(&word[id >> 5], 1u << (id & 31));
    });
    __syncthreads();
    static_assert(kWords <= kOne, "a thread's word");
    uint32_t all;
    const uint32_t below = sum_before<kOne>(tid < words ? __popc(word[tid]) : 0, &all);
    if (tid < words) before[tid] = below;
    if (tid == 0) before[words] = all;
    __syncthreads();
    const Bits bits = {word, before};
    Moves m;
    m.used = all;
    m.below = bits.below(all);
    m.made = min(m.used - m.below, a.moves);
    for (int64_t id = tid; id < a.blocks; id += kOne)
        m.place(id, bits.has(id), bits.below(id), [&](int64_t i, int64_t x) { a.source[i] = (int32_t)x; },
                [&](int64_t i, int64_t x) { a.to[i] = (int32_t)x; },
                [&](int64_t i, int64_t x) { if (a.free) a.free[i] = (int32_t)x; });
    for (int64_t i = m.made + tid; i < a.moves; i += kOne) a.source[i] = a.to[i] = -1;
    if (a.free)
        for (int64_t i = a.blocks - m.used + tid; i < a.blocks; i += kOne) a.free[i] = -1;
    if (a.info && tid == 0) {
        a.info[0] = m.used;
        a.info[1] = m.made;
        a.info[2] = a.blocks - m.used;
    }
    if (m.made == 0) return;
    __syncthreads();  // to[] is read
    for_few_entries<kOne>(a, [&](uint32_t e, int id) {
        if (id < m.used || id >= a.blocks) return;
        const int64_t r = bits.below(id) - m.below;
        if (r < m.made) a.table[e] = a.to[r];
    });
}

// The same in several launches, with the bits in the workspace: clear, mark, count
// (used blocks of every kSpan words), list, and, with moves, the tables.
constexpr int kSpan = 2048, kShare = 256;  // words of a count, and of a workgroup that lists
__global__ __launch_bounds__(256) void kv_clear_kernel(uint32_t *bits, int64_t words)
{
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < words; w += (int64_t)gridDim.x * 256) bits[w] = 0;
}

__global__ __launch_bounds__(256) void kv_mark_kernel(KvReclaim a)
{
    for_entries<256>(a, [&](int64_t e) {
        const int id = a.table[e];
        if (id >= 0 && id < a.blocks) atomicOr(&a.bits[id >> 5], 1u << (id & 31));
    });
}

__global__ __launch_bounds__(256) void kv_count_kernel(KvReclaim a, int64_t words)
{
    uint32_t n = 0, all;
    for (int k = 0; k < kSpan / 256; ++k) {
        const int64_t w = (int64_t)blockIdx.x * kSpan + 256 * k + threadIdx.x;
        if (w < words) n += __popc(a.bits[w]);
    }
    sum_before<256>(n, &all);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = all;
}

// Blocks in use below word w of the bits: counts of whole spans, then words. All threads call it.
__device__ int64_t used_below(const KvReclaim &a, int64_t w)
{
    const int64_t span = w / kSpan;
    uint32_t n = 0, all;  // fewer than 2^31 blocks
    for (int64_t i = threadIdx.x; i < span; i += 256) n += a.counts[i];
    for (int64_t i = span * kSpan + threadIdx.x; i < w; i += 256) n += __popc(a.bits[i]);
    sum_before<256>(n, &all);
    return all;
}

__global__ __launch_bounds__(256) void kv_list_kernel(KvReclaim a, int64_t words)
{
    __shared__ uint32_t word[kShare], before[kShare];
    const int tid = threadIdx.x;
    const int64_t w0 = (int64_t)blockIdx.x * kShare, id0 = w0 * 32;
    Moves m;
    m.used = used_below(a, words);
    m.below = used_below(a, m.used >> 5);
    if (m.used >> 5 < words) m.below += __popc(a.bits[m.used >> 5] & ((1u << (m.used & 31)) - 1));
    m.made = min(m.used - m.below, a.moves);
    const int64_t base = used_below(a, w0);
    uint32_t all;
    word[tid] = w0 + tid < words ? a.bits[w0 + tid] : 0;
    before[tid] = sum_before<256>(__popc(word[tid]), &all);
    __syncthreads();
    const Bits bits = {word, before};
    for (int i = tid; i < 32 * kShare; i += 256) {
        const int64_t id = id0 + i;
        if (id >= a.blocks) break;
        m.place(id, bits.has(i), base + bits.below(i),
                [&](int64_t r, int64_t x) {
                    a.source[r] = (int32_t)x;
                    a.rank[x] = (int32_t)r;
                },
                [&](int64_t r, int64_t x) { a.to[r] = (int32_t)x; },
                [&](int64_t r, int64_t x) { if (a.free) a.free[r] = (int32_t)x; });
        if (a.moves && bits.has(i) && id >= m.used && base + bits.below(i) - m.below >= m.made) a.rank[id] = -1;
        if (a.free && id >= a.blocks - m.used) a.free[id] = -1;
    }
    for (int64_t i = m.made + (int64_t)blockIdx.x * 256 + tid; i < a.moves; i += (int64_t)gridDim.x * 256)
        a.source[i] = a.to[i] = -1;
    if (blockIdx.x == 0 && tid == 0) {
        a.counts[(words + kSpan - 1) / kSpan] = (uint32_t)m.used;  // for the tables
        if (a.info) {
            a.info[0] = m.used;
            a.info[1] = m.made;
            a.info[2] = a.blocks - m.used;
        }
    }
}

__global__ __launch_bounds__(256) void kv_retable_kernel(KvReclaim a, int64_t words)
{
    const int64_t used = a.counts[(words + kSpan - 1) / kSpan];
    for_entries<256>(a, [&](int64_t e) {
        const int id = a.table[e];
        if (id < used || id >= a.blocks) return;
        const int r = a.rank[id];
        if (r >= 0) a.table[e] = a.to[r];
    });
}

unsigned entry_groups(const KvReclaim &a, int num_cus)
{
    const int64_t units = a.B * ((a.cols + kChunk - 1) / kChunk);
    return (unsigned)std::max<int64_t>(1, std::min<int64_t>((units + 3) / 4, (int64_t)num_cus * 8));
}

// One workgroup takes tables of few entries and blocks in one launch, without moves and with: 16,000 entries, 4,000
// blocks 9.8 and 15.2 us, in several launches 22.1 and 25.4; 16,000 blocks 15.3 and 20.8, 25.3 and 30.4; 65,000
// blocks 37.5 and 43.9, 28.9 and 34.2; 64,000 entries, 16,000 blocks 29.9 and 51.8, 33.2 and 36.0.
bool in_one(int64_t blocks, int64_t entries) { return blocks <= kKvFewBlocks && entries <= kKvFewBlocks; }

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

hipError_t launch_kv_fork(const int32_t *parent, const int32_t *child, int n, int32_t *cached, int B, int shift,
                          int32_t *table, int cols, const int32_t *free_blocks, int64_t n_free, int32_t *source,
                          int32_t *to, int64_t *info, int num_cus, hipStream_t s)
{
    const bool few = n <= 2048 && B <= 2048;
    const int waves = (few ? 256 : 1024) / 64;
    const int64_t units = (int64_t)n * ((cols + kChunk - 1) / kChunk);
    // (with info a workgroup more, which the CUs still hold at once)
    const int64_t most = std::max<int64_t>((int64_t)num_cus * (few ? 4 : 1) - (info != nullptr), 1);
    const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>((units + waves - 1) / waves, most)) + (info != nullptr);
    if (few)
        hipLaunchKernelGGL((kv_fork_kernel<256, 8>), dim3(grid), dim3(256), 0, s, parent, child, n, cached, B, shift,
                           table, cols, free_blocks, n_free, source, to, info);
    else
        hipLaunchKernelGGL((kv_fork_kernel<1024, 16>), dim3(grid), dim3(1024), 0, s, parent, child, n, cached, B, shift,
                           table, cols, free_blocks, n_free, source, to, info);
    return hipGetLastError();
}

hipError_t launch_kv_copy(const KvCache &dst, const KvCache &src, const int32_t *to, const int32_t *source, int64_t n,
                          int num_cus, hipStream_t s)
{
    const uint32_t pieces = (uint32_t)((src.rec_bytes() * src.heads + kPiece - 1) / kPiece);
    const int64_t units = n * pieces;
    const unsigned grid = (unsigned)std::min<int64_t>(units, (int64_t)num_cus * 8);
    hipLaunchKernelGGL(kv_copy_kernel, dim3(grid), dim3(256), 0, s, dst, src, to, source, units, pieces);
    return hipGetLastError();
}

size_t kv_reclaim_workspace(int64_t blocks, int64_t entries, int64_t moves, size_t *counts, size_t *rank)
{
    if (in_one(blocks, entries)) return 0;
    const int64_t words = (blocks + 31) / 32;
    *counts = align256((size_t)words * 4);
    *rank = *counts + align256((size_t)((words + kSpan - 1) / kSpan + 1) * 4);
    return *rank + (moves ? align256((size_t)blocks * 4) : 0);
}

hipError_t launch_kv_reclaim(const KvReclaim &a, int num_cus, hipStream_t s)
{
    if (in_one(a.blocks, a.B * a.cols)) {
        hipLaunchKernelGGL(kv_reclaim_one_kernel, dim3(1), dim3(kOne), 0, s, a);
        return hipGetLastError();
    }
    const int64_t words = (a.blocks + 31) / 32;
    const unsigned groups = entry_groups(a, num_cus);
    hipLaunchKernelGGL(kv_clear_kernel, dim3((unsigned)std::min<int64_t>((words + 255) / 256, (int64_t)num_cus * 8)), dim3(256),
                       0, s, a.bits, words);
    if (a.B) hipLaunchKernelGGL(kv_mark_kernel, dim3(groups), dim3(256), 0, s, a);
    hipLaunchKernelGGL(kv_count_kernel, dim3((unsigned)((words + kSpan - 1) / kSpan)), dim3(256), 0, s, a, words);
    hipLaunchKernelGGL(kv_list_kernel, dim3((unsigned)((words + kShare - 1) / kShare)), dim3(256), 0, s, a, words);
    if (a.B && a.moves) hipLaunchKernelGGL(kv_retable_kernel, dim3(groups), dim3(256), 0, s, a, words);
    return hipGetLastError();
}

}  // namespace ivf
