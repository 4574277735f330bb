// The stable order of n assignments by their expert: a counting sort.
//
// Every warp owns a run of neighbouring assignments.  It counts its experts (lanes with the same one find each other and count once), the counts of
// all warps are made into the places at which each warp's assignments of each expert begin, and the warp walks its run again and deals
// the places out in order.  Whole numbers throughout: the same result every time.
//
// One block does it all for a few thousand assignments.  For more, a first launch counts by blocks, and in the second every block adds up the counts
// of the blocks before it (from L2: a table of at most one row for each SM) before it does the same.  Bound by latency: 24 bytes an assignment
// are little, the chain load - count - barrier - scan - barrier - deal is what takes the time.
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint32_t kSortThreads = 1024;
constexpr uint32_t kOneBlock = 8192;                 // assignments that one block sorts by itself
constexpr uint32_t kSortChunk = 2048;                // and that a block of many takes at least

struct Sort {
    SortArgs a;
    uint32_t blocks, chunk, warps;                   // warps: that have a run (and a table) of their own
};

__device__ __forceinline__ uint32_t expert_of(const SortArgs& a, uint64_t i) {
    const int64_t e = a.wide ? ((const int64_t*)a.experts)[i] : (int64_t)((const int32_t*)a.experts)[i];
    return e >= 0 && e < (int64_t)a.groups ? (uint32_t)e : a.groups;
}

// counts the run [from, to) of this warp into its table
__device__ __forceinline__ void count_run(const SortArgs& a, uint64_t from, uint64_t to, uint32_t* table) {
    const uint32_t lane = threadIdx.x & 31;
    for (uint64_t i = from; i < to; i += 32) {
        const uint32_t there = __ballot_sync(0xffffffffu, i + lane < to);
        if (i + lane < to) {
            const uint32_t e = expert_of(a, i + lane), same = __match_any_sync(there, e);
            if (lane == __ffs(same) - 1) table[e] += __popc(same);
        }
        __syncwarp();
    }
}

// one row of counts for each block
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ Sort s) {
    extern __shared__ uint32_t count[];
    const uint32_t keys = s.a.groups + 1;
    for (uint32_t g = threadIdx.x; g < keys; g += kSortThreads) count[g] = 0;
    chain_acquire();
    __syncthreads();
    const uint64_t from = (uint64_t)blockIdx.x * s.chunk, to = min(from + s.chunk, s.a.n);
    for (uint64_t i = from + threadIdx.x; i < to; i += kSortThreads) atomicAdd(count + expert_of(s.a, i), 1u);
    __syncthreads();
    for (uint32_t g = threadIdx.x; g < keys; g += kSortThreads) s.a.workspace[(uint64_t)blockIdx.x * keys + g] = count[g];
}

__global__ void __launch_bounds__(kSortThreads) k_sort(const __grid_constant__ Sort s) {
    extern __shared__ uint32_t memory[];
    __shared__ uint32_t sums[kSortThreads / 32];
    const uint32_t keys = s.a.groups + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t *table = memory, *total = memory + s.warps * keys, *before = total + keys;      // counts in all blocks, in the blocks before
    for (uint32_t i = threadIdx.x; i < (s.warps + 2) * keys; i += kSortThreads) memory[i] = 0;
    chain_acquire();
    __syncthreads();

    const uint64_t first = (uint64_t)blockIdx.x * s.chunk, end = min(first + s.chunk, s.a.n);
    const uint64_t run = ((end - first + s.warps - 1) / s.warps + 31) / 32 * 32;
    const uint64_t from = min(first + warp * run, end), to = min(from + run, end);
    if (warp < s.warps) count_run(s.a, from, to, table + warp * keys);
    if (s.blocks > 1) {
        const uint32_t all = s.blocks * keys, mine = blockIdx.x * keys;
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < all; i += kSortThreads) {
            const uint32_t c = s.a.workspace[i];
            if (c) {
                const uint32_t g = i % keys;
                atomicAdd(total + g, c);
                if (i < mine) atomicAdd(before + g, c);
            }
        }
    }
    __syncthreads();

    // every warp's first place of each expert: the experts before, the blocks before, the warps before
    uint32_t carry = 0;
    for (uint32_t at = 0; at < keys; at += kSortThreads) {
        const uint32_t g = at + threadIdx.x;
        uint32_t here = 0;
        if (g < keys)
            for (uint32_t w = 0; w < s.warps; ++w) {
                const uint32_t c = table[w * keys + g];
                table[w * keys + g] = here;
                here += c;
            }
        const uint32_t all = s.blocks > 1 ? (g < keys ? total[g] : 0) : here;
        uint32_t sum = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += u;
        }
        if (lane == 31) sums[warp] = sum;
        __syncthreads();
        if (warp == 0) {
            uint32_t v = sums[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            sums[lane] = v;
        }
        __syncthreads();
        const uint32_t start = carry + (warp ? sums[warp - 1] : 0) + sum - all;
        if (g < keys) {
            const uint32_t base = start + before[g];
            for (uint32_t w = 0; w < s.warps; ++w) table[w * keys + g] += base;
            if (blockIdx.x == 0) s.a.offsets[g] = start;         // of the ones that belong to no expert: where those of the last one end
        }
        carry += sums[kSortThreads / 32 - 1];
        __syncthreads();
    }
    if (warp >= s.warps) return;

    uint32_t* next = table + warp * keys;
    for (uint64_t i = from; i < to; i += 32) {
        const uint32_t there = __ballot_sync(0xffffffffu, i + lane < to);
        if (i + lane < to) {
            const uint32_t e = expert_of(s.a, i + lane), same = __match_any_sync(there, e);
            const uint32_t place = next[e] + __popc(same & ((1u << lane) - 1));
            __syncwarp(there);
            if (lane == __ffs(same) - 1) next[e] += __popc(same);
            if (s.a.order) s.a.order[place] = (int64_t)(i + lane);
            if (s.a.places) s.a.places[i + lane] = place;
        }
        __syncwarp();
    }
}

uint32_t blocks_of(uint64_t n, int sm_count) {
    if (n <= kOneBlock) return 1;
    const uint64_t want = (n + kSortChunk - 1) / kSortChunk;
    return (uint32_t)(want < (uint64_t)sm_count ? want : sm_count);
}

}  // namespace

uint64_t sort_workspace(uint64_t n, uint32_t groups, int sm_count) {
    const uint32_t b = blocks_of(n, sm_count);
    return b > 1 ? (uint64_t)b * (groups + 1) * 4 : 0;
}

int launch_sort(const SortArgs& a, int sm_count, cudaStream_t st) {
    Sort s{a, blocks_of(a.n, sm_count), 0, 0};
    s.chunk = (uint32_t)((a.n + s.blocks - 1) / s.blocks);
    s.blocks = (uint32_t)((a.n + s.chunk - 1) / s.chunk);
    const uint64_t keys = a.groups + 1, most = 200 << 10;        // bytes of shared memory
    s.warps = kSortThreads / 32;
    while ((s.warps + 2) * keys * 4 > most) s.warps /= 2;
    const uint32_t smem = (uint32_t)((s.warps + 2) * keys * 4);
    if (smem > 48 << 10) SK_OP_CUDA(cudaFuncSetAttribute(k_sort, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
    if (s.blocks > 1) SK_OP_CUDA(launch_kernel(true, k_sort_count, dim3(s.blocks), kSortThreads, keys * 4, st, s));
    SK_OP_CUDA(launch_kernel(true, k_sort, dim3(s.blocks), kSortThreads, smem, st, s));
    return SK_OK;
}

}  // namespace sk
