// The stable order of n assignments by their expert: a counting sort.
//
// Every warp owns a run of neighbouring assignments.  It counts its experts (lanes with the same one find each other and count once), the counts of
// all warps are made into the places at which each warp's assignments of each expert begin, and the warp walks its run again and deals
// the places out in order.  Whole numbers throughout: the same result every time.
//
// One block does it all for up to 2048 assignments.  For more, a first launch counts by blocks, and in the second every block adds up the counts
// of the blocks before it (from L2: a table of at most one row for each SM) before it does the same.  Bound by latency: 24 bytes an assignment
// are little, the chain load - count - barrier - scan - barrier - deal is what takes the time. 16 assignments 3.4 us, 8192 of 64 experts 6.6, 262144 of 8 / 256 / 512 experts 7.6 / 11.6 /
// 15.3 (the blocks' counts, read by every block, grow with the experts).
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint32_t kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr uint32_t kOneBlock = 2048;                 // assignments that one block sorts by itself
constexpr uint32_t kSortChunk = 1024;                // and that a block of many takes at least

struct Sort {
    SortArgs a;
    uint32_t blocks, chunk, warps, row, pitch, bits; // warps: that have a run (and a table) of their own; row and pitch: of the tables; bits: of an expert's number
};

__device__ __forceinline__ uint32_t expert_of(const SortArgs& a, uint64_t i) {
    const int64_t e = a.wide ? ((const int64_t*)a.experts)[i] : (int64_t)((const int32_t*)a.experts)[i];
    return e >= 0 && e < (int64_t)a.groups ? (uint32_t)e : a.groups;
}

// The lanes of `there` with the same expert as this one's, a bit of its number at a time.  (The match instruction takes longer the more different values
// there are: 262144 assignments to 8, 256, 512 experts take 7.1, 12.3, 15.7 us with it.)
__device__ __forceinline__ uint32_t same_expert(uint32_t there, uint32_t e, uint32_t bits) {
    uint32_t same = there;
    for (uint32_t b = 0; b < bits; ++b) {
        const uint32_t set = __ballot_sync(there, e >> b & 1);
        same &= e >> b & 1 ? set : ~set;
    }
    return same;
}

// A warp's run, 32 assignments at a time, kAhead of them loaded at once.
constexpr uint32_t kAhead = 4, kNone = 0xffffffffu;
struct Ahead { uint32_t e[kAhead]; };
__device__ __forceinline__ Ahead load_ahead(const SortArgs& a, uint64_t i, uint64_t to) {
    Ahead r;
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) r.e[j] = i + 32 * j < to ? expert_of(a, i + 32 * j) : kNone;
    return r;
}
// each(expert, lanes with the same, assignment) for the run [from, to); `first`: what is loaded already
template <class Each>
__device__ __forceinline__ void walk(const SortArgs& a, const Ahead& first, uint64_t from, uint64_t to, uint32_t bits, Each each) {
    const uint32_t lane = threadIdx.x & 31;
    Ahead now = first;
    for (uint64_t i = from; i < to; i += 32 * kAhead) {
        const Ahead next = i + 32 * kAhead < to ? load_ahead(a, i + 32 * kAhead + lane, to) : now;
#pragma unroll
        for (uint32_t j = 0; j < kAhead; ++j) {
            const uint32_t there = __ballot_sync(0xffffffffu, now.e[j] != kNone);
            if (now.e[j] != kNone) each(now.e[j], there, same_expert(there, now.e[j], bits), i + 32 * j + lane);
            __syncwarp();
        }
        now = next;
    }
}

// One row of counts for each block, a whole number of 16-byte accesses long
__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ Sort s) {
    extern __shared__ uint32_t count[];
    const uint32_t keys = s.a.groups + 1;
    for (uint32_t g = threadIdx.x; g < s.row; g += kSortThreads) count[g] = 0;
    chain_acquire();
    __syncthreads();
    const uint64_t from = (uint64_t)blockIdx.x * s.chunk, to = min(from + s.chunk, s.a.n);
    for (uint64_t i = from + threadIdx.x; i < to; i += kSortThreads) atomicAdd(count + expert_of(s.a, i), 1u);
    __syncthreads();
    for (uint32_t g = threadIdx.x; g < s.row; g += kSortThreads) s.a.workspace[(uint64_t)blockIdx.x * s.row + g] = g < keys ? count[g] : 0;
}

// inclusive sum over the warp
__device__ __forceinline__ uint32_t warp_scan(uint32_t v) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += u;
    }
    return v;
}

__global__ void __launch_bounds__(kSortThreads) k_sort(const __grid_constant__ Sort s) {
    extern __shared__ __align__(16) uint32_t memory[];
    __shared__ uint32_t sums[kSortWarps];
    const uint32_t keys = s.a.groups + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // counts in all blocks, in the blocks before this one; by warps
    uint32_t *total = memory, *before = total + s.row, *table = before + s.row;
    for (uint32_t i = threadIdx.x; i < 2 * s.row + s.warps * s.pitch; i += kSortThreads) memory[i] = 0;
    chain_acquire();
    __syncthreads();

    const uint64_t first = (uint64_t)blockIdx.x * s.chunk, end = min(first + s.chunk, s.a.n);
    const uint64_t run = ((end - first + s.warps - 1) / s.warps + 31) / 32 * 32;
    const uint64_t from = min(first + warp * run, end), to = min(from + run, end);
    const Ahead loaded = load_ahead(s.a, from + lane, to);       // on its way while the blocks' counts are added up
    if (s.blocks > 1) {                              // a thread adds up four experts over some of the blocks, several loads on their way at once
        const uint32_t quads = s.row / 4, parts = kSortThreads / quads, part = threadIdx.x / quads, q = threadIdx.x - part * quads;
        if (part < parts) {
            const uint4* counts = (const uint4*)s.a.workspace + q;
            uint4 all = make_uint4(0, 0, 0, 0), earlier = all;
#pragma unroll 8
            for (uint32_t b = part; b < s.blocks; b += parts) {
                const uint4 c = counts[(uint64_t)b * quads];
                all.x += c.x; all.y += c.y; all.z += c.z; all.w += c.w;
                if (b < blockIdx.x) { earlier.x += c.x; earlier.y += c.y; earlier.z += c.z; earlier.w += c.w; }
            }
            const uint32_t a4[4] = {all.x, all.y, all.z, all.w}, e4[4] = {earlier.x, earlier.y, earlier.z, earlier.w};
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                if (a4[i]) atomicAdd(total + 4 * q + i, a4[i]);
                if (e4[i]) atomicAdd(before + 4 * q + i, e4[i]);
            }
        }
    }
    uint32_t* const mine = table + warp * s.pitch;
    if (warp < s.warps)
        walk(s.a, loaded, from, to, s.bits, [mine, lane](uint32_t e, uint32_t, uint32_t same, uint64_t) {
            if (lane == __ffs(same) - 1) mine[e] += __popc(same);
        });
    __syncthreads();

    // the warps before, for each expert: a thread an expert, eight warps' counts at once
    for (uint32_t g = threadIdx.x; g < keys; g += kSortThreads) {
        uint32_t sum = 0;
        for (uint32_t w = 0; w < s.warps; w += 8) {
            uint32_t c[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) c[i] = table[(w + i) * s.pitch + g];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                table[(w + i) * s.pitch + g] = sum;
                sum += c[i];
            }
        }
        if (s.blocks == 1) total[g] = sum;
    }
    __syncthreads();
    // the experts before and the blocks before: where this block's assignments of each expert begin
    uint32_t carry = 0;
    for (uint32_t at = 0; at < keys; at += kSortThreads) {
        const uint32_t g = at + threadIdx.x, all = g < keys ? total[g] : 0, sum = warp_scan(all);
        if (lane == 31) sums[warp] = sum;
        __syncthreads();
        if (warp == 0) sums[lane] = warp_scan(sums[lane]);
        __syncthreads();
        const uint32_t start = carry + (warp ? sums[warp - 1] : 0) + sum - all;
        if (g < keys) {
            before[g] += start;
            if (blockIdx.x == 0) s.a.offsets[g] = start;         // of those that belong to no expert: where those of the last one end
        }
        carry += sums[kSortWarps - 1];
        __syncthreads();
    }
    if (warp >= s.warps) return;

    walk(s.a, loaded, from, to, s.bits, [&](uint32_t e, uint32_t there, uint32_t same, uint64_t i) {
        const uint32_t place = before[e] + mine[e] + __popc(same & ((1u << lane) - 1));
        __syncwarp(there);
        if (lane == __ffs(same) - 1) mine[e] += __popc(same);
        if (s.a.order) s.a.order[place] = (int64_t)i;
        if (s.a.places) s.a.places[i] = place;
    });
}

uint32_t row_of(uint32_t groups) { return (groups + 1 + 3) / 4 * 4; }
uint32_t blocks_of(uint64_t n, int sm_count) {
    if (n <= kOneBlock) return 1;
    const uint64_t want = (n + kSortChunk - 1) / kSortChunk;
    return (uint32_t)(want < (uint64_t)sm_count ? want : sm_count);
}

}  // namespace

uint64_t sort_workspace(uint64_t n, uint32_t groups, int sm_count) {
    const uint32_t b = blocks_of(n, sm_count);
    return b > 1 ? (uint64_t)b * row_of(groups) * 4 : 0;
}

int launch_sort(const SortArgs& a, int sm_count, cudaStream_t st) {
    Sort s{a, blocks_of(a.n, sm_count), 0, kSortWarps, row_of(a.groups), a.groups + 1, 0};
    while (a.groups >> s.bits) ++s.bits;
    s.chunk = (uint32_t)((a.n + s.blocks - 1) / s.blocks);
    s.blocks = (uint32_t)((a.n + s.chunk - 1) / s.chunk);
    const uint64_t most = 200 << 10;                 // bytes of shared memory
    while ((2ull * s.row + s.warps * s.pitch) * 4 > most) s.warps /= 2;
    const uint32_t smem = (2 * s.row + s.warps * s.pitch) * 4;
    // the limit without leave is that of the tables and the kernel's own variables together (360 experts are over it by those alone)
    if (smem + kSortWarps * 4 > 48 << 10) SK_OP_CUDA(cudaFuncSetAttribute(k_sort, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most));
    if (s.blocks > 1) SK_OP_CUDA(launch_kernel(true, k_sort_count, dim3(s.blocks), kSortThreads, s.row * 4, st, s));
    SK_OP_CUDA(launch_kernel(true, k_sort, dim3(s.blocks), kSortThreads, smem, st, s));
    return SK_OK;
}

}  // namespace sk
