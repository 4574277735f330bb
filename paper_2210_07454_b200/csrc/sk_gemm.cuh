// Matrix products on the tensor cores (tcgen05), for the operators whose epilogues and schedules differ: one kernel, templated on
// the tile, on the plan that says which tiles there are, and on what happens to a finished tile.
//
//   D(i, j) = sum_k A(i, k) * B(j, k)      16-bit operands, 32-bit sums
//
// Each operand may be stored with k contiguous ("K-major") or with its row index contiguous ("MN-major"); no operand is
// ever transposed in memory.  A tile may go over two or three pairs of operands (matrices held as the sum of two 16-bit matrices).
//
// A block (CG = 1) or a pair of blocks on two SMs (CG = 2) works on one output tile of 128*CG rows by BN columns at a
// time and walks over tiles until none is left.  One warp feeds a ring of kStages shared-memory stages by TMA (64 values of k a
// stage, 128-byte swizzle), one thread issues the matrix instructions, eight warps empty the accumulators (sixteen,
// with less shared memory for the ring: 67 against 63 us for the gradient of 8 x 50257 x 768).  Two
// accumulators in tensor memory take turns, so the next tile's products run while this tile's epilogue does.
//
// The tensor cores truncate what they add to an accumulator: a sum of 4096 bf16 products of one sign comes out 1.1e-5 too small, one of 256 by 3e-7.
// Where an epilogue needs its sums to 32 bits (kParts), a tile's products are cut along K and the accumulators take turns part by part: the
// epilogue adds the parts up in registers, with rounding.
//
// Every wait has a limit (Waits).  A role whose wait runs out counts it and leaves its loop: it waits for nothing
// more but what it has set going itself (copies, matrix instructions), once and with the same limit.  The others follow when their
// own waits, begun at most a tile later, run out.  So the kernel ends within about two limits, and the host reads an error instead of hanging.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {

constexpr int kGemmK = 64;                    // values of k per stage: 128 bytes, the width of the swizzle
constexpr int kStageWords = 1024;             // of shared memory that store_tile32 needs, for each epilogue warp

// What the kernel's roles have to know of a tile.
struct TileJob {
    uint32_t M, N;                            // extents of the output
    uint32_t m, n, b, slice;                  // the tile: row, column, matrix, slice of K
    uint32_t kind, step;                      // which product: for the epilogue
    uint32_t part;                            // stages to an accumulation, for epilogues with kParts
    uint32_t k_stages, pass;                  // stages (none: begin() does it all); the first `pass` of them over a and b, the next over a2 and b2, a3 and b3
    int k_first, z;                           // first k, matrix of the operands
    uint32_t a_mn, b_mn;                      // 1: MN-major
    uint32_t a_rows;                          // rows of A a block loads: 128, or fewer where a single tile row has no more
    uint32_t k_rows;                          // values of k in a stage: 64, or fewer where K has no more (in steps of 16)
    uint32_t bf16;                            // operand type: 1 bf16, 0 fp16
    const CUtensorMap *map_a, *map_b, *map_a2, *map_b2, *map_a3, *map_b3;
};

// Of a ragged plan, whose tiles differ in their columns and in the rows of their last stage
struct RaggedJob : TileJob {
    uint32_t cols;                            // columns of the matrix instruction: a multiple of 16, at most BN
    uint32_t last_rows;                       // values of k in the last stage, rounded up to 16
    uint32_t last_valid;                      // and those that are the tile's
    uint32_t first;                           // first row of the ragged side
};

// ---- instruction wrappers -------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// bar: a shared::cluster address (a block's own shared::cta addresses are valid ones).  What it orders is the reading of tensor memory, which
// the tcgen05 fences around it do; a release to the whole cluster would wait for the epilogue's global stores as well.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {      // does not suspend the thread: cheaper where it is ready
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t clock_ns() {
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
// Tries until `ready` says so: some ten thousand at once, as ordinary waits need, then with pauses of about half a microsecond, until the
// limit has passed on the GPU's clock.  A try may itself take long (mbarrier.try_wait suspends the thread for a time that the hardware
// chooses), so tries alone do not bound a wait; they do so as the last resort, should the clock stand still.
constexpr uint32_t kQuickTries = 256, kQuickRounds = 64, kSlowTries = 1u << 28;
template <class Ready>
__device__ __forceinline__ bool wait_longer(Ready ready, const Waits& w) {
    const uint64_t end = clock_ns() + w.limit_ms * 1000000ull;
    for (uint32_t r = 1; r < kQuickRounds && clock_ns() <= end; ++r)
        for (uint32_t i = 0; i < kQuickTries; ++i)
            if (ready()) return true;
    for (uint32_t i = 0; i < kSlowTries && clock_ns() <= end; ++i) {
        if (ready()) return true;
        __nanosleep(500);
    }
    atomicAdd(w.status, 1u);
    return false;
}
template <class Ready>
__device__ __forceinline__ bool wait_until(Ready ready, const Waits& w) {
    for (uint32_t i = 0; i < kQuickTries; ++i)
        if (ready()) return true;
    return wait_longer(ready, w);
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const Waits& w) {
    return wait_until([bar, parity] { return mbar_try(bar, parity); }, w);
}
// the same for a warp that stays together
__device__ __forceinline__ bool mbar_wait_warp(uint32_t bar, uint32_t parity, const Waits& w) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, w)); }
__device__ __forceinline__ uint32_t map_to_leader(uint32_t addr) {      // the same address in block 0 of the cluster
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One lane of a whole warp.  The compiler knows that a single thread runs what depends on it, and hands it the operands that the copy engine and the tensor
// cores take from uniform registers without a loop over the lanes, which `lane == 0` costs: 16384 x 2048 x 2048 100 us with that, 90.7 so.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z) {
    if constexpr (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
            ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t cols) {
    if constexpr (CG == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
    if constexpr (CG == 2) {
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
    } else {
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
    }
}
template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier at this address of every block of the pair once all products issued so far are done
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void tmem_load8(uint32_t addr, float (&v)[8]) {
    uint32_t r[8];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
// 16 of a warp's rows and 32 columns, as fragments of 8 x 8: of the j-th eight columns a lane has row lane / 4 in v[4 j], v[4 j + 1] and row lane / 4 + 8 in
// the next two, columns 2 (lane mod 4) and the one after it.
__device__ __forceinline__ void tmem_load_fragments(uint32_t addr, float (&v)[32], int at) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) v[at + i] = __uint_as_float(r[i]);
}
// Shared-memory descriptor, 128-byte swizzle.  K-major: rows of 128 bytes, groups of eight rows 1024 bytes apart.
// MN-major: blocks of 64 row indices (block_bytes from one to the next: 8192 if they are 64 k deep), groups of eight k 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr, bool mn, uint32_t block_bytes = 8192) {
    const uint64_t lead = mn ? (block_bytes >> 4) : 1u;
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (lead << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// ---- one product, or two that do not depend on each other ---------------------------------------------------------------
struct GemmGroup {
    uint32_t M, N;                            // output extents
    uint32_t k_blocks, k_total;               // stages per tile, and along K: more where K is split
    uint32_t slices;                          // of K: slice s writes a result of its own
    uint32_t tiles_m, tiles_n, tiles;
    uint32_t band;                            // tiles are walked in bands of this many tile rows, row index fastest
    uint32_t a_mn, b_mn, a_rows, k_rows, bf16, part;
};
// The product with the longer tiles is the first.  Each of the `units` (blocks or pairs) takes the first's tiles in turn; `early` is how
// many rounds of the second's tiles the units that got one tile less of the first are ahead.
struct GemmPlan {
    CUtensorMap map[4];                       // A and B of the first, of the second
    GemmGroup g[2];
    uint32_t groups, early;
    Waits waits;
    static constexpr bool kCooperative = false, kEmpty = false, kThree = false;      // kThree: a third pair of operands
    static constexpr bool kRagged = false;

    __device__ __forceinline__ bool job(uint32_t p, uint32_t units, uint32_t i, TileJob& j) const {
        uint32_t t = p + i * units, group = 0;
        if (t >= g[0].tiles) {
            if (groups < 2) return false;
            group = 1;
            const uint32_t q = g[0].tiles / units, r = g[0].tiles - q * units;   // units below r had q + 1 tiles, the others q
            const uint32_t k = i - (q + (p < r)), head = early * (units - r);
            if (p >= r) t = k < early ? k * (units - r) + (p - r) : head + (k - early) * units + p;
            else t = head + k * units + p;
            if (t >= g[1].tiles) return false;
        }
        const GemmGroup& s = g[group];
        const uint32_t per = s.tiles_m * s.tiles_n;
        j.b = 0;
        j.slice = t / per;
        uint32_t q = t - j.slice * per;
        const uint32_t band = q / (s.band * s.tiles_n);
        q -= band * s.band * s.tiles_n;
        const uint32_t rows = min(s.band, s.tiles_m - band * s.band);
        j.n = q / rows;
        j.m = band * s.band + (q - j.n * rows);
        j.M = s.M;
        j.N = s.N;
        j.kind = group;
        j.step = 0;
        j.k_stages = j.pass = min(s.k_blocks, s.k_total - j.slice * s.k_blocks);
        j.k_first = (int)(j.slice * s.k_blocks * kGemmK);
        j.z = 0;
        j.a_mn = s.a_mn;
        j.b_mn = s.b_mn;
        j.a_rows = s.a_rows;
        j.k_rows = s.k_rows;
        j.bf16 = s.bf16;
        j.part = s.part;
        j.map_a = j.map_a2 = &map[2 * group];
        j.map_b = j.map_b2 = &map[2 * group + 1];
        return true;
    }
    __device__ __forceinline__ bool wait(const TileJob&) const { return true; }
    __device__ __forceinline__ void done(const TileJob&) const {}
    __device__ __forceinline__ const CUtensorMap* descriptor(uint32_t i) const { return i < 2 * groups ? &map[i] : nullptr; }
};

// Epi::kWarps epilogue warps with kWords of shared memory each.  The ring takes what is left of the 227 KB, six stages of 32 KB beside 4 KB a warp: two would cover
// the 1600 cycles from a copy's issue to its arrival, more even out the waits.
template <int CG, int BN, class Epi>
struct GemmTile {
    static constexpr int kEpiBytes = Epi::kWarps * Epi::kWords * 4;
    static constexpr int kThreads = 64 + 32 * Epi::kWarps;
    static constexpr int kStageBytes = 128 * 128 + (BN / CG) * 128;      // both operands, 64 values of k
    static constexpr int kFixed = kEpiBytes + 1024 + 512;    // the epilogue's, alignment of the swizzle, barriers
    static constexpr int kStages = (232448 - kFixed) / kStageBytes;
    static constexpr int kSmem = kStages * kStageBytes + kEpiBytes + 1024;
};

// Plan: job(unit, units, i, job): the unit's i-th tile; wait(job): until its operands are there; done(job): called by every epilogue warp
// when its share of the tile is written.  kRagged: the tiles depend on data; prepare(shared address of all epilogue warps' memory) is called once by the
// whole block before the first job(); Feed(plan, job, rank) holds what the copies of a tile's stages need: copy(k, ...) issues them, bytes(k) is what they bring to a
// block.  Epi: load() reads 32 columns of the accumulator, column() says which, nothing() writes a tile without products, finish() is called after the last tile.
// Epi: struct Args; __device__ Epi(const Args&, job, row, part, shared address of the warp's memory); begin(plan, first column) before the
// accumulator is waited for, false (in the whole warp) if a wait of its own ran out; kParts: see above; chunk(col, v[32], last); end(); kWords of shared memory for each warp.  A thread holds one
// row of the tile and gets its columns 32 at a time; the kWarps / 4 warps that share a row take a part of the columns each.  Rows >= M
// are passed too (the epilogue skips them: all lanes of a warp stay together), columns >= N may be.
template <int CG, int BN, class Plan, class Epi>
__global__ void __launch_bounds__(64 + 32 * Epi::kWarps, 1)
k_gemm(const __grid_constant__ Plan plan, const __grid_constant__ typename Epi::Args ea) {
    constexpr int kStages = GemmTile<CG, BN, Epi>::kStages;
    constexpr int kRowsB = BN / CG;
    constexpr int kBytesA = 128 * 128, kBytesB = kRowsB * 128;
    constexpr uint32_t kTmemCols = 2 * BN;                       // a power of two >= 32
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bars[2 * kStages + 4];
    __shared__ uint32_t tmem_slot;

    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const uint32_t stages = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](uint32_t s) { return bar0 + 8 * s; };
    auto empty = [&](uint32_t s) { return bar0 + 8 * (kStages + s); };
    auto acc_full = [&](uint32_t a) { return bar0 + 8 * (2 * kStages + a); };
    auto acc_empty = [&](uint32_t a) { return bar0 + 8 * (2 * kStages + 2 + a); };

    if (threadIdx.x == 0) {
        for (uint32_t s = 0; s < (uint32_t)kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (uint32_t a = 0; a < 2; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), CG * Epi::kWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tmem_alloc<CG>(smem_u32(&tmem_slot), kTmemCols);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)&tmem_slot;
    if (threadIdx.x < 16) {                                      // the descriptors depend on no other kernel
        const CUtensorMap* m = plan.descriptor(threadIdx.x);
        if (m) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }

    // A ragged product may begin while the one before it in the stream, whose results it does not need, still runs: that one's blocks have all passed their
    // own chain_acquire() by now, so whatever was launched before it is complete. The wait is made up for at the end.
    bool waited = true;
    if constexpr (Plan::kRagged) waited = !plan.beside;
    if (waited) chain_acquire();
    // the grid fits the SMs, so it is resident as a whole: the next kernel's blocks may take the slots that are free
    chain_release();

    const uint32_t unit = blockIdx.x / CG, units = gridDim.x / CG;
    std::conditional_t<Plan::kRagged, RaggedJob, TileJob> t;
    constexpr uint32_t kBytes = kBytesA + kBytesB;
    if constexpr (Plan::kRagged) {
        plan.prepare(smem_raw + (stages - smem_u32(smem_raw)) + kStages * kBytes);
        __syncthreads();
    }

    // The two single threads that feed the tensor cores have a stage's time, some 600 cycles, for each trip of their loops: what is constant
    // over a tile is in registers, and the ring's slot and its parity go round without divisions.
    bool feeds = true;                                           // no copies: the waits for them, and for what would come of them, run out
    if constexpr (Plan::kRagged) feeds = !plan.withheld;
    if (warp == 0) {
        if (feeds && elect_one()) {
            uint32_t s = 0, parity = 1;                          // a fresh barrier counts as having completed its previous phase
            bool ok = true, any = false;
            for (uint32_t i = 0; ok && plan.job(unit, units, i, t); ++i) {
                if constexpr (Plan::kRagged) {
                    any = true;
                    const uint32_t kb = t.k_stages;
                    typename Plan::Feed feed(plan, t, rank);
                    for (uint32_t k = 0; k < kb; ++k) {
                        if (!(ok = mbar_wait(empty(s), parity, plan.waits))) break;
                        const uint32_t sa = stages + s * kBytes;
                        uint32_t bar = full(s);
                        if (rank == 0) mbar_expect(bar, CG * feed.bytes(k));
                        if constexpr (CG == 2) bar = map_to_leader(bar);
                        feed.copy(k, sa, sa + kBytesA, bar);
                        if (++s == (uint32_t)kStages) { s = 0; parity ^= 1; }
                    }
                    continue;
                }
                if (!(ok = plan.wait(t))) break;
                const uint32_t kb = t.k_stages, pass = t.pass;
                const bool a_mn = t.a_mn, b_mn = t.b_mn;
                const int z = t.z;
                const int row_a = (int)(t.m * (128 * CG) + rank * 128);
                const int row_b = (int)(t.n * BN + rank * kRowsB);
                const uint32_t bytes = CG * 128 * ((a_mn ? 2 * t.k_rows : t.a_rows) + (b_mn ? kRowsB / 64 * t.k_rows : kRowsB));
                const CUtensorMap *ma = t.map_a, *mb = t.map_b;
                int k0 = t.k_first;
                any = true;
                for (uint32_t k = 0; k < kb; ++k, k0 += kGemmK) {
                    if (k == pass) {                             // the second pair of operands, from the start of K
                        ma = t.map_a2;
                        mb = t.map_b2;
                        k0 = t.k_first;
                    }
                    if (Plan::kThree && k == 2 * pass) {
                        ma = t.map_a3;
                        mb = t.map_b3;
                        k0 = t.k_first;
                    }
                    if (!(ok = mbar_wait(empty(s), parity, plan.waits))) break;
                    const uint32_t sa = stages + s * kBytes, sb = sa + kBytesA;
                    uint32_t bar = full(s);
                    if (rank == 0) mbar_expect(bar, bytes);
                    if constexpr (CG == 2) bar = map_to_leader(bar);
                    if (a_mn) {
                        tma_load<CG>(sa, ma, bar, row_a, k0, z);
                        tma_load<CG>(sa + 8192, ma, bar, row_a + 64, k0, z);
                    } else {
                        tma_load<CG>(sa, ma, bar, k0, row_a, z);
                    }
                    if (b_mn) {
#pragma unroll
                        for (int q = 0; q < kRowsB / 64; ++q) tma_load<CG>(sb + q * 8192, mb, bar, row_b + q * 64, k0, z);
                    } else {
                        tma_load<CG>(sb, mb, bar, k0, row_b, z);
                    }
                    if (++s == (uint32_t)kStages) { s = 0; parity ^= 1; }
                }
            }
            // this block's own copies land in its shared memory: all of them are waited for before the block may end (where the products
            // have been given up, for the limit, in which they land)
            if (any)
                for (uint32_t q = 0; q < (uint32_t)kStages; ++q) {
                    if (!mbar_wait(empty(s), parity, plan.waits)) break;
                    if (++s == (uint32_t)kStages) { s = 0; parity ^= 1; }
                }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            uint32_t s = 0, parity = 0, m = 0;                   // m: accumulations so far
            bool ok = true;
            for (uint32_t n = 0; ok && plan.job(unit, units, n, t); ++n) {
                const uint32_t kb = t.k_stages, most = Epi::kParts ? t.part : kb;
                uint32_t steps = t.k_rows / 16, columns = BN;
                if constexpr (Plan::kRagged) {
                    steps = t.last_rows / 16;
                    columns = t.cols;
                }
                const uint32_t whole = steps == kGemmK / 16 ? kb : kb - 1;       // of a ragged tile: stages of four instructions
                if (Plan::kRagged && !kb) continue;              // nothing to add up, no accumulator taken
                // D fp32; A, B bf16 or fp16; majors; N / 8; M / 16
                const uint32_t idesc = (1u << 4) | (t.bf16 << 7) | (t.bf16 << 10) | (t.a_mn << 15) | (t.b_mn << 16) |
                                       ((columns / 8) << 17) | ((uint32_t)(128 * CG / 16) << 24);
                const uint64_t step_a = (t.a_mn ? 2048u : 32u) >> 4, step_b = (t.b_mn ? 2048u : 32u) >> 4;
                const uint64_t desc_a = smem_desc(stages, t.a_mn), desc_b = smem_desc(stages + kBytesA, t.b_mn);
                uint32_t from = 0;
                do {
                    const uint32_t a = m & 1, d = tmem + a * BN, stages_here = Epi::kParts ? min(kb - from, most) : kb;
                    if (m >= 2 && !(Epi::kParts && mbar_test(acc_empty(a), ((m >> 1) - 1) & 1)) &&
                        !(ok = mbar_wait(acc_empty(a), ((m >> 1) - 1) & 1, plan.waits))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (uint32_t k = 0; k < stages_here; ++k) {
                        if (!(ok = mbar_wait(full(s), parity, plan.waits))) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t da = desc_a + s * (kBytes >> 4), db = desc_b + s * (kBytes >> 4);
                        if (Plan::kRagged ? from + k < whole : steps == kGemmK / 16) {
#pragma unroll
                            for (uint32_t q = 0; q < kGemmK / 16; ++q) mma_f16<CG>(d, da + q * step_a, db + q * step_b, idesc, (k | q) != 0);
                        } else {
                            for (uint32_t q = 0; q < steps; ++q) mma_f16<CG>(d, da + q * step_a, db + q * step_b, idesc, (k | q) != 0);
                        }
                        mma_commit<CG>(empty(s));
                        if (++s == (uint32_t)kStages) { s = 0; parity ^= 1; }
                    }
                    mma_commit<CG>(acc_full(a));
                    ++m;
                    from += stages_here;
                } while (Epi::kParts && ok && from < kb);
            }
            if (!ok && m) mbar_wait(acc_full((m - 1) & 1), ((m - 1) >> 1) & 1, plan.waits);      // the products begun, which no epilogue waits for
        }
    } else {
        const uint32_t w = warp - 2, quarter = warp & 3, part = w >> 2;
        constexpr uint32_t kCols = BN / (Epi::kWarps / 4);           // of a warp
        const uint32_t stage = stages + kStages * kBytes + w * Epi::kWords * 4;
        uint32_t m = 0;                                              // accumulations so far
        uint32_t taken = 0;                                          // accumulators so far, of a ragged plan
        for (uint32_t n = 0; plan.job(unit, units, n, t); ++n) {
            const uint32_t turn = Plan::kRagged ? taken : n, a = turn & 1;
            const uint32_t row = t.m * (128 * CG) + rank * 128 + quarter * 32 + lane;
            const uint32_t col0 = t.n * BN + part * kCols;
            Epi epi(ea, t, row, part, stage);
            if (!epi.begin(plan, col0)) break;                   // what it reads travels while the products run
            if constexpr (Plan::kRagged) {
                if (!t.k_stages) {                               // a sum over nothing
                    epi.nothing(part, kCols, BN, rank);
                    continue;
                }
                ++taken;
            }
            if constexpr (Epi::kParts) {
                float sum[kCols / 32][32] = {};                      // 128 of a thread's 168 registers with the widest tile: loads of eight
                bool ok = true;
                const uint32_t kb = t.k_stages, most = t.part;
#pragma unroll 1
                for (uint32_t k = 0; k < kb; k += most, ++m) {
                    const uint32_t b = m & 1;
                    if (!(ok = mbar_wait_warp(acc_full(b), (m >> 1) & 1, plan.waits))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (uint32_t q = 0; q < kCols / 8; ++q) {
                        float v[8];
                        tmem_load8(tmem + b * BN + part * kCols + q * 8 + ((quarter * 32) << 16), v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[q / 4][8 * (q & 3) + i] += v[i];
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_leader(acc_empty(b)) : acc_empty(b));
                }
                if (!ok) break;
                if constexpr (Plan::kRagged) {
#pragma unroll
                    for (uint32_t q = 0; q < kCols / 32; ++q) {
                        const uint32_t col = Epi::column(t, part, q * 32, kCols, BN);
                        if (col < t.N) epi.chunk(col, sum[q], q * 32 + 32 == kCols || Epi::column(t, part, q * 32 + 32, kCols, BN) >= t.N);
                    }
                    continue;
                }
#pragma unroll
                for (uint32_t q = 0; q < kCols / 32; ++q)
                    if (col0 + q * 32 < t.N) epi.chunk(col0 + q * 32, sum[q], q * 32 + 32 == kCols || col0 + q * 32 + 32 >= t.N);
                epi.end();
                plan.done(t);
                continue;
            }
            if (!mbar_wait_warp(acc_full(a), (turn >> 1) & 1, plan.waits)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (Plan::kEmpty && !t.k_stages) {                   // no products
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_leader(acc_empty(a)) : acc_empty(a));
                plan.done(t);
                continue;
            }
            if constexpr (Plan::kRagged) {
                // interleaved or in halves, as the epilogue has it; the accumulator is free after the last columns that exist
                bool more = true;
#pragma unroll 1
                for (uint32_t c = 0; more; c += 32) {
                    const uint32_t col = Epi::column(t, part, c, kCols, BN), at = Epi::kInterleaved ? col : part * kCols + c;
                    more = c + 32 < kCols && Epi::column(t, part, c + 32, kCols, BN) < t.N;
                    float v[32];
                    __syncwarp();
                    if (col < t.N) Epi::load(tmem + a * BN + at + ((quarter * 32) << 16), v);
                    if (!more) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_leader(acc_empty(a)) : acc_empty(a));
                    }
                    if (col < t.N) epi.chunk(col, v, !more);
                }
                continue;
            }
#pragma unroll 1
            for (uint32_t c = 0; c < kCols; c += 32) {
                float v[32];
                __syncwarp();                                    // the load needs the whole warp
                tmem_load32(tmem + a * BN + part * kCols + c + ((quarter * 32) << 16), v);
                if (c + 32 == kCols) {                          // everything is in registers: the accumulator is free
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(CG == 2 ? map_to_leader(acc_empty(a)) : acc_empty(a));
                }
                if (col0 + c < t.N) epi.chunk(col0 + c, v, c + 32 == kCols || col0 + c + 32 >= t.N);
            }
            epi.end();
            plan.done(t);
        }
        if constexpr (Plan::kRagged) Epi::finish();
    }
    if (!waited) chain_acquire();

    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();                   // the other block may still signal this one's barriers
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free<CG>(tmem, kTmemCols);
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------
// A matrix of `rows` x `cols` 16-bit values, cols contiguous, ld and the batch stride in elements (multiples of 8), as the tile
// source of a product: K-major when its columns are k, MN-major when its rows are.
struct Operand {
    const void* p;
    uint64_t rows, cols, ld, batch_stride;
    uint32_t batch;
    bool mn;
};

bool encode_operand(CUtensorMap* map, const Operand& o, bool bf16, uint32_t box_rows);
// outputs that are written in boxes of box_rows rows and 32 columns, with a swizzle as wide as that: 64 bytes, or 128 for fp32
bool encode_out(CUtensorMap* map, void* out, uint64_t batch, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t stride, int type, uint32_t box_rows);

// Launches a plan on at most `units` blocks or pairs.
template <int CG, int BN, class Plan, class Epi>
cudaError_t launch_plan(bool chain, const Plan& plan, const typename Epi::Args& ea, uint32_t units, cudaStream_t st) {
    auto kernel = k_gemm<CG, BN, Plan, Epi>;
    static std::atomic<bool> prepared[64];                       // the attribute is a property of the kernel on a device
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= 64 || !prepared[device]) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GemmTile<CG, BN, Epi>::kSmem);
        if (e != cudaSuccess) return e;
        if (device < 64) prepared[device] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(units * CG);
    cfg.blockDim = dim3(GemmTile<CG, BN, Epi>::kThreads);
    cfg.dynamicSmemBytes = GemmTile<CG, BN, Epi>::kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    uint32_t n = 0;
    if (CG > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = CG;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (Plan::kCooperative) {                                    // its blocks wait for one another: all of them resident, or an error
        attr[n].id = cudaLaunchAttributeCooperative;
        attr[n].val.cooperative = 1;
        ++n;
    } else if (chain) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, plan, ea);
}

// The tile-dependent part of a product.  slices > 1 splits K.
template <int CG, int BN>
void set_tiles(GemmGroup& g, const Operand& a, const Operand& b, uint32_t slices) {
    g.a_mn = a.mn;
    g.b_mn = b.mn;
    const uint64_t K = a.mn ? a.rows : a.cols;
    g.k_total = (uint32_t)((K + kGemmK - 1) / kGemmK);
    g.k_rows = K < kGemmK ? (uint32_t)((K + 15) / 16 * 16) : kGemmK;
    g.k_blocks = (g.k_total + slices - 1) / slices;
    g.slices = (g.k_total + g.k_blocks - 1) / g.k_blocks;            // no empty slice, and never more than asked for
    g.tiles_m = (g.M + 128 * CG - 1) / (128 * CG);
    g.tiles_n = (g.N + BN - 1) / BN;
    g.tiles = g.slices * g.tiles_m * g.tiles_n;
    // The rest of the stage's rows stay what they were and give sums that nobody reads.  Loading them as zeros is not free: 8 tokens
    // against 128,000 x 4096 took 285 us so, and takes 186 us without (reading the matrix alone 172).
    g.a_rows = CG == 1 && !g.a_mn && g.M < 128 ? (g.M + 7) / 8 * 8 : 128;
    // Tiles that run at the same time share operands through L2.  Where A is the smaller operand and fits, its whole height is walked
    // first, so that B is read once; where B is, a band is just high enough for the SMs to span the width: A is read
    // once and whole rows of D are written together.
    const uint64_t a_bytes = g.M * K * 2, b_bytes = g.N * K * 2;
    uint32_t band = 16;
    if (a_bytes <= b_bytes && a_bytes <= (32u << 20)) band = g.tiles_m;
    if (a_bytes > b_bytes) band = g.tiles_n >= 74 ? 1 : 74 / g.tiles_n < 8 ? 74 / g.tiles_n : 8;
    g.band = band < g.tiles_m ? band : g.tiles_m;
}

// What a tile costs beside its stages, in stages (its epilogue where nothing hides it)
constexpr uint32_t kTileCost = 6;

// One product, or two in one launch with the longer tiles first; slices: K of the first is split into so many.
template <int CG, int BN, class Epi>
cudaError_t launch_products(bool chain, const Operand& a, const Operand& b, GemmGroup g0, uint32_t slices, const Operand* a2, const Operand* b2,
                            const GemmGroup* g1, const Waits& waits, const typename Epi::Args& ea, int sm_count, cudaStream_t st) {
    GemmPlan p{};
    set_tiles<CG, BN>(g0, a, b, slices);
    p.g[0] = g0;
    p.groups = 1;
    p.waits = waits;
    uint32_t tiles = g0.tiles;
    auto encode = [&](CUtensorMap* map, const GemmGroup& g, const Operand& x, const Operand& y) {
        return encode_operand(map, x, g.bf16, x.mn ? g.k_rows : g.a_rows) && encode_operand(map + 1, y, g.bf16, y.mn ? g.k_rows : BN / CG);
    };
    if (!encode(p.map, g0, a, b)) return cudaErrorInvalidValue;
    if (g1) {
        p.g[1] = *g1;
        set_tiles<CG, BN>(p.g[1], *a2, *b2, 1);
        p.groups = 2;
        const uint32_t c0 = g0.k_blocks + kTileCost, c1 = p.g[1].k_blocks + kTileCost;
        p.early = (c0 + c1 / 2) / c1;
        tiles += p.g[1].tiles;
        if (!encode(p.map + 2, p.g[1], *a2, *b2)) return cudaErrorInvalidValue;
    }
    const uint32_t slots = (uint32_t)sm_count / CG;
    return launch_plan<CG, BN, GemmPlan, Epi>(chain, p, ea, tiles < slots ? tiles : slots, st);
}

// Which tile for a product on its own: pairs of blocks on 256 x 256, or single blocks on 128 x 128.  Both take about 620 cycles a stage
// at an SM, because 32 KB of operands a stage come from L2 at 50 bytes a cycle: measured 617 (pair; its products alone take 512) and 636
// (570 for the pair since the feeding threads are elected; the choice keeps the figures it was made with).  The
// pair does twice the work per SM in that time; the small tile ends sooner (its epilogue and start take about 7000 cycles, the pair's
// 12,000, measured with K = 64) and spreads a small product over more SMs.  The one whose last wave ends first wins.
inline bool wide_tiles(uint64_t M, uint64_t N, uint64_t stages, int sm_count) {
    auto count = [&](uint64_t t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
    const uint64_t slots = (uint64_t)sm_count;
    const uint64_t wide = (count(256) + slots / 2 - 1) / (slots / 2) * stages * 620 + 12000;
    const uint64_t small = (count(128) + slots - 1) / slots * stages * 620 + 7000;
    return wide <= small;
}

}  // namespace sk
