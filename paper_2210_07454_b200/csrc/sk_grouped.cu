// Matrix products grouped by expert: group g's rows of x (offsets[g] .. offsets[g + 1], sizes known on the device only) times matrix g.
//
//   y_i = W_g x_i;   dx_i = W_g^T dy_i;   dW_g = sum over the group's rows of dy_i x_i^T
//
// Bound by the tensor cores (2 rows width out flops a product), by reading the matrices that have a row where there are few, and for dW by
// writing it (a plain fill of memory runs at 3.9 TB/s here, a copy at 6.5).
//
// y and dx: the matrix is the first operand, with 128 or 256 of the output's columns in a tile, and the rows of the group are the second, so that
// a tile ends within 15 (31) rows of its group's end: the matrix instruction has as many columns as the tile has rows, rounded up to 16 (pairs of
// blocks: 32), and only those rows are copied. (With rows of x as the first operand a group of 300 rows takes two tiles of 256, of which 41 % are
// nobody's.) A group's rows are shared out evenly among its tiles. The tile comes out transposed and is turned round on its way through shared
// memory. Every block makes the list of tiles for itself, from the offsets, in shared memory.
// 16384 x 768 x 2048 in one group 38 us (1.36 PFLOP/s), in 32 groups of 102 to 1684 rows 48; 16 groups of 4096 x 2048 197 (1.4); a row for each of 64
// experts of 2048 x 2048 83, reading 537 MB (6.5 TB/s); 64 rows drawn for 34 of them 48 (285 MB).
//
// dW: a tile of W_g, K the group's rows. The last stage of a group is copied in boxes of 32, 16, ... 1 rows, and what is missing to the 16
// rows of a matrix instruction comes as zeros from behind the last row of the matrix: rows of the next group, which may hold
// anything, never reach shared memory. 32 groups as above 53 us, in 32 bits 65; 64 matrices of 2048 x 2048 from a row each 139, writing 537 MB
// (3.9 TB/s), of which 34 have a row 123.
//
// Rows that TMA cannot address (a base off the 16-byte boundary, or rows no multiple of 16 bytes apart) are copied first.
#include "sk_gemm.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint32_t kSegments = kMaxGroups + 2;       // the groups, the rows before the first and behind the last
constexpr uint32_t kTableWords = 2 * (kSegments + 1);

// What the tensor cores truncate grows with the length of a sum: 6.5e-9 of a sum of one sign for each of its products (32768 to 1048576 of them), so that it would pass the half step
// of an fp16 output (4.9e-4) beyond 75000, of a bf16 one (3.9e-3) beyond 600000. Sums longer than these, where it is less than half of that, are taken in parts of kPartStages
// stages, which the epilogue adds up with rounding; for dW it goes by all rows together, and those of fp16 and fp32 are always in parts. 4096 rows of 4 groups of 32832 x 4096 fp16
// 870 -> 1050 us so, 2048 of 2 of 131136 x 2048 bf16 755 -> 1005 (in tiles of single blocks); dW of 131073 rows, 768 x 2048, 296 -> 298 in 32 groups, 400 -> 421 in 256.
constexpr uint32_t kPartStages = 16;
constexpr uint64_t long_sum(bool bf16) { return bf16 ? 131072 : 32768; }

// A boundary of a group as the kernels take it: never outside 0..rows, whatever the offsets hold. (Offsets that decrease: the plans differ in what they make of them, nothing is read or
// written outside the tensors.)
__device__ __forceinline__ uint32_t bounded(int64_t v, uint32_t rows) { return v < 0 ? 0 : v > (int64_t)rows ? rows : (uint32_t)v; }

// 16 rows of 64 bytes in shared memory (64-byte swizzle) to rows that begin anywhere: every row's aligned words, two rows at a time, then the values before
// and behind those, of all rows at once. (Single values throughout take twice the stores: dweight of 5001 rows of 1001 x 1500 53 us.)
__device__ __forceinline__ void store_unaligned(uint32_t at, uint16_t* o, uint64_t ld, uint32_t rows, uint32_t there) {
    const uint32_t lane = threadIdx.x & 31, c = lane & 15;
    const uint32_t odd0 = (uint32_t)((uintptr_t)o >> 1) & 1, step = (uint32_t)ld & 1;                  // row r begins off a word if odd0 + r step is odd
#pragma unroll
    for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t r = 2 * i + (lane >> 4), odd = (odd0 + r * step) & 1;
        uint32_t w;
        asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at + r * 64 + (((c >> 2) ^ (r >> 1 & 3)) << 4) + (c & 3) * 4) : "memory");
        const uint32_t next = __shfl_down_sync(0xffffffffu, w, 1);
        if (odd) w = __byte_perm(w, next, 0x5432);   // columns 2 c + 1 and 2 c + 2
        if (r < rows && 2 * c + odd + 1 < there && !(odd && c == 15)) *(uint32_t*)(o + r * ld + 2 * c + odd) = w;
    }
    const uint32_t r = c, odd = (odd0 + r * step) & 1, last = there - 1, col = lane < 16 ? 0 : last;
    if (r < rows && (lane < 16 ? odd : (there - odd) & 1)) {
        uint16_t w;
        asm volatile("ld.shared.b16 %0, [%1];" : "=h"(w) : "r"(at + r * 64 + (((col >> 3) ^ (r >> 1 & 3)) << 4) + (col & 7) * 2) : "memory");
        o[r * ld + col] = w;
    }
}

// A warp holds 32 output columns (rows of the transposed tile) and takes 32 of the group's rows at a time, as fragments that the transposing stores to shared
// memory turn round: 16 rows of 64 bytes are written as one box by the copy engine, or, where it cannot write (the last rows of a group, outputs it cannot address),
// by the lanes.  Two boxes take turns.
struct RowsEpi {
    static constexpr uint32_t kBox = 1024;
    static constexpr int kWarps = 8, kWords = (kTableWords + 7) / 8 + 2 * kBox / 4 + 32;      // the list of tiles, then the boxes, each on a 512-byte boundary
    static constexpr bool kParts = false, kInterleaved = true;
    struct Args { CUtensorMap map; uint16_t* out; uint64_t ld; uint32_t bf16, align, by_box; };
    const Args& a;
    const RaggedJob& t;
    uint32_t first, box, turn = 0;
    __device__ RowsEpi(const Args& a_, const RaggedJob& t_, uint32_t row, uint32_t, uint32_t stage) : a(a_), t(t_), first(row - (threadIdx.x & 31)) {
        const uint32_t w = (threadIdx.x >> 5) - 2, memory = stage - w * kWords * 4;            // of all warps
        box = ((memory + kTableWords * 4 + 511) & ~511u) + w * 2 * kBox;
    }
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) {
        finish();                                    // the boxes are free
        return true;
    }
    __device__ static void finish() {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    // the warps that share a column take turns, 32 rows each: of a tile of few rows both have some
    __device__ static uint32_t column(const RaggedJob&, uint32_t part, uint32_t c, uint32_t, uint32_t) { return 2 * c + 32 * part; }
    __device__ static void load(uint32_t addr, float (&v)[32]) {
        tmem_load_fragments(addr, v, 0);
        tmem_load_fragments(addr + (16u << 16), v, 16);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    }
    __device__ void chunk(uint32_t col, float (&v)[32], bool) {
        if (first >= t.M) return;
        const uint32_t lane = threadIdx.x & 31, rows = t.N - col;
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {           // 16 rows each
            if (16 * h >= rows) break;
            const uint32_t at = box + (turn & 1) * kBox;
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");      // all but the other box' copy
            __syncwarp();
            ++turn;
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j) {       // eight rows: four blocks of eight columns, one to every eight lanes' addresses
                const uint32_t row = 8 * j + (lane & 7), to = at + row * 64 + (((lane >> 3) ^ (row >> 1 & 3)) << 4), i = 8 * h + 4 * j;
                asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(pack16(v[i], v[i + 1], a.bf16)),
                             "r"(pack16(v[i + 2], v[i + 3], a.bf16)), "r"(pack16(v[16 + i], v[17 + i], a.bf16)), "r"(pack16(v[18 + i], v[19 + i], a.bf16)) : "memory");
            }
            if (a.by_box && rows >= 16 * h + 16) {
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0)
                    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(&a.map), "r"(first),
                                 "r"(t.first + col + 16 * h), "r"(0), "r"(at) : "memory");
            } else {
                __syncwarp();
                by_lanes(at, t.first + col + 16 * h, rows - 16 * h < 16 ? rows - 16 * h : 16);
            }
            if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");           // an empty one too: they are counted
        }
    }
    __device__ void end() {}
    __device__ void nothing(uint32_t part, uint32_t cols, uint32_t bn, uint32_t) {
        float v[32] = {};
#pragma unroll 1
        for (uint32_t c = 0; c < cols && column(t, part, c, cols, bn) < t.N; c += 32) chunk(column(t, part, c, cols, bn), v, false);
    }
    // `rows` rows of the box at `at` to rows from `row` on, neighbouring lanes at neighbouring addresses: 16 bytes each, 4 or 2, as the rows are aligned
    __device__ __forceinline__ void by_lanes(uint32_t at, uint32_t row, uint32_t rows) {
        const uint32_t lane = threadIdx.x & 31;
        uint16_t* o = a.out + (uint64_t)row * a.ld + first;
        const uint32_t there = min(t.M - first, 32u);            // columns
        if (a.align == 16 && there == 32) {
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i) {
                const uint32_t r = 8 * i + (lane >> 2), c = lane & 3;
                if (r < rows) *(uint4*)(o + r * a.ld + 8 * c) = load_shared16(at + r * 64 + ((c ^ (r >> 1 & 3)) << 4));
            }
        } else if (a.align >= 4) {
            const uint32_t c = lane & 15;                        // a pair of columns
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) {
                const uint32_t r = 2 * i + (lane >> 4);
                uint32_t w;
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w) : "r"(at + r * 64 + (((c >> 2) ^ (r >> 1 & 3)) << 4) + (c & 3) * 4) : "memory");
                if (r < rows && 2 * c < there) {
                    if (2 * c + 1 < there) *(uint32_t*)(o + r * a.ld + 2 * c) = w;
                    else o[r * a.ld + 2 * c] = (uint16_t)w;
                }
            }
        } else {
            store_unaligned(at, o, a.ld, rows, there);
        }
        __syncwarp();
    }
};

// y (or dx) by tiles of BN rows of the ragged side and 128 CG columns of the output
template <int CG, int BN>
struct RowsPlan {
    CUtensorMap matrix, rows_map[4];                 // boxes of 128, 64, 32 and 16 rows
    const int64_t* offsets;
    uint32_t groups, rows, features, tiles_m;        // tiles_m: of the features
    uint32_t k_stages, last_k;                       // K is the same for all tiles
    uint32_t beside;                                 // no
    uint32_t slices, each;                           // of K, and their stages
    uint32_t mn, k_rows, bf16, fill;                 // mn: the matrix is read along its rows; fill: rows of no group become zero
    uint32_t withheld;                               // see k_gemm
    Waits waits;
    static constexpr bool kCooperative = false, kEmpty = false, kThree = false, kRagged = true;
    static constexpr uint32_t kStep = 16 * CG;       // of a tile's rows: a block's own are whole groups of eight, as the swizzle has them, and more

    // In shared memory: where each segment begins, and the number of tiles before it.  Segment 0 is what lies before the first group.
    __device__ void prepare(void* memory) const {
        uint32_t *begin = (uint32_t*)memory, *before = begin + kSegments + 1;
        for (uint32_t g = threadIdx.x; g <= groups; g += blockDim.x) begin[g + 1] = bounded(offsets[g], rows);
        if (threadIdx.x == 0) {
            begin[0] = 0;
            begin[groups + 2] = rows;
        }
        __syncthreads();
        if (threadIdx.x >= 32) return;
        const uint32_t lane = threadIdx.x, segments = groups + 2;
        uint32_t top = 0, tiles = 0;                 // of all before this round
        for (uint32_t at = 0; at < segments; at += 32) {
            const uint32_t i = at + lane;
            // the round's beginnings, made never to decrease, and the next one's first
            uint32_t b = i <= segments ? begin[i] : rows, e = i < segments ? begin[i + 1] : rows;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, b, o), v = __shfl_up_sync(0xffffffffu, e, o);
                if (lane >= o) { b = max(b, u); e = max(e, v); }
            }
            b = max(b, top);
            e = max(e, b);
            const bool counts = i < segments && (fill || (i > 0 && i <= groups));
            const uint32_t mine = counts ? (e - b + BN - 1) / BN * tiles_m * slices : 0;
            uint32_t sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += u;
            }
            __syncwarp();
            if (i < segments) {
                begin[i] = b;
                before[i] = tiles + sum - mine;
            }
            top = __shfl_sync(0xffffffffu, b, 31);
            tiles += __shfl_sync(0xffffffffu, sum, 31);
            __syncwarp();
        }
        if (lane == 0) before[segments] = tiles;
    }
    __device__ __forceinline__ bool job(uint32_t p, uint32_t units, uint32_t i, RaggedJob& j) const {
        const uint32_t *begin = table(), *before = begin + kSegments + 1, t = p + i * units, segments = groups + 2;
        if (t >= before[segments]) return false;
        uint32_t low = 0, high = segments;           // before[low] <= t < before[high]
        while (high - low > 1) {
            const uint32_t middle = (low + high) / 2;
            if (before[middle] <= t) low = middle;
            else high = middle;
        }
        const uint32_t from = begin[low], length = begin[low + 1] - from, all = t - before[low], slice = all % slices, q = all / slices, tile = q / tiles_m;
        const uint32_t count = (length + BN - 1) / BN, each = ((length + count - 1) / count + kStep - 1) & ~(kStep - 1);
        const bool real = low > 0 && low <= groups;
        j.M = features;
        j.m = q - tile * tiles_m;
        j.n = 0;
        j.first = from + tile * each;
        j.N = min(each, length - tile * each);
        j.cols = (j.N + kStep - 1) & ~(kStep - 1);
        j.z = (int)low - 1;
        j.slice = slice;
        j.k_first = (int)(slice * this->each * kGemmK);
        j.k_stages = real ? min(this->each, k_stages - slice * this->each) : 0;
        j.last_rows = (slice + 1) * this->each >= k_stages ? last_k : kGemmK;
        j.k_rows = k_rows;
        j.a_mn = mn;
        j.b_mn = 0;
        j.bf16 = bf16;
        j.part = kPartStages;
        return true;
    }
    __device__ __forceinline__ const uint32_t* table() const {
        extern __shared__ uint8_t smem_raw[];
        const uint32_t base = smem_u32(smem_raw), first = ((base + 1023u) & ~1023u) - base;
        return (const uint32_t*)(smem_raw + first + kTableOffset);
    }
    static constexpr uint32_t kTableOffset = (232448 - RowsEpi::kWarps * RowsEpi::kWords * 4 - 1536) / (128 * 128 + BN / CG * 128) * (128 * 128 + BN / CG * 128);
    // The rows come in two boxes at most: a thread has a stage's time, some 600 cycles, for all it does, and a third copy costs more of it than 16 rows too
    // many cost to bring (112 rows are fetched as 128).
    struct Feed {
        const CUtensorMap *matrix, *first_map, *second_map;
        int feature, z, row, k_first;
        uint32_t first, total, mn;
        __device__ __forceinline__ Feed(const RowsPlan& p, const RaggedJob& j, uint32_t rank) {
            const uint32_t mine = j.cols / CG;       // a multiple of 16: the swizzle's groups of eight rows stay whole
            uint32_t q = __clz(mine) - 24;           // the largest power of two in it: 128 >> q
            uint32_t second = mine - (128 >> q);
            if (second & (second - 1)) {             // not a power of two: 112 only
                --q;
                second = 0;
            }
            first = 128 >> q;
            total = 128 * ((p.mn ? 2 * p.k_rows : 128) + first + second);
            first_map = &p.rows_map[q];
            second_map = second ? &p.rows_map[__clz(second) - 24] : nullptr;
            matrix = &p.matrix;
            mn = p.mn;
            feature = (int)(j.m * (128 * CG) + rank * 128);
            z = j.z;
            row = (int)(j.first + rank * mine);
            k_first = j.k_first;
        }
        __device__ __forceinline__ uint32_t bytes(uint32_t) const { return total; }
        __device__ __forceinline__ void copy(uint32_t k, uint32_t sa, uint32_t sb, uint32_t bar) const {
            const int k0 = k_first + (int)(k * kGemmK);
            if (mn) {
                tma_load<CG>(sa, matrix, bar, feature, k0, z);
                tma_load<CG>(sa + 8192, matrix, bar, feature + 64, k0, z);
            } else {
                tma_load<CG>(sa, matrix, bar, k0, feature, z);
            }
            tma_load<CG>(sb, first_map, bar, k0, row, 0);
            if (second_map) tma_load<CG>(sb + first * 128, second_map, bar, k0, row + (int)first, 0);
        }
    };
    __device__ __forceinline__ bool wait(const TileJob&) const { return true; }
    __device__ __forceinline__ void done(const TileJob&) const {}
    __device__ __forceinline__ const CUtensorMap* descriptor(uint32_t i) const { return i == 0 ? &matrix : i < 5 ? &rows_map[i - 1] : nullptr; }
};

// The tile written by the lanes, which hold an output column each, so that a warp writes 32 neighbouring ones of a row. Where there are few tiles and K is long, it is split:
// slices' sums in 32 bits, rows and columns as in the output, joined by k_grouped_sum. FINAL: the output itself, of sums that are taken in parts (PARTS, see long_sum), whose
// epilogue is nothing beside their length.
template <bool PARTS, bool FINAL>
struct LanesEpi {
    static constexpr int kWarps = RowsEpi::kWarps, kWords = RowsEpi::kWords;
    static constexpr bool kParts = PARTS, kInterleaved = !PARTS;
    using Out = std::conditional_t<FINAL, uint16_t, float>;
    struct Args { Out* out; uint64_t ld, stride; uint32_t bf16; };           // stride: from slice to slice
    const Args& a;
    const RaggedJob& t;
    uint32_t feature;
    __device__ LanesEpi(const Args& a_, const RaggedJob& t_, uint32_t row, uint32_t, uint32_t) : a(a_), t(t_), feature(row) {}
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) { return true; }
    __device__ static void finish() {}
    __device__ static uint32_t column(const RaggedJob& t, uint32_t part, uint32_t c, uint32_t cols, uint32_t bn) {
        return PARTS ? part * cols + c : RowsEpi::column(t, part, c, cols, bn);
    }
    __device__ static void load(uint32_t addr, float (&v)[32]) { tmem_load32(addr, v); }
    __device__ void chunk(uint32_t col, float (&v)[32], bool) {
        Out* o = a.out + (FINAL ? 0 : t.slice * a.stride) + (uint64_t)(t.first + col) * a.ld + feature;
        const uint32_t rows = t.N - col;
        if (feature < t.M) {
#pragma unroll
            for (uint32_t i = 0; i < 32; ++i)
                if (i < rows) {
                    if constexpr (FINAL) o[i * a.ld] = (uint16_t)pack16(v[i], 0.0f, a.bf16);
                    else o[i * a.ld] = v[i];
                }
        }
        __syncwarp();
    }
    __device__ void end() {}
    __device__ void nothing(uint32_t part, uint32_t cols, uint32_t bn, uint32_t) {           // rows of no group: slices leave them to what joins them
        if constexpr (FINAL) {
            float v[32] = {};
#pragma unroll 1
            for (uint32_t c = 0; c < cols && column(t, part, c, cols, bn) < t.N; c += 32) chunk(column(t, part, c, cols, bn), v, false);
        }
    }
};
// The slices in order, a thread a value. Rows of no group become zero with fill, else stay.
__global__ void __launch_bounds__(256) k_grouped_sum(const float* sums, uint64_t ld_sums, uint64_t stride, uint32_t slices, const int64_t* offsets, uint32_t groups,
                                                     uint32_t rows, uint32_t cols, uint16_t* out, uint64_t ld, int bf16, int fill) {
    chain_acquire();
    const uint32_t col = blockIdx.x * 256 + threadIdx.x, from = bounded(offsets[0], rows), to = bounded(offsets[groups], rows);
    if (col >= cols) return;
    for (uint32_t r = blockIdx.y; r < rows; r += gridDim.y) {
        float v = 0;
        if (r >= from && r < to) {
            const float* p = sums + r * ld_sums + col;
            v = *p;
#pragma unroll 8
            for (uint32_t s = 1; s < slices; ++s) v += p[s * stride];
        } else if (!fill) {
            continue;
        }
        out[r * ld + col] = (uint16_t)pack16(v, 0.0f, bf16);
    }
}

// dW by tiles of 128 CG x BN of every matrix, the longest groups first; units take them up and down in turn, so that what one has too much in one round
// it has too little in the next (in the groups' own order, 32 groups of 16384 rows kept one pair of blocks busy for 82,000 cycles and another for 55,000).
// Where there are few tiles, K is split: the longest slice is made as short as it can be with as many slices as there are units, or twice as many. A group
// in several slices leaves their sums in 32 bits in the workspace, and k_grouped_join adds them up in order.
constexpr uint32_t kSorted = 256;                    // groups that are put in order, and may be split
constexpr uint32_t kShortest = 8;                    // stages of a slice: it has to be worth its epilogue and its way through the workspace
template <int CG, int BN>
struct MatrixPlan {
    CUtensorMap a[7], b[7];                          // dy and x, boxes of 64, 32, ... 1 rows
    const int64_t* offsets;
    uint32_t groups, rows, M, N, tiles_m, tiles_n, bf16;
    uint32_t most_slices;                            // of all groups together; 0: none is split
    uint32_t beside;                                 // it may run beside the kernel before it, the product that gives dx
    uint32_t* slices;                                // for each group their number, and that of the first one's sums
    uint32_t withheld;                               // see k_gemm
    Waits waits;
    static constexpr bool kCooperative = false, kEmpty = false, kThree = false, kRagged = true;
    struct Table { uint16_t order[kSorted], first[kSorted + 1]; };       // groups by length, slices before each
    __device__ static Table& table() {
        __shared__ Table t;
        return t;
    }
    // from L2: a kernel that begins beside the one before it has not passed the wait at which a first-level cache is sure to hold nothing old
    __device__ __forceinline__ uint32_t border(uint32_t g) const { return bounded((int64_t)__ldcg((const long long*)offsets + g), rows); }
    __device__ __forceinline__ uint32_t length(uint32_t g) const {
        const uint32_t from = border(g), to = border(g + 1);
        return to > from ? to - from : 0;
    }
    __device__ void prepare(void* memory) const {
        if (groups > kSorted) return;
        uint32_t *stages = (uint32_t*)memory, *sorted = stages + kSorted;
        for (uint32_t g = threadIdx.x; g < groups; g += blockDim.x) stages[g] = (length(g) + kGemmK - 1) / kGemmK;
        __syncthreads();
        for (uint32_t g = threadIdx.x; g < groups; g += blockDim.x) {
            uint32_t rank = 0;
            for (uint32_t h = 0; h < groups; ++h) rank += stages[h] > stages[g] || (stages[h] == stages[g] && h < g);
            table().order[rank] = (uint16_t)g;
            sorted[rank] = stages[g];
        }
        __syncthreads();
        if (threadIdx.x >= 32) return;
        const uint32_t lane = threadIdx.x, most = sorted[0];
        auto count = [&](uint32_t longest) {         // slices, if none may be longer
            uint32_t n = 0;
            for (uint32_t r = lane; r < groups; r += 32) n += (sorted[r] + longest - 1) / longest;
            return __reduce_add_sync(0xffffffffu, n);
        };
        uint32_t longest = max(most, 1u), best = ~0u;
        if (most_slices) {
            const uint32_t units = gridDim.x / CG, per = tiles_m * tiles_n;
            for (uint32_t rounds = 1; rounds <= 2; ++rounds) {
                const uint32_t fit = min(rounds * units / per, most_slices);
                uint32_t low = 1, high = max(most, 1u);              // the least length that fits, if any does
                if (count(high) > fit) continue;
                while (low < high) {
                    const uint32_t middle = (low + high) / 2;
                    if (count(middle) <= fit) high = middle;
                    else low = middle + 1;
                }
                low = max(low, min(kShortest, max(most, 1u)));
                const uint32_t cost = rounds * (low + kTileCost);
                if (cost < best) {
                    best = cost;
                    longest = low;
                }
            }
        }
        uint32_t before = 0;
        for (uint32_t at = 0; at < groups; at += 32) {
            const uint32_t r = at + lane, mine = r < groups ? max((sorted[r] + longest - 1) / longest, 1u) : 0;
            uint32_t sum = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += u;
            }
            if (r < groups) {
                table().first[r] = (uint16_t)(before + sum - mine);
                if (most_slices && blockIdx.x == 0) *(uint2*)(slices + 2 * table().order[r]) = make_uint2(mine, before + sum - mine);
            }
            before += __shfl_sync(0xffffffffu, sum, 31);
        }
        if (lane == 0) table().first[groups] = (uint16_t)before;
    }
    __device__ __forceinline__ bool job(uint32_t p, uint32_t units, uint32_t i, RaggedJob& j) const {
        const uint32_t t = i * units + (i & 1 ? units - 1 - p : p), per = tiles_m * tiles_n, c = t / per, q = t - c * per;
        uint32_t g = c, slice = 0, count = 1;
        if (groups <= kSorted) {
            const Table& order = table();
            if (c >= order.first[groups]) return false;
            uint32_t low = 0, high = groups;         // first[low] <= c < first[high]
            if (order.first[groups] == groups) {
                low = c;
            } else {
                while (high - low > 1) {
                    const uint32_t middle = (low + high) / 2;
                    if (order.first[middle] <= c) low = middle;
                    else high = middle;
                }
            }
            g = order.order[low];
            slice = c - order.first[low];
            count = order.first[low + 1] - order.first[low];
        }
        if (g >= groups) return false;
        const uint32_t from = border(g), rest = length(g), stages = (rest + kGemmK - 1) / kGemmK, each = (stages + count - 1) / count;
        const uint32_t valid = min(rest - slice * each * kGemmK, each * kGemmK);
        j.M = M;
        j.N = N;
        j.n = q / tiles_m;
        j.m = q - j.n * tiles_m;
        j.b = g;
        j.slice = count > 1 ? c + 1 : 0;             // c: what is split comes first, so this is the number of the slice among those of all groups
        j.first = from + slice * each * kGemmK;
        j.cols = BN;
        j.k_stages = (valid + kGemmK - 1) / kGemmK;
        j.last_valid = valid - (j.k_stages ? j.k_stages - 1 : 0) * kGemmK;
        j.last_rows = (j.last_valid + 15) & ~15u;
        j.k_rows = kGemmK;
        j.a_mn = j.b_mn = 1;
        j.bf16 = bf16;
        j.part = kPartStages;
        return true;
    }
    struct Feed {
        const MatrixPlan& p;
        int m, n, row, rows;
        uint32_t stages, last_valid, last_rows;
        static constexpr int kRows = BN / CG;
        __device__ __forceinline__ Feed(const MatrixPlan& p_, const RaggedJob& j, uint32_t rank)
            : p(p_), m((int)(j.m * (128 * CG) + rank * 128)), n((int)(j.n * BN + rank * kRows)), row((int)j.first), rows((int)p_.rows), stages(j.k_stages),
              last_valid(j.last_valid), last_rows(j.last_rows) {}
        __device__ __forceinline__ uint32_t bytes(uint32_t k) const { return 128 * (2 + kRows / 64) * (k + 1 == stages ? last_rows : kGemmK); }
        // rows from `from` on (a box of 64 >> q) to row `at` of the stage
        __device__ __forceinline__ void box(uint32_t q, int from, uint32_t at, uint32_t sa, uint32_t sb, uint32_t bar) const {
#pragma unroll
            for (int i = 0; i < 2; ++i) tma_load<CG>(sa + i * 8192 + at * 128, &p.a[q], bar, m + 64 * i, from, 0);
#pragma unroll
            for (int i = 0; i < kRows / 64; ++i) tma_load<CG>(sb + i * 8192 + at * 128, &p.b[q], bar, n + 64 * i, from, 0);
        }
        __device__ __forceinline__ void copy(uint32_t k, uint32_t sa, uint32_t sb, uint32_t bar) const {
            const int from = row + (int)(k * kGemmK);
            if (k + 1 < stages || last_valid == kGemmK) {
                box(0, from, 0, sa, sb, bar);
                return;
            }
            uint32_t at = 0;
            for (uint32_t q = 1; q < 7; ++q)             // large boxes first: each begins at a multiple of its size
                if (last_valid & (64u >> q)) {
                    box(q, from + (int)at, at, sa, sb, bar);
                    at += 64u >> q;
                }
            for (uint32_t q = 6; at < last_rows; --q)    // zeros up to a multiple of 16, small boxes first
                if (at & (64u >> q)) {
                    box(q, rows, at, sa, sb, bar);
                    at += 64u >> q;
                }
        }
    };
    __device__ __forceinline__ bool wait(const TileJob&) const { return true; }
    __device__ __forceinline__ void done(const TileJob&) const {}
    __device__ __forceinline__ const CUtensorMap* descriptor(uint32_t i) const { return i < 7 ? &a[i] : i < 14 ? &b[i - 7] : nullptr; }
};

// A lane holds a row of the output and 32 of its columns. They go out in boxes of 32 rows through the copy engine, 16-bit ones from two boxes in turn, or, where
// that cannot write and for the sums of slices, by the lanes.
template <bool PARTS>
struct MatrixEpi {
    static constexpr int kWarps = 8, kWords = kStageWords;
    static constexpr bool kParts = PARTS, kInterleaved = false;
    // zeros: where a matrix without rows is one run of values, else null
    struct Args { CUtensorMap map; void* out; uint64_t ld, stride; int type; uint32_t align, by_box; float* sums; uint64_t ld_sums; uint8_t* zeros; uint64_t zeros_stride; };
    const Args& a;
    const RaggedJob& t;
    uint32_t row0, rows, stage, turn = 0;
    __device__ MatrixEpi(const Args& a_, const RaggedJob& t_, uint32_t row, uint32_t, uint32_t stage_)
        : a(a_), t(t_), row0(row - (threadIdx.x & 31)), stage(stage_) { rows = row0 >= t.M ? 0 : t.M - row0 < 32 ? t.M - row0 : 32; }
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) {
        finish();                                    // the boxes are free
        return true;
    }
    __device__ static void finish() {
        if ((threadIdx.x & 31) == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    }
    __device__ static uint32_t column(const RaggedJob& t, uint32_t part, uint32_t c, uint32_t cols, uint32_t bn) { return t.n * bn + part * cols + c; }
    __device__ static void load(uint32_t addr, float (&v)[32]) { tmem_load32(addr, v); }
    __device__ void chunk(uint32_t col, float (&v)[32], bool last) {
        if (!rows) return;
        if (t.slice) {
            store_tile32(a.sums + (uint64_t)(t.slice - 1) * t.M * a.ld_sums, SK_F32, a.ld_sums, row0, rows, col, (uint32_t)a.ld_sums, v, 16, stage, false, last);
        } else if (!a.by_box && (a.type == SK_F32 || a.align >= 4)) {
            store_tile32((uint8_t*)a.out + t.b * a.stride * (a.type == SK_F32 ? 4 : 2), a.type, a.ld, row0, rows, col, t.N, v, a.align, stage, true, last);
        } else {
            const uint32_t lane = threadIdx.x & 31;
            uint32_t at = stage;
            if (a.type == SK_F32) {
                finish();
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    store_shared16(at + lane * 128 + ((i ^ (lane & 7)) << 4), make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]),
                                                                                         __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])));
            } else {
                at += (turn++ & 1) * 2048;
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");  // all but the other box' copy
                __syncwarp();
                const bool bf16 = a.type == SK_BF16;
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i)
                    store_shared16(at + lane * 64 + ((i ^ (lane >> 1 & 3)) << 4), make_uint4(pack16(v[8 * i], v[8 * i + 1], bf16), pack16(v[8 * i + 2], v[8 * i + 3], bf16),
                                                                                             pack16(v[8 * i + 4], v[8 * i + 5], bf16), pack16(v[8 * i + 6], v[8 * i + 7], bf16)));
            }
            if (!a.by_box) {
                __syncwarp();
                uint16_t* o = (uint16_t*)a.out + t.b * a.stride + (uint64_t)row0 * a.ld + col;
                const uint32_t there = min(t.N - col, 32u);
                store_unaligned(at, o, a.ld, min(rows, 16u), there);
                if (rows > 16) store_unaligned(at + 1024, o + 16 * a.ld, a.ld, rows - 16, there);
                __syncwarp();
                return;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(&a.map), "r"(col), "r"(row0), "r"(t.b), "r"(at)
                             : "memory");
                asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
        }
    }
    __device__ void end() {}
    // A tile of a matrix without rows: zeros, written as a part of the whole run (in boxes of 64 bytes, rows whose length is no multiple of 32 bytes go out at 2.2 TB/s)
    __device__ void nothing(uint32_t part, uint32_t cols, uint32_t bn, uint32_t rank) {
        if (!a.zeros) {
            float v[32] = {};
#pragma unroll 1
            for (uint32_t c = 0; c < cols; c += 32) {
                const uint32_t col = column(t, part, c, cols, bn);
                if (col < t.N) chunk(col, v, c + 32 == cols || col + 32 >= t.N);
            }
            return;
        }
        const uint32_t lane = threadIdx.x & 31, high = bn == 256 ? 256 : 128, tiles_m = (t.M + high - 1) / high, tiles = tiles_m * ((t.N + bn - 1) / bn);
        const uint32_t units = tiles * (bn == 256 ? 2 : 1) * kWarps, unit = ((t.n * tiles_m + t.m) * (bn == 256 ? 2 : 1) + rank) * kWarps + (threadIdx.x >> 5) - 2;
        const uint64_t size = a.type == SK_F32 ? 4 : 2, total = (uint64_t)t.M * t.N * size, each = (total / units + 512) / 512 * 512;
        const uint64_t from = unit * each;
        if (from >= total) return;
        uint8_t *p = a.zeros + t.b * a.zeros_stride + from, *end = p + (total - from < each ? total - from : each);
        uint8_t* whole = (uint8_t*)(((uintptr_t)p + 15) & ~(uintptr_t)15);           // from here on 16 bytes at a time
        if (p + 2 * lane < whole && p + 2 * lane < end) *(uint16_t*)(p + 2 * lane) = 0;
        for (whole += 16 * lane; whole + 16 <= end; whole += 512) *(uint4*)whole = make_uint4(0, 0, 0, 0);
        for (; whole < end && whole + 16 > end; whole += 16)                                // the lane that comes to the last piece
            for (uint8_t* q = whole; q < end; q += 2) *(uint16_t*)q = 0;
    }
};

// dW of the groups whose K was split: the sums of their slices in order, by a thread for four columns where that keeps the GPU busy, else by eight warps every eighth
// each and then those eight in order (2 groups of 30000 rows of 64 x 200: 30 us by single threads, 18; 16384 rows of 768 x 2048: 55, and 72 by eight warps).
constexpr uint64_t kManyQuads = 1 << 17;
__global__ void __launch_bounds__(256) k_grouped_join(const uint32_t* slices, const float* sums, uint64_t ld_sums, uint32_t M, uint32_t N, void* out, uint64_t ld,
                                                      uint64_t stride, int type) {
    __shared__ float4 part[8][32];
    chain_acquire();
    const uint32_t quads = (N + 3) / 4, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = blockIdx.y;
    const uint64_t total = (uint64_t)M * quads;
    const uint2 s = *(const uint2*)(slices + 2 * g);
    if (s.x < 2) return;
    const float* first = sums + (uint64_t)s.y * M * ld_sums;
    if (total >= kManyQuads) {
        for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < total; i += gridDim.x * 256ull) {
            const uint64_t row = i / quads;
            const uint32_t col = (uint32_t)(i - row * quads) * 4;
            const float* p = first + row * ld_sums + col;
            float4 v = *(const float4*)p;
#pragma unroll 4
            for (uint32_t k = 1; k < s.x; ++k) {
                const float4 w = *(const float4*)(p + (uint64_t)k * M * ld_sums);
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
            const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (col + e < N) store_as(out, type, g * stride + row * ld + col + e, f[e]);
        }
        return;
    }
    for (uint64_t i0 = blockIdx.x * 32ull; i0 < total; i0 += gridDim.x * 32ull) {
        const uint64_t i = i0 + lane, row = i / quads;
        const uint32_t col = (uint32_t)(i - row * quads) * 4;
        float4 v = make_float4(0, 0, 0, 0);
        if (i < total) {
#pragma unroll 4
            for (uint32_t k = warp; k < s.x; k += 8) {
                const float4 w = *(const float4*)(first + row * ld_sums + col + (uint64_t)k * M * ld_sums);
                v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            }
        }
        part[warp][lane] = v;
        __syncthreads();
        if (warp < 4) {                              // a value of the four each
            float f = 0;
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k) f += ((const float*)&part[k][0])[warp * 32 + lane];
            const uint64_t j = i0 + (warp * 32 + lane) / 4, r = j / quads;
            const uint32_t c = (uint32_t)(j - r * quads) * 4 + (lane & 3);
            if (j < total && c < N) store_as(out, type, g * stride + r * ld + c, f);
        }
        __syncthreads();
    }
}

// Rows of up to three batches of matrices copied to where TMA can address them, in one launch. A thread makes 16 bytes of a row out of the two aligned
// accesses that they lie in, wherever the row begins; at the ends of the tensor, where those would reach outside, and of a row, out of single values.
struct PackedOne {
    const uint16_t* src;
    uint16_t* dst;
    uint64_t ld, stride;
    uint32_t rows, matrices, cols, ld_dst, blocks;   // blocks: of each matrix
    const int64_t* offsets;                          // not null: only matrices whose group has rows
};
struct PackedArgs { PackedOne m[3]; uint32_t rows; };
constexpr uint32_t kPackEach = 4;                    // of a thread, on their way at once
__global__ void __launch_bounds__(256) k_grouped_pack(const __grid_constant__ PackedArgs a) {
    chain_acquire();
    uint32_t block = blockIdx.x, which = 0;
    while (block >= a.m[which].blocks * a.m[which].matrices) {
        block -= a.m[which].blocks * a.m[which].matrices;
        ++which;
    }
    const PackedOne& m = a.m[which];
    const uint32_t z = block / m.blocks;
    block -= z * m.blocks;
    if (m.offsets && bounded(m.offsets[z + 1], a.rows) <= bounded(m.offsets[z], a.rows)) return;
    const uint32_t pieces = m.ld_dst / 8;            // of 16 bytes in a row
    uint32_t lanes = 32;                             // that share a row: so many that its pieces keep them busy
    while (lanes > 1 && lanes / 2 >= pieces) lanes /= 2;
    const uint32_t lane = threadIdx.x & (lanes - 1), each = 256 / lanes;
    const uint64_t begin = (uint64_t)(uintptr_t)m.src, end = begin + ((m.matrices - 1) * m.stride + (m.rows - 1) * m.ld + m.cols) * 2;
    for (uint64_t r = (uint64_t)block * each + threadIdx.x / lanes; r < m.rows; r += (uint64_t)m.blocks * each) {
        const uint16_t* row = m.src + z * m.stride + r * m.ld;
        uint4* to = (uint4*)(m.dst + ((uint64_t)z * m.rows + r) * m.ld_dst);
        const uint32_t by = (uint32_t)(uintptr_t)row & 15, more = by ? 1 : 0, shift = (by & 2) * 8;
        const uint4* p = (const uint4*)((uintptr_t)row - by);
        // pieces [low, high) lie in whole accesses inside the tensor
        const uint32_t low = (uint64_t)(uintptr_t)p < begin, inside = (uint32_t)min((end - (uint64_t)(uintptr_t)p) / 16, (uint64_t)m.ld_dst);
        const uint32_t high = min(m.cols / 8, inside > more ? inside - more : 0);
        for (uint32_t c0 = lane; c0 < pieces; c0 += lanes * kPackEach) {
            uint4 x[kPackEach], y[kPackEach];
#pragma unroll
            for (uint32_t e = 0; e < kPackEach; ++e) {
                const uint32_t c = c0 + e * lanes;
                if (c >= low && c < high) {
                    x[e] = p[c];
                    y[e] = p[c + more];
                }
            }
#pragma unroll
            for (uint32_t e = 0; e < kPackEach; ++e) {
                const uint32_t c = c0 + e * lanes;
                if (c >= pieces) break;
                if (c >= low && c < high) {
                    uint32_t w[8] = {x[e].x, x[e].y, x[e].z, x[e].w, y[e].x, y[e].y, y[e].z, y[e].w};
                    if (by & 8) {
#pragma unroll
                        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                    }
                    if (by & 4) {
#pragma unroll
                        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                    }
                    to[c] = make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift), __funnelshift_r(w[2], w[3], shift),
                                       __funnelshift_r(w[3], w[4], shift));
                } else {
                    uint32_t v[8];
#pragma unroll
                    for (uint32_t i = 0; i < 8; ++i) v[i] = 8 * c + i < m.cols ? row[8 * c + i] : 0;
                    to[c] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
                }
            }
        }
    }
}

// M x N values from rows that the copy engine wrote, ld_src apart, to rows that begin anywhere, one behind the other: 16 aligned bytes at a time, out of the two
// accesses in which they lie, and the few values before and behind those one by one. (Written from the tiles, rows that are no multiple of 32 bytes leave at
// 0.6 to 2 TB/s: most sectors are written in two parts.) matrices: of the groups that have rows; else rows offsets[0] to offsets[groups] of one matrix, or,
// with fill, all of it.
struct UnpackArgs {
    const uint8_t* src;
    uint8_t* dst;
    const int64_t* offsets;
    uint64_t ld_src, M;
    uint32_t N, groups, rows, matrices, fill;            // matrices: dW; else y or dx
};
constexpr uint32_t kUnpackEach = 4;
template <int SIZE>
__global__ void __launch_bounds__(256) k_grouped_unpack(const __grid_constant__ UnpackArgs a) {
    using V = std::conditional_t<SIZE == 2, uint16_t, uint32_t>;
    constexpr uint32_t kN = 16 / SIZE;
    chain_acquire();
    const uint32_t g = blockIdx.y;
    uint32_t from = 0, to = (uint32_t)a.M;
    if (a.matrices) {
        if (bounded(a.offsets[g + 1], a.rows) <= bounded(a.offsets[g], a.rows)) return;
    } else if (!a.fill) {
        from = bounded(a.offsets[0], a.rows);
        to = bounded(a.offsets[a.groups], a.rows);
    }
    const uint32_t pieces = a.N / kN + 1;            // of a row, at most
    uint32_t lanes = 32;                             // that share a row
    while (lanes > 1 && lanes / 2 >= pieces) lanes /= 2;
    const uint32_t lane = threadIdx.x & (lanes - 1), each = 256 / lanes;
    for (uint64_t r = from + (uint64_t)blockIdx.x * each + threadIdx.x / lanes; r < to; r += (uint64_t)gridDim.x * each) {
        const V* src = (const V*)a.src + ((uint64_t)g * a.M + r) * a.ld_src;             // on a 16-byte boundary
        V* dst = (V*)a.dst + ((uint64_t)g * a.M + r) * a.N;
        const uint32_t head = min(((16 - (uint32_t)((uintptr_t)dst & 15)) & 15) / SIZE, a.N), whole = (a.N - head) / kN, by = head * SIZE, more = by ? 1 : 0;
        const uint4* p = (const uint4*)src;
        uint4* o = (uint4*)(dst + head);
        for (uint32_t i = lane; i < head; i += lanes) dst[i] = src[i];
        for (uint32_t i = head + whole * kN + lane; i < a.N; i += lanes) dst[i] = src[i];
        for (uint32_t c0 = lane; c0 < whole; c0 += lanes * kUnpackEach) {
            uint4 x[kUnpackEach], y[kUnpackEach];
#pragma unroll
            for (uint32_t e = 0; e < kUnpackEach; ++e) {
                const uint32_t c = c0 + e * lanes;
                if (c < whole) {                     // 16 bytes behind the last row may be read
                    x[e] = p[c];
                    y[e] = p[c + more];
                }
            }
#pragma unroll
            for (uint32_t e = 0; e < kUnpackEach; ++e) {
                const uint32_t c = c0 + e * lanes;
                if (c >= whole) break;
                uint32_t w[8] = {x[e].x, x[e].y, x[e].z, x[e].w, y[e].x, y[e].y, y[e].z, y[e].w};
                if (by & 8) {
#pragma unroll
                    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
                }
                if (by & 4) {
#pragma unroll
                    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
                }
                const uint32_t shift = (by & 2) * 8;
                o[c] = make_uint4(__funnelshift_r(w[0], w[1], shift), __funnelshift_r(w[1], w[2], shift), __funnelshift_r(w[2], w[3], shift),
                                  __funnelshift_r(w[3], w[4], shift));
            }
        }
    }
}

bool addressable(const void* p, uint64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }
// The copy engine writes whole pieces of 16 bytes: behind a row that ends inside one it puts zeros. What lies there is not the output's, unless the rows are the workspace's own.
bool by_boxes(const void* p, uint64_t ld_bytes, uint64_t stride_bytes, uint64_t row_bytes, bool own) {
    return ((uintptr_t)p | ld_bytes | stride_bytes) % 16 == 0 && (own || row_bytes % 16 == 0);
}

// Copies that a call needs, and where they lie in the workspace.
struct GroupedLayout {
    bool pack_x, pack_w, pack_dy;
    uint64_t ld_x, ld_w, ld_dy, off_x, off_w, off_dy, total;
    bool wide;                                       // tiles of dW
    uint32_t most_slices;                            // of the products that give dW, see MatrixPlan; 0: none is split
    uint64_t off_slices, off_sums, ld_sums;
    uint32_t slices;                                 // of K, of the product that gives y or dx
    uint64_t off_row_sums, ld_row_sums;
    bool unpack_rows, unpack_matrices;               // y or dx, dW: through the workspace, where rows are whole lines
    uint64_t ld_rows, ld_matrices, off_rows, off_matrices;
};
// An output goes through the workspace if it is one run of values, large enough for another launch, and its rows cannot be written by the copy engine (dW; 14 rows of 15 groups
// of 2822 x 832: 74 us from the tiles, 46 so) or not even in words (y and dx; 12928 rows of 2073: 68 and 58, but of 1954 61 and 65).
constexpr uint64_t kUnpackBytes = 4 << 20;
constexpr uint32_t kPlanSms = 148;                   // the slices, and with them the workspace, are planned for a B200
// How many slices all groups of dW may be cut into, 0: K is not split. Few groups of few tiles, rows enough to be worth another launch (4096 are some 19 us of one
// tile), and a slice's worth of them in a group of the mean length.
constexpr uint64_t kSplitRows = 4096;
uint64_t slices_of(const GroupedArgs& a, bool wide) {
    const uint64_t tile = wide ? 256 : 128, tiles = ((a.out + tile - 1) / tile) * ((a.width + tile - 1) / tile), most = 2 * (kPlanSms / (wide ? 2 : 1)) / tiles;
    return most >= 2 && most >= a.groups && a.groups <= kSorted && a.rows >= kSplitRows && a.rows >= a.groups * kShortest * kGemmK ? most : 0;
}
// Pairs of blocks or single ones: the one that is through first, at some 600 cycles a stage, if the groups are of one length (see wide_tiles for the constants).
bool wide_matrices(const GroupedArgs& a) {
    auto cycles = [&](bool wide) {
        const uint64_t tile = wide ? 256 : 128, units = kPlanSms / (wide ? 2 : 1), tiles = ((a.out + tile - 1) / tile) * ((a.width + tile - 1) / tile);
        const uint64_t stages = a.rows / kGemmK + a.groups;
        uint64_t longest = (a.groups * tiles + units - 1) / units * (stages / a.groups + kTileCost);
        if (slices_of(a, wide))
            for (uint64_t rounds = 1; rounds <= 2; ++rounds) {
                const uint64_t slices = rounds * units / tiles, each = slices >= a.groups ? rounds * (stages / slices + 1 + kTileCost) : longest;
                if (each < longest) longest = each;
            }
        return longest * 620 + (wide ? 12000 : 7000);
    };
    return cycles(true) <= cycles(false);
}
// Slices of K for y or dx. Single blocks with a tile each, if all the tiles there can be leave at least half of the SMs without work; a slice has kShortest stages or more, and what
// is saved, at some 350 cycles a stage of few rows, has to be worth another launch.
uint32_t row_slices(const GroupedArgs& a, uint64_t features, uint64_t k_stages) {
    const uint64_t live = a.groups < a.rows ? a.groups : a.rows, tiles = (a.rows / 128 + live) * ((features + 127) / 128);
    uint64_t slices = kPlanSms / tiles < k_stages / kShortest ? kPlanSms / tiles : k_stages / kShortest;
    if (slices < 2 || k_stages < 2 * kShortest) return 1;
    const uint64_t each = (k_stages + slices - 1) / slices;
    return (uint32_t)((k_stages + each - 1) / each);
}
GroupedLayout layout_of(const GroupedArgs& a, bool backward) {
    GroupedLayout l{};
    auto take = [&](bool pack, uint64_t rows, uint64_t ld) {
        const uint64_t at = l.total;
        if (pack) l.total += round_up(rows * ld * 2, 256);
        return at;
    };
    l.pack_x = !addressable(a.x, a.ld_x);
    l.pack_dy = backward && !addressable(a.dy, a.ld_dy);
    l.pack_w = !addressable(a.weight, a.ld_weight) || (a.groups > 1 && (a.stride_weight % 8 || !a.stride_weight));
    l.ld_x = round_up(a.width, 64);                  // whole 128-byte lines for what is read by every tile
    l.ld_dy = round_up(a.out, 64);
    l.ld_w = round_up(a.width, 8);
    l.off_x = take(l.pack_x, a.rows, l.ld_x);
    l.off_dy = take(l.pack_dy, a.rows, l.ld_dy);
    l.off_w = take(l.pack_w, a.groups * a.out, l.ld_w);
    if (backward) {
        l.wide = wide_matrices(a);
        l.most_slices = a.dweight ? (uint32_t)slices_of(a, l.wide) : 0;
        if (l.most_slices) {
            l.ld_sums = round_up(a.width, 32);
            l.off_slices = l.total;
            l.off_sums = l.off_slices + round_up(a.groups * 8, 256);
            l.total = l.off_sums + round_up(l.most_slices * a.out * l.ld_sums * 4, 256);
        }
        const uint64_t size = type_size(a.dweight_type), stride = a.groups > 1 ? a.stride_dweight : a.out * a.ld_dweight;
        if (a.dweight && a.ld_dweight == a.width && stride == a.out * a.width && ((uintptr_t)a.dweight | a.width * size) % 16 &&
            a.groups * a.out * a.width * size >= kUnpackBytes) {
            l.unpack_matrices = true;
            l.ld_matrices = round_up(a.width, 128 / size);
            l.off_matrices = l.total;
            l.total += round_up(a.groups * a.out * l.ld_matrices * size + 32, 256);      // 16 bytes may be read behind the last row
        }
    }
    const void* rows = backward ? a.dx : a.y;
    const uint64_t cols = backward ? a.width : a.out, ld = backward ? a.ld_dx : a.ld_y;
    l.slices = rows ? row_slices(a, cols, ((backward ? a.out : a.width) + kGemmK - 1) / kGemmK) : 1;
    if (l.slices > 1) {
        l.ld_row_sums = round_up(cols, 32);
        l.off_row_sums = l.total;
        l.total += round_up(l.slices * a.rows * l.ld_row_sums * 4, 256);
    } else if (rows && ld == cols && row_alignment(rows, ld, SK_BF16) < 4 && a.rows * cols * 2 >= kUnpackBytes) {
        l.unpack_rows = true;
        l.ld_rows = round_up(cols, 64);
        l.off_rows = l.total;
        l.total += round_up(a.rows * l.ld_rows * 2 + 32, 256);
    }
    return l;
}

// the operands as TMA can address them
int pack_operands(GroupedArgs& a, const GroupedLayout& l, int sm_count, cudaStream_t st) {
    uint8_t* ws = (uint8_t*)a.workspace;
    PackedArgs p{};
    uint32_t n = 0, blocks = 0;
    auto add = [&](const void*& src, uint64_t& ld, uint64_t stride, uint64_t rows, uint64_t matrices, uint64_t cols, uint64_t off, uint64_t ld_dst, const int64_t* offsets) {
        const uint64_t want = (rows * (ld_dst / 8) + 255) / 256, share = (uint64_t)sm_count * 8 / matrices, most = share > 64 ? share : 64;      // there may be rows in one group only
        p.m[n] = {(const uint16_t*)src, (uint16_t*)(ws + off), ld, stride, (uint32_t)rows, (uint32_t)matrices, (uint32_t)cols, (uint32_t)ld_dst,
                  (uint32_t)(want < most ? want : most), offsets};
        blocks += p.m[n].blocks * p.m[n].matrices;
        ++n;
        src = ws + off;
        ld = ld_dst;
    };
    p.rows = (uint32_t)a.rows;
    if (l.pack_x && (a.y || a.dweight)) add(a.x, a.ld_x, 0, a.rows, 1, a.width, l.off_x, l.ld_x, nullptr);
    if (l.pack_dy) add(a.dy, a.ld_dy, 0, a.rows, 1, a.out, l.off_dy, l.ld_dy, nullptr);
    if (l.pack_w && (a.y || a.dx)) {
        add(a.weight, a.ld_weight, a.stride_weight, a.out, a.groups, a.width, l.off_w, l.ld_w, a.offsets);
        a.stride_weight = a.out * l.ld_w;
    }
    if (n) SK_OP_CUDA(launch_kernel(true, k_grouped_pack, dim3(blocks), 256, 0, st, p));
    return SK_OK;
}

// Pairs of blocks or single ones for y and dx, from what the host knows: the mean number of rows of the groups that can have one.  A stage costs what
// it brings to an SM, at 50 bytes a cycle; the constants are those of plain products (see wide_tiles).
bool wide_rows(const GroupedArgs& a, uint64_t features, uint64_t k_stages, int sm_count) {
    const uint64_t live = a.groups < a.rows ? a.groups : a.rows, mean = (a.rows + live - 1) / live;
    auto last = [&](uint64_t high, uint64_t wide, uint64_t blocks, uint64_t units, uint64_t fixed) {
        const uint64_t count = (mean + wide - 1) / wide, cols = round_up((mean + count - 1) / count, 16);
        const uint64_t tiles = live * count * ((features + high - 1) / high), stage = (16384 + cols / blocks * 128) / 50;
        return (tiles + units - 1) / units * k_stages * stage + fixed;
    };
    return last(256, 256, 2, sm_count / 2, 12000) <= last(128, 128, 1, sm_count, 7000);
}

int launch_unpack(const GroupedArgs& a, const void* src, uint64_t ld_src, void* dst, uint64_t M, uint64_t N, int type, bool matrices, int sm_count, cudaStream_t st) {
    const UnpackArgs u{(const uint8_t*)src, (uint8_t*)dst, a.offsets, ld_src, M, (uint32_t)N, (uint32_t)a.groups, (uint32_t)a.rows, matrices, (uint32_t)a.fill};
    const uint64_t batch = matrices ? a.groups : 1, each = 256 * kUnpackEach * (16 / type_size(type)), want = (M * N + each - 1) / each;
    const uint64_t most = ((uint64_t)sm_count * 16 + batch - 1) / batch;
    const dim3 grid((uint32_t)(want < most ? want : most), (uint32_t)batch);
    SK_OP_CUDA(type == SK_F32 ? launch_kernel(true, k_grouped_unpack<4>, grid, 256, 0, st, u) : launch_kernel(true, k_grouped_unpack<2>, grid, 256, 0, st, u));
    return SK_OK;
}

// What y and dx are made from and go to.
struct RowsCall {
    const void* rows;
    uint64_t ld_rows;
    bool transposed;                                 // the matrix is read along its rows
    void* out;
    uint64_t ld_out;
};

template <int CG, int BN>
int launch_rows(const GroupedArgs& a, const GroupedLayout& l, const RowsCall& c, const OpDevice& dev, cudaStream_t st) {
    using Plan = RowsPlan<CG, BN>;
    static_assert(Plan::kTableOffset == GemmTile<CG, BN, RowsEpi>::kStages * GemmTile<CG, BN, RowsEpi>::kStageBytes);
    Plan p{};
    const uint32_t K = (uint32_t)(c.transposed ? a.out : a.width);
    const bool bf16 = a.type == SK_BF16;
    p.offsets = a.offsets;
    p.groups = (uint32_t)a.groups;
    p.rows = (uint32_t)a.rows;
    p.features = (uint32_t)(c.transposed ? a.width : a.out);
    p.tiles_m = (p.features + 128 * CG - 1) / (128 * CG);
    p.k_stages = (K + kGemmK - 1) / kGemmK;
    p.last_k = (K - (p.k_stages - 1) * kGemmK + 15) / 16 * 16;
    p.k_rows = K < kGemmK ? p.last_k : kGemmK;
    p.slices = l.slices;
    p.each = (p.k_stages + l.slices - 1) / l.slices;
    p.mn = c.transposed;
    p.bf16 = bf16;
    p.fill = a.fill;
    p.waits = a.waits(dev);
    p.withheld = a.withhold_ms != 0;
    const Operand w{a.weight, a.out, a.width, a.ld_weight, a.stride_weight, (uint32_t)a.groups, c.transposed};
    const Operand x{c.rows, a.rows, K, c.ld_rows, 0, 1, false};
    bool ok = encode_operand(&p.matrix, w, bf16, c.transposed ? p.k_rows : 128);
    for (int q = 0; q < 4; ++q) ok = ok && encode_operand(&p.rows_map[q], x, bf16, 128 >> q);
    if (!ok) return set_error(SK_ECUDA, "%s: the tensors cannot be described to the copy engine", __func__);
    // rows over BN of each segment, at most one tile more in each
    const uint64_t live = (a.groups < a.rows ? a.groups : a.rows) + (a.fill ? 2 : 0), most = (a.rows / BN + live) * p.tiles_m * l.slices;
    const uint64_t slots = (uint64_t)dev.sm_count / CG;
    const uint32_t units = (uint32_t)(most < slots ? most : slots);
    if constexpr (CG == 1) {
        const bool parts = K > long_sum(bf16);
        if (l.slices > 1) {
            float* sums = (float*)((uint8_t*)a.workspace + l.off_row_sums);
            const uint64_t stride = a.rows * l.ld_row_sums;
            if (parts) SK_OP_CUDA((launch_plan<CG, BN, Plan, LanesEpi<true, false>>(true, p, {sums, l.ld_row_sums, stride, bf16}, units, st)));
            else SK_OP_CUDA((launch_plan<CG, BN, Plan, LanesEpi<false, false>>(true, p, {sums, l.ld_row_sums, stride, bf16}, units, st)));
            SK_OP_CUDA(launch_kernel(true, k_grouped_sum, dim3((p.features + 255) / 256, (uint32_t)(a.rows < 4096 ? a.rows : 4096)), 256, 0, st, (const float*)sums, l.ld_row_sums,
                                     stride, l.slices, a.offsets, p.groups, p.rows, p.features, (uint16_t*)c.out, c.ld_out, (int)bf16, a.fill));
            return SK_OK;
        }
        if (parts) {
            SK_OP_CUDA((launch_plan<CG, BN, Plan, LanesEpi<true, true>>(true, p, {(uint16_t*)c.out, c.ld_out, 0, bf16}, units, st)));
            return SK_OK;
        }
    }
    RowsEpi::Args ea{{}, (uint16_t*)c.out, c.ld_out, bf16, row_alignment(c.out, c.ld_out, a.type), by_boxes(c.out, c.ld_out * 2, 0, p.features * 2, l.unpack_rows)};
    if (ea.by_box && !encode_out(&ea.map, c.out, 1, a.rows, p.features, c.ld_out, a.rows * c.ld_out, a.type, 16))
        return set_error(SK_ECUDA, "%s: the output cannot be described to the copy engine", __func__);
    SK_OP_CUDA((launch_plan<CG, BN, Plan, RowsEpi>(true, p, ea, units, st)));
    return SK_OK;
}
// y or dx, to where the layout says
int launch_rows_any(const GroupedArgs& a, const GroupedLayout& l, bool backward, const OpDevice& dev, cudaStream_t st) {
    RowsCall c{a.x, a.ld_x, false, a.y, a.ld_y};
    if (backward) c = {a.dy, a.ld_dy, true, a.dx, a.ld_dx};
    if (l.unpack_rows) {
        c.out = (uint8_t*)a.workspace + l.off_rows;
        c.ld_out = l.ld_rows;
    }
    const uint64_t features = backward ? a.width : a.out, K = backward ? a.out : a.width;
    return l.slices == 1 && K <= long_sum(a.type == SK_BF16) && wide_rows(a, features, (K + kGemmK - 1) / kGemmK, dev.sm_count) ? launch_rows<2, 256>(a, l, c, dev, st) : launch_rows<1, 128>(a, l, c, dev, st);
}

template <int CG, int BN, bool PARTS>
int launch_matrices(const GroupedArgs& a, const GroupedLayout& l, const OpDevice& dev, cudaStream_t st) {
    using Plan = MatrixPlan<CG, BN>;
    static_assert(GemmTile<CG, BN, MatrixEpi<PARTS>>::kSmem + sizeof(typename Plan::Table) + 256 <= 232448);
    Plan p{};
    const bool bf16 = a.type == SK_BF16;
    p.offsets = a.offsets;
    p.groups = (uint32_t)a.groups;
    p.rows = (uint32_t)a.rows;
    p.M = (uint32_t)a.out;
    p.N = (uint32_t)a.width;
    p.tiles_m = (p.M + 128 * CG - 1) / (128 * CG);
    p.tiles_n = (p.N + BN - 1) / BN;
    p.bf16 = bf16;
    p.waits = a.waits(dev);
    p.withheld = a.withhold_ms != 0;
    const Operand dy{a.dy, a.rows, a.out, a.ld_dy, 0, 1, true}, x{a.x, a.rows, a.width, a.ld_x, 0, 1, true};
    bool ok = true;
    for (int q = 0; q < 7; ++q) ok = ok && encode_operand(&p.a[q], dy, bf16, 64 >> q) && encode_operand(&p.b[q], x, bf16, 64 >> q);
    if (!ok) return set_error(SK_ECUDA, "%s: the tensors cannot be described to the copy engine", __func__);
    p.most_slices = l.most_slices;
    p.beside = a.dx && l.slices == 1;                // the kernel before is the product itself, which releases its successors
    p.slices = (uint32_t*)((uint8_t*)a.workspace + l.off_slices);
    typename MatrixEpi<PARTS>::Args ea{{}, a.dweight, a.ld_dweight, a.groups > 1 ? a.stride_dweight : a.out * a.ld_dweight, a.dweight_type, 0, 0,
                                       (float*)((uint8_t*)a.workspace + l.off_sums), l.ld_sums, nullptr, 0};
    const uint64_t size = type_size(a.dweight_type);
    if (ea.ld == a.width) {                          // the distance between the matrices is that of the output itself in any case
        ea.zeros = (uint8_t*)a.dweight;
        ea.zeros_stride = ea.stride * size;
    }
    if (l.unpack_matrices) {
        ea.out = (uint8_t*)a.workspace + l.off_matrices;
        ea.ld = l.ld_matrices;
        ea.stride = a.out * l.ld_matrices;
    }
    ea.by_box = by_boxes(ea.out, ea.ld * size, ea.stride * size, a.width * size, l.unpack_matrices);
    if (ea.by_box && !encode_out(&ea.map, ea.out, a.groups, a.out, a.width, ea.ld, ea.stride, ea.type, 32))
        return set_error(SK_ECUDA, "%s: the output cannot be described to the copy engine", __func__);
    const uint32_t by_row = row_alignment(ea.out, ea.ld, ea.type), by_matrix = row_alignment(ea.out, ea.stride, ea.type);
    ea.align = by_matrix < by_row ? by_matrix : by_row;
    const uint64_t tiles = (l.most_slices ? l.most_slices : a.groups) * p.tiles_m * p.tiles_n, slots = (uint64_t)dev.sm_count / CG;
    SK_OP_CUDA((launch_plan<CG, BN, Plan, MatrixEpi<PARTS>>(true, p, ea, (uint32_t)(tiles < slots ? tiles : slots), st)));
    if (l.most_slices) {
        const uint64_t want = (a.out * ((a.width + 3) / 4) + 31) / 32, most = (uint64_t)dev.sm_count * 8;
        SK_OP_CUDA(launch_kernel(true, k_grouped_join, dim3((uint32_t)(want < most ? want : most), p.groups), 256, 0, st, (const uint32_t*)p.slices,
                                 (const float*)ea.sums, l.ld_sums, p.M, p.N, ea.out, ea.ld, ea.stride, ea.type));
    }
    return l.unpack_matrices ? launch_unpack(a, ea.out, ea.ld, a.dweight, a.out, a.width, a.dweight_type, true, dev.sm_count, st) : SK_OK;
}

}  // namespace

uint64_t grouped_workspace(const GroupedArgs& a, bool backward) { return layout_of(a, backward).total; }

int launch_grouped(GroupedArgs a, const OpDevice& dev, cudaStream_t st) {
    const GroupedLayout l = layout_of(a, false);
    if (int rc = pack_operands(a, l, dev.sm_count, st)) return rc;
    if (int rc = launch_rows_any(a, l, false, dev, st)) return rc;
    return l.unpack_rows ? launch_unpack(a, (uint8_t*)a.workspace + l.off_rows, l.ld_rows, a.y, a.rows, a.out, a.type, false, dev.sm_count, st) : SK_OK;
}

int launch_grouped_backward(GroupedArgs a, const OpDevice& dev, cudaStream_t st) {
    const GroupedLayout l = layout_of(a, true);
    if (int rc = pack_operands(a, l, dev.sm_count, st)) return rc;
    if (a.dx)
        if (int rc = launch_rows_any(a, l, true, dev, st)) return rc;
    auto unpack_dx = [&] {                           // behind both products: the second one begins while the first still runs
        return a.dx && l.unpack_rows ? launch_unpack(a, (uint8_t*)a.workspace + l.off_rows, l.ld_rows, a.dx, a.rows, a.width, a.type, false, dev.sm_count, st) : SK_OK;
    };
    if (!a.dweight) return unpack_dx();
    // The accumulators' truncation grows with the rows added up: 16-bit gradients of fp16 and 32-bit ones show it, bf16's coarser rounding that of long groups only.
    const bool parts = a.dweight_type == SK_F32 || a.type == SK_F16 || a.rows > long_sum(true);
    auto launch = parts ? (l.wide ? launch_matrices<2, 256, true> : launch_matrices<1, 128, true>)
                        : (l.wide ? launch_matrices<2, 256, false> : launch_matrices<1, 128, false>);
    if (int rc = launch(a, l, dev, st)) return rc;
    return unpack_dx();
}

}  // namespace sk
