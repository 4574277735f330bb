// Orthogonalising matrix updates by Newton-Schulz products.
//
//   U = the update, or with a momentum M: M <- beta M + G and U = G + beta M (Nesterov) or U = M
//   X_0 = U / (|U|_F + eps);   A = X X^T,  P = a I + b A + c A^2,  X <- P X     (`steps` times, on the shorter side)
//
// Bound by the tensor cores for large matrices (3 m^2 n + m^3 multiply-adds a step for m <= n, the half of the symmetric
// products above the diagonal left out), by the latency of 3 * steps dependent products for small ones.
//
// Number format.  X, A and P are held as fp16 times 2^12 and every sum in 32 bits.  The iteration maps singular values of
// the normalised matrix into [0, 1.25], so fp16 times 2^12 neither overflows (the largest entry of P is a * 2^12)
// nor loses small entries (full precision down to 2^-26), and it has eight times bf16's resolution at the same speed.
// That is not enough where a few strong directions stand over noise, as in real gradients: X's rounding error,
// relative to the strong directions, is amplified together with the weak ones (up to a^steps).  So in all but the last two
// steps X is the sum of two fp16 matrices (22 bits) in the product P X, whose errors stay in the direction they arise in;
// A and P are single.  Errors of the result against 64 bits, before the output's own rounding (2-norm,
// rank 8 plus 5 % noise / gaussian): bf16 throughout 1.1e-1 / 1.0e-2, single fp16 1.4e-2 / 1.3e-3, this 1.1e-3 / 1.1e-3.
// That is below a bf16 output's own rounding (1.7e-3), but five times an fp16 output's (2.1e-4).  For those, PRECISE: X, A and P are pairs in every
// product, which is then the sum of three (high high, high low, low high; what is left out is 2^-22 of it).  Modelled: 5e-7, and any one of the
// matrices single in any three steps costs 2e-4 to 2e-3.  Three times the products take 1.4 times as long for 100 x 130 (31 -> 42 us), 1.8 for
// 12 x 768 x 768 (206 -> 373) and 2.2 for 8192 x 4096 (2.52 -> 5.66 ms).
//
// No operand is transposed: for a tall matrix (rows > cols) the same kernels take X in the other major
// (A = X^T X, X <- X P).
#include "sk_gemm.cuh"
#include "sk_operators.h"

#include <type_traits>

namespace sk {
namespace {

constexpr float kScale = 4096.0f, kUnscale = 1.0f / 4096.0f;     // 2^12
constexpr uint32_t kPadCols = 64;                                // leading dimensions: whole 128-byte lines

// ---- all products of the iteration in one launch --------------------------------------------------------------------------
// The tiles of A = X X^T, P = a I + b A + c A^2 and X <- P X of all steps and matrices, in this order, dealt out to the units in
// turn.  A tile may start when all tiles of the products before it of ITS matrix are written: a counter per matrix says how many epilogue
// warps have written theirs.  Waiting for a matrix instead of for everything keeps the units busy across the products' ends: 12 matrices of
// 768 x 768 take 200 us, with a launch per product 252.  What a product costs beside its stages of some 620 cycles: 1500 cycles from the first
// copy's issue to its arrival, 600 from the last product to the accumulator, 2000 (128 columns) to 7000 (256, mirrored) in the
// epilogue, 1100 to 2400 until its stores are seen, and as much again until the counter is read.
// Where A has few tiles and a long K, K is split: the slices' sums go to memory in 32 bits, and tiles without products, of kJoinParts to a tile
// of A, add them up in order (2688 x 256: 150 -> 122 us, 768 x 4096: 252 -> 209).  SLICED has its own kernels, as the longer way to a tile's
// place costs the others 4 %.
// A unit takes its tiles in order, every tile waits for earlier ones only, and the blocks are all resident (a cooperative launch): so the waits
// end; they have a limit all the same.
constexpr uint32_t kJoinParts = 4;               // of 32 rows of each block
enum ChainKind : uint32_t { kGram, kPoly, kApply, kJoin };   // kGram: A, or with slices a slice of it; kJoin, after it: A from its slices
struct ChainShape {
    CUtensorMap gram_x[2], apply_hi[2], apply_lo[2], gram, poly;     // [2]: the two buffers that X alternates between
    uint32_t steps, exact, tall, batch;
    uint32_t m, rows, cols;                      // shorter side; X's extents
    uint32_t side, square;                       // tile rows of A, its tiles on and below the diagonal
    uint32_t tiles_m, tiles_n, apply;            // of X
    uint32_t k_gram, k_poly;                     // stages along the longer and the shorter side
    uint32_t slices, k_slice;                    // of the longer side in A, stages of one
    uint32_t signals;                            // of every tile: its epilogue warps
    uint32_t* count;                             // per matrix, zero before the launch
    Waits waits;

    // X is the sum of two matrices in all but the last two steps, and in the first where one is exact
    __host__ __device__ bool pair(uint32_t step) const { return step + 2 < steps && !(step == 0 && exact); }
};
struct ChainLow {                                // PRECISE: the second matrices of the pairs, where ChainShape has none
    CUtensorMap gram_xlo[2], gram_lo, poly_lo;
};
template <bool SLICED, bool PRECISE>
struct ChainPlan : ChainShape, std::conditional<PRECISE, ChainLow, std::false_type>::type {
    static constexpr bool kCooperative = true, kEmpty = SLICED, kThree = PRECISE;    // kEmpty: has tiles without products
    static constexpr bool kRagged = false;
    // tiles of one matrix and step before those of a kind, and of all kinds
    __device__ __forceinline__ uint32_t tiles_before(uint32_t kind) const {
        if (!SLICED) return kind * square;
        return kind == kGram ? 0 : square * (slices + (kind == kJoin ? 0 : kJoinParts + (kind == kPoly ? 0 : 1)));
    }
    __device__ __forceinline__ uint32_t tiles_per_step() const { return tiles_before(kApply) + apply; }
    __device__ __forceinline__ bool job(uint32_t p, uint32_t units, uint32_t i, TileJob& j) const {
        const uint32_t per = batch * tiles_per_step(), t = p + i * units;
        j.step = t / per;
        if (j.step >= steps) return false;
        uint32_t q = t - j.step * per;
        const uint32_t from = j.step & 1;
        j.kind = q < batch * tiles_before(kPoly) ? kGram : q < batch * tiles_before(kApply) ? kPoly : kApply;
        if (SLICED && j.kind == kGram && q >= batch * tiles_before(kJoin)) j.kind = kJoin;
        q -= batch * tiles_before(j.kind);
        j.k_first = 0;
        j.a_rows = 128;
        j.k_rows = kGemmK;
        j.bf16 = 0;
        if (j.kind != kApply) {
            const uint32_t each = SLICED && j.kind != kPoly ? square * (j.kind == kGram ? slices : kJoinParts) : square;
            j.b = q / each;
            q -= j.b * each;
            if (SLICED) {
                j.slice = q / square;
                q -= j.slice * square;
            }
            uint32_t r = (uint32_t)((sqrtf(8.0f * (float)q + 1.0f) - 1.0f) * 0.5f);
            while (r * (r + 1) / 2 > q) --r;
            while ((r + 1) * (r + 2) / 2 <= q) ++r;
            j.m = r;
            j.n = q - r * (r + 1) / 2;
            j.M = j.N = m;
            j.a_mn = j.b_mn = j.kind == kGram && tall;
            j.k_stages = j.pass = j.kind == kGram ? k_gram : k_poly;
            if (SLICED && j.kind == kGram) {
                j.k_first = (int)(j.slice * k_slice * kGemmK);
                j.k_stages = j.pass = min(k_slice, k_gram - j.slice * k_slice);
            }
            if (SLICED && j.kind == kJoin) j.k_stages = 0;
            j.map_a = j.map_b = j.map_a2 = j.map_b2 = j.kind == kGram ? &gram_x[from] : &gram;
            if constexpr (PRECISE) {
                j.map_b2 = j.map_a3 = j.kind == kGram ? &this->gram_xlo[from] : &this->gram_lo;
                j.map_b3 = j.map_b;
                if (j.kind == kPoly || (j.kind == kGram && !(j.step == 0 && exact))) j.k_stages *= 3;
            }
        } else {
            j.b = q / apply;
            q -= j.b * apply;
            const uint32_t band = q / (8 * tiles_n), high = min(8u, tiles_m - band * 8);
            q -= band * 8 * tiles_n;
            j.n = q / high;
            j.m = band * 8 + (q - j.n * high);
            j.M = rows;
            j.N = cols;
            // X with its columns contiguous is the K-major first factor of X P, and the MN-major second one of P X
            j.a_mn = 0;
            j.b_mn = !tall;
            j.pass = k_poly;
            j.k_stages = pair(j.step) ? 2 * k_poly : k_poly;
            j.map_a = tall ? &apply_hi[from] : &poly;
            j.map_b = tall ? &poly : &apply_hi[from];
            j.map_a2 = tall ? &apply_lo[from] : &poly;
            j.map_b2 = tall ? &poly : &apply_lo[from];
            if constexpr (PRECISE) {             // P's second matrix goes before X's, which the first step may not have
                j.k_stages = (j.step == 0 && exact ? 2 : 3) * k_poly;
                j.map_a3 = j.map_a2;
                j.map_b3 = j.map_b2;
                j.map_a2 = tall ? j.map_a : &this->poly_lo;
                j.map_b2 = tall ? &this->poly_lo : j.map_b;
            }
        }
        j.z = (int)j.b;
        return true;
    }
    __device__ __forceinline__ bool wait(const TileJob& j) const {
        const uint32_t need = (j.step * tiles_per_step() + tiles_before(j.kind)) * signals;
        if (!need) return true;
        const uint32_t* counter = count + j.b;
        const bool ok = wait_until([counter, need] {
            uint32_t have;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(have) : "l"(counter) : "memory");
            return have >= need;
        }, waits);
        asm volatile("fence.proxy.async;" ::: "memory");             // what was written by stores is read by TMA
        return ok;
    }
    __device__ __forceinline__ void done(const TileJob& j) const {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) {
            __threadfence();
            atomicAdd(count + j.b, 1u);
        }
    }
    __device__ __forceinline__ const CUtensorMap* descriptor(uint32_t i) const {
        if (i < 8) return &gram_x[0] + i;
        if constexpr (PRECISE) return i < 12 ? &this->gram_xlo[0] + (i - 8) : nullptr;
        return nullptr;
    }
};

struct ChainArgs {
    __half *gram, *poly, *hi[2], *lo[2];     // [2]: as the plan's
    __half *gram_lo, *poly_lo;               // PRECISE
    float* slices;                           // A's: slice by slice, like A but in 32 bits
    uint64_t slice_stride;
    uint32_t slice_count, join_cols;         // join_cols: a warp's columns when they are added up
    uint64_t a_stride, x_stride;
    uint32_t ld_a, ld_x;
    float a, b, c;
    const float* factor;                     // per matrix: the first step's X = factor * (the matrix that is stored)
    void* out;                               // the last step's, in the caller's type and layout
    uint64_t out_stride, ld_out;
    int out_type;
    uint32_t align, steps;
};

// The epilogues of the three products.  A warp has two areas of staging memory: one for the lines of the matrix it writes, one for those of the second
// matrix of a pair, or for A's lines on their way to P, which are fetched while the products run.
template <bool SLICED, bool PRECISE>
struct ChainEpi {
    static constexpr int kWarps = 8, kWords = 2 * kStageWords;
    static constexpr bool kParts = false;
    using Args = ChainArgs;
    const Args& e;
    const TileJob& t;
    uint32_t row, row0, rows;                    // the lane's row, the warp's first, how many of the warp's exist
    uint32_t stage;
    float scale = kUnscale;
    __device__ ChainEpi(const Args& a, const TileJob& t_, uint32_t row_, uint32_t, uint32_t stage_)
        : e(a), t(t_), row(row_), row0(row_ - (threadIdx.x & 31)), stage(stage_) {
        rows = row0 >= t.M ? 0 : t.M - row0 < 32 ? t.M - row0 : 32;
        if (t.step == 0 && t.kind != kPoly) {
            const float f = a.factor[t.b];
            scale *= t.kind == kApply ? f : f * f;
        }
        if (t.kind == kApply && t.step + 1 == e.steps) scale *= kUnscale;
    }
    // A's 64 columns from `col` of the warp's rows into the second area
    __device__ void fetch(uint32_t col) {
        const uint32_t lane = threadIdx.x & 31, c = lane & 7;
        const __half* src = e.gram + t.b * e.a_stride + (uint64_t)row0 * e.ld_a + col + 8 * c;
        if (col + 8 * c < e.ld_a) {
#pragma unroll
            for (uint32_t r = lane >> 3; r < 32; r += 4)
                if (r < rows)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(staged(stage + kStageWords * 4, r, c)), "l"(src + (uint64_t)r * e.ld_a) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // A's slices added up: of 32 rows of the block, the warp's share of the columns, 16 at a time.  Four lanes have the 64 bytes of a row;
    // the sums of all slices are on their way at once, four slices to a batch.
    __device__ void join(uint32_t col0) {
        const uint32_t lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - 2, quarter = (threadIdx.x >> 5) & 3;
        const uint32_t first_row = row0 - quarter * 32 + t.slice * 32, r = lane >> 2, c = 4 * (lane & 3);
        if (first_row >= t.M) return;
        __half* out = e.gram + t.b * e.a_stride;
        for (uint32_t q = 0; q < e.join_cols; q += 16) {
            const uint32_t col = col0 + (warp & 3) * e.join_cols + q;
            if (col >= t.N) break;
            const float* p = e.slices + t.b * e.a_stride + (uint64_t)(first_row + r) * e.ld_a + col + c;
            float4 sum[4] = {};
            for (uint32_t k = 0; k < e.slice_count; k += 4) {
                float4 f[4][4];
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        f[j][i] = make_float4(0, 0, 0, 0);
                        if (k + j < e.slice_count && first_row + r + 8 * i < t.M)
                            f[j][i] = __ldcg((const float4*)(p + (k + j) * e.slice_stride + (uint64_t)(8 * i) * e.ld_a));
                    }
#pragma unroll
                for (uint32_t j = 0; j < 4; ++j)
#pragma unroll
                    for (uint32_t i = 0; i < 4; ++i) {
                        sum[i].x += f[j][i].x; sum[i].y += f[j][i].y; sum[i].z += f[j][i].z; sum[i].w += f[j][i].w;
                    }
            }
#pragma unroll
            for (uint32_t which = 0; which < (PRECISE ? 2u : 1u); ++which) {
                if (which) out = e.gram_lo + t.b * e.a_stride;
                __syncwarp();
#pragma unroll
                for (uint32_t i = 0; i < 4; ++i) {
                    float4& f = sum[i];
                    if (!which) f = make_float4(f.x * scale, f.y * scale, f.z * scale, f.w * scale);
                    const uint32_t lo = pack16(f.x, f.y, false), hi = pack16(f.z, f.w, false);
                    if (first_row + r + 8 * i < t.M) *(uint2*)(out + (uint64_t)(first_row + r + 8 * i) * e.ld_a + col + c) = make_uint2(lo, hi);
                    if (t.m != t.n) {            // the mirror image: 16 rows of 80 bytes in the staging memory
                        const uint32_t at = stage + c * 80 + (r + 8 * i) * 2;
                        store_shared2(at, lo);
                        store_shared2(at + 80, lo >> 16);
                        store_shared2(at + 160, hi);
                        store_shared2(at + 240, hi >> 16);
                    }
                    if (PRECISE && !which) {     // what the first matrix leaves
                        const float2 a = __half22float2(*(const __half2*)&lo), b = __half22float2(*(const __half2*)&hi);
                        f = make_float4(f.x - a.x, f.y - a.y, f.z - b.x, f.w - b.y);
                    }
                }
                if (t.m == t.n) continue;
                __syncwarp();
#pragma unroll
                for (uint32_t i = 0; i < 2; ++i) {
                    const uint32_t y = r + 8 * i;
                    const uint4 w = load_shared16(stage + y * 80 + (lane & 3) * 16);
                    if (col + y < t.N) *(uint4*)(out + (uint64_t)(col + y) * e.ld_a + first_row + 8 * (lane & 3)) = w;
                }
            }
            out = e.gram + t.b * e.a_stride;
        }
    }
    template <class Plan>
    __device__ bool begin(const Plan& plan, uint32_t col0) {
        if (SLICED && t.kind == kJoin) {
            if (!__all_sync(0xffffffffu, plan.wait(t))) return false;            // no products wait for the warps that have nothing to add up
            join(col0);
        }
        if (t.kind != kPoly || !rows) return true;
        if (!__all_sync(0xffffffffu, plan.wait(t))) return false;
        fetch(col0);
        return true;
    }
    __device__ void square(__half* out, uint32_t col, float (&v)[32], bool last) {
        store_tile32(out, SK_F16, e.ld_a, row0, rows, col, e.ld_a, v, 16, stage, true, last);
        const bool second = col & 32;
        if (t.m == t.n || !(second || last)) return;
        // The mirror image, from the staged lines.  A transposing load of four 8 x 8 matrices gives a lane two neighbouring rows of one column from each;
        // with rows 8 s + 2 i, 8 s + 2 i + 1 (s = 0..3) in matrix i they are eight neighbours: four lanes write a row of the image.
        const uint32_t lane = threadIdx.x & 31, first = col & ~63u, count = second ? 64 : 32;
        const uint32_t from = 8 * ((lane & 7) >> 1) + 2 * (lane >> 3) + (lane & 1);
        uint4 q[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                         : "=r"(q[i].x), "=r"(q[i].y), "=r"(q[i].z), "=r"(q[i].w) : "r"(staged(stage, from, i)) : "memory");
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            const uint32_t c = 8 * i + (lane >> 2);
            if (c < count && first + c < t.N) *(uint4*)(out + (uint64_t)(first + c) * e.ld_a + row0 + 8 * (lane & 3)) = q[i];
        }
    }
    // A pair of matrices and their mirror images, 32 columns at a time, one matrix after the other through the first area: the second holds
    // what is fetched.
    __device__ void square_pair(__half* hi, __half* lo, uint32_t col, float (&v)[32]) {
        const uint32_t lane = threadIdx.x & 31, from = 8 * ((lane & 7) >> 1) + 2 * (lane >> 3) + (lane & 1);
#pragma unroll 1
        for (uint32_t which = 0; which < 2; ++which) {
            __half* out = which ? lo : hi;
            store_tile32(out, SK_F16, e.ld_a, row0, rows, col, e.ld_a, v, 16, stage, false, true);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
            if (t.m == t.n) continue;
            uint4 q[4];
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i)
                asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                             : "=r"(q[i].x), "=r"(q[i].y), "=r"(q[i].z), "=r"(q[i].w) : "r"(staged(stage, from, i)) : "memory");
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) {
                const uint32_t c = col + 8 * i + (lane >> 2);
                if (c < t.N) *(uint4*)(out + (uint64_t)c * e.ld_a + row0 + 8 * (lane & 3)) = q[i];
            }
        }
    }
    __device__ void chunk(uint32_t col, float (&v)[32], bool last) {
        if (!rows) return;
        if (SLICED && t.kind == kGram) {       // scaled when the slices are joined
            store_tile32(e.slices + t.slice * e.slice_stride + t.b * e.a_stride, SK_F32, e.ld_a, row0, rows, col, e.ld_a, v, 16, stage, false, last);
            return;
        }
        if (t.kind == kPoly) {
            if (!(col & 32)) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint4 w = load_shared16(staged(stage + kStageWords * 4, row - row0, ((col & 32) >> 3) + q));
                const uint32_t r[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = __half22float2(*(const __half2*)&r[i]);
                    v[8 * q + 2 * i] = e.b * f.x + e.c * kUnscale * v[8 * q + 2 * i];
                    v[8 * q + 2 * i + 1] = e.b * f.y + e.c * kUnscale * v[8 * q + 2 * i + 1];
                }
            }
            if (PRECISE && row < t.M) {          // A's second matrix straight from L2, where the other SMs have written it
                const __half* low = e.gram_lo + t.b * e.a_stride + (uint64_t)row * e.ld_a + col;
                uint4 w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] = __ldcg((const uint4*)low + q);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t r[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 f = __half22float2(*(const __half2*)&r[i]);
                        v[8 * q + 2 * i] += e.b * f.x;
                        v[8 * q + 2 * i + 1] += e.b * f.y;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i == row) v[i] += e.a * kScale;
            __syncwarp();
            if ((col & 32) && !last) fetch(col + 32);                // while this pair is written
            if constexpr (PRECISE) square_pair(e.poly + t.b * e.a_stride, e.poly_lo + t.b * e.a_stride, col, v);
            else square(e.poly + t.b * e.a_stride, col, v, last);
            return;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= scale;
        if (t.kind == kGram) {
            if constexpr (PRECISE) square_pair(e.gram + t.b * e.a_stride, e.gram_lo + t.b * e.a_stride, col, v);
            else square(e.gram + t.b * e.a_stride, col, v, last);
            return;
        }
        if (t.step + 1 == e.steps) {
            store_tile32((uint16_t*)e.out + t.b * e.out_stride, e.out_type, e.ld_out, row0, rows, col, t.N, v, e.align, stage, true, last);
            return;
        }
        const uint32_t to = (t.step + 1) & 1;
        store_tile32(e.hi[to] + t.b * e.x_stride, SK_F16, e.ld_x, row0, rows, col, e.ld_x, v, 16, stage, true, last);
        if (PRECISE || t.step + 3 < e.steps) {   // the next step's X is a pair
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
            store_tile32(e.lo[to] + t.b * e.x_stride, SK_F16, e.ld_x, row0, rows, col, e.ld_x, v, 16, stage + kStageWords * 4, true, last);
        }
    }
    __device__ void end() {}
};

// ---- the normalised matrix ------------------------------------------------------------------------------------------
constexpr uint32_t kNormBlocks = 1024;           // most partial sums of squares per matrix

// eight neighbouring values of a row (vec: on a 16-byte boundary and all of them there), zero beyond the row's end
__device__ __forceinline__ void load8(const void* p, int type, uint64_t at, uint32_t valid, bool vec, float (&v)[8]) {
    if (vec) {
        if (type == SK_F32) {
            const float4 a = *(const float4*)((const float*)p + at), b = *(const float4*)((const float*)p + at + 4);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            return;
        }
        const uint4 r = *(const uint4*)((const uint16_t*)p + at);
        const uint32_t q[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = type == SK_BF16 ? __bfloat1622float2(*(const __nv_bfloat162*)&q[i]) : __half22float2(*(const __half2*)&q[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (uint32_t)i < valid ? load_as(p, type, at + i) : 0.0f;
}

// 2^12 / (norm + eps) as a product of two factors that are ordinary 32-bit values each: by itself it may be beyond their range (a norm
// below 2^-115).  exact: both are powers of two, and `rest` in [1, 2) what is left.
struct Scale { float first, second, rest; };
__device__ __forceinline__ Scale scale_of(double squares, float eps, bool exact) {
    const double scale = (double)kScale / (sqrt(squares) + (double)eps);
    const bool large = scale > 0x1p100, tiny = scale < 0x1p-100;
    const float first = large ? 0x1p64f : tiny ? 0x1p-64f : 1.0f;
    const double other = large ? scale * 0x1p-64 : tiny ? scale * 0x1p64 : scale;
    if (!exact || !(scale > 0.0 && isfinite(scale))) return {first, (float)other, 1.0f};         // (not: infinities or NaN in the update)
    int e = 0;
    const double m = 2.0 * frexp(other, &e);                         // other = m 2^(e-1), m in [1, 2)
    return {first, (float)ldexp(1.0, e - 1), (float)m};
}

struct SquareArgs {
    OrthoArgs a;
    double* partial;                             // [batch][kNormBlocks]
    float* factor;                               // [batch]: X = factor * (the matrix that is stored)
    uint32_t blocks, vec_u, vec_m;
    __half *hi, *lo;
    uint32_t ld;
    uint64_t stride;
    uint32_t exact;                              // U is the 16-bit update itself: stored exactly, times a power of two
    uint32_t* count;                             // [batch], set to zero
};

// Sums of squares of U per block, in 64 bits (an update in fp32 may have squares beyond its range); updates the momentum.
__global__ void __launch_bounds__(256) k_ortho_square(const __grid_constant__ SquareArgs s) {
    __shared__ double sums[8];
    const OrthoArgs& a = s.a;
    chain_acquire();
    const uint32_t b = blockIdx.y, groups = ((uint32_t)a.cols + 7) / 8;
    const uint32_t total = (uint32_t)a.rows * groups;
    double sum = 0;
#pragma unroll 2
    for (uint32_t q = blockIdx.x * 256 + threadIdx.x; q < total; q += gridDim.x * 256) {
        const uint32_t row = q / groups, col = (q - row * groups) * 8, valid = (uint32_t)a.cols - col;
        float u[8];
        load8(a.update, a.type, b * a.stride_update + row * a.ld_update + col, valid, s.vec_u, u);
        if (a.momentum) {
            float m[8];
            const uint64_t at = b * a.stride_momentum + row * a.ld_momentum + col;
            load8(a.momentum, SK_F32, at, valid, s.vec_m, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = a.beta * m[i] + u[i];
                u[i] = a.nesterov ? u[i] + a.beta * m[i] : m[i];
            }
            if (s.vec_m) {
                *(float4*)(a.momentum + at) = make_float4(m[0], m[1], m[2], m[3]);
                *(float4*)(a.momentum + at + 4) = make_float4(m[4], m[5], m[6], m[7]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((uint32_t)i < valid) a.momentum[at + i] = m[i];
            }
        }
        float part = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) part += u[i] * u[i];
        if (part > 1e-30f && part < 1e30f) sum += (double)part;       // the eight squares are well inside the 32-bit range
        else
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)u[i] * (double)u[i];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += sums[i];
        s.partial[(uint64_t)b * kNormBlocks + blockIdx.x] = sum;
    }
}

// The matrix the products start from.  16-bit updates without a momentum are stored exactly, times the power of two next to
// 2^12 / |U| (their significands fit fp16's); the rest of the normalisation is a factor that the first step's epilogues apply, and the
// first product needs no second matrix.  Otherwise X itself, as the sum of two fp16 matrices.
__global__ void __launch_bounds__(256) k_ortho_scale(const __grid_constant__ SquareArgs s) {
    __shared__ double sums[8];
    __shared__ Scale s_scale;
    const OrthoArgs& a = s.a;
    chain_acquire();
    const uint32_t b = blockIdx.y, groups = ((uint32_t)a.cols + 7) / 8;
    double sum = 0;
    for (uint32_t i = threadIdx.x; i < s.blocks; i += 256) sum += s.partial[(uint64_t)b * kNormBlocks + i];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += sums[i];
        s_scale = scale_of(sum, a.eps, s.exact);
        if (blockIdx.x == 0) {
            s.factor[b] = s_scale.rest;
            s.count[b] = 0;
        }
    }
    __syncthreads();
    const float first = s_scale.first, second = s_scale.second;
    const uint32_t total = (uint32_t)a.rows * groups;
#pragma unroll 2
    for (uint32_t q = blockIdx.x * 256 + threadIdx.x; q < total; q += gridDim.x * 256) {
        const uint32_t row = q / groups, col = (q - row * groups) * 8, valid = (uint32_t)a.cols - col;
        float u[8];
        load8(a.update, a.type, b * a.stride_update + row * a.ld_update + col, valid, s.vec_u, u);
        if (a.momentum) {
            float m[8];
            load8(a.momentum, SK_F32, b * a.stride_momentum + row * a.ld_momentum + col, valid, s.vec_m, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = a.nesterov ? u[i] + a.beta * m[i] : m[i];
        }
        uint32_t h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x = u[2 * i] * first * second, y = u[2 * i + 1] * first * second;
            const __half2 p = __floats2half2_rn(x, y);
            const float2 f = __half22float2(p);
            h[i] = *(const uint32_t*)&p;
            l[i] = pack16(x - f.x, y - f.y, false);
        }
        const uint64_t at = b * s.stride + (uint64_t)row * s.ld + col;   // ld is a multiple of 64: whole groups fit
        *(uint4*)(s.hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
        if (s.lo) *(uint4*)(s.lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

// How the products are cut: pairs of blocks on 256 x 256 or single ones on 128 x 128, and slices of the longer side in A.  A stage takes
// both tiles the same time (some 620 cycles, see wide_tiles), the pair does twice the work per SM in it.  The time is about that of
// the work on all units, but at least that of one matrix's dependent products, whose starts and epilogues are shorter with the
// small tile (7000 cycles, 12,000).  Slices shorten the path by their stages and add kJoinCost (256 x 1024 is slower with them: 114 us for
// 107).  Planned for the SMs of a B200, as the workspace's size depends on it.
constexpr uint64_t kJoinCost = 9000;             // cycles: writing slices, their signal, and adding them up
struct ChainTiles { bool wide; uint32_t slices; };
ChainTiles chain_tiles(const OrthoArgs& a, bool precise) {
    const uint64_t m = a.rows < a.cols ? a.rows : a.cols, n = a.rows < a.cols ? a.cols : a.rows, sms = 148;
    const uint64_t square_passes = precise ? 3 : 1, apply_passes = precise ? 3 : 2;       // most of a step's
    const uint64_t k_gram = (n + kGemmK - 1) / kGemmK, k_poly = (m + kGemmK - 1) / kGemmK;
    ChainTiles best = {false, 1};
    uint64_t least = ~0ull;
    for (int wide = 1; wide >= 0; --wide) {
        const uint64_t tile = wide ? 256 : 128, units = wide ? sms / 2 : sms, start = wide ? 12000 : 7000;
        const uint64_t side = (m + tile - 1) / tile, square = side * (side + 1) / 2, apply = side * ((n + tile - 1) / tile);
        for (uint64_t slices = 1; slices <= 8; ++slices) {
            const uint64_t each = (k_gram + slices - 1) / slices;
            if (slices > 1 && (a.batch * square * slices > units || (slices - 1) * each >= k_gram)) break;       // no empty slice
            const uint64_t work = a.batch * (square * square_passes * (k_gram + k_poly) + apply * apply_passes * k_poly +
                                             ((1 + slices) * square + apply) * kTileCost);
            auto rounds = [&](uint64_t tiles) { return (tiles + units - 1) / units; };
            const uint64_t path = ((rounds(square * slices) * each + rounds(square) * k_poly) * square_passes + rounds(apply) * apply_passes * k_poly) * 620 +
                                  3 * start + (slices > 1 ? kJoinCost : 0), even = work * 620 / units, cost = path > even ? path : even;
            if (cost < least) {
                least = cost;
                best = {wide != 0, (uint32_t)slices};
            }
        }
    }
    return best;
}

struct OrthoLayout {
    uint32_t ld_x, ld_a, m;
    uint64_t x_elems, a_elems;                   // per matrix
    uint64_t off_partial, off_factor, off_count, off_x[2], off_lo, off_a, off_p, off_a_lo, off_p_lo, off_slices, total;
};
// for either type of output
OrthoLayout layout_of(const OrthoArgs& a) {
    OrthoLayout l;
    l.m = (uint32_t)(a.rows < a.cols ? a.rows : a.cols);
    l.ld_x = (uint32_t)round_up(a.cols, kPadCols);
    l.ld_a = (uint32_t)round_up(l.m, kPadCols);
    l.x_elems = (uint64_t)a.rows * l.ld_x;
    l.a_elems = (uint64_t)l.m * l.ld_a;
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t r = at; at += round_up(bytes, 256); return r; };
    l.off_partial = take(a.batch * kNormBlocks * 8);
    l.off_factor = take(a.batch * 4);
    l.off_count = take(a.batch * 4);
    l.off_x[0] = take(a.batch * l.x_elems * 2);
    l.off_x[1] = take(a.batch * l.x_elems * 2);
    l.off_lo = take(2 * round_up(a.batch * l.x_elems * 2, 256));
    l.off_a = take(a.batch * l.a_elems * 2);
    l.off_p = take(a.batch * l.a_elems * 2);
    l.off_a_lo = take(a.batch * l.a_elems * 2);
    l.off_p_lo = take(a.batch * l.a_elems * 2);
    const uint32_t plain = chain_tiles(a, false).slices, precise = chain_tiles(a, true).slices, slices = plain > precise ? plain : precise;
    l.off_slices = take(slices > 1 ? slices * a.batch * l.a_elems * 4 : 0);
    l.total = at;
    return l;
}

// ---- the whole iteration in one launch --------------------------------------------------------------------------------
// Matrices whose shorter side is at most 128 (Y: m x n, m <= 128, the update or its transpose) and whose longer one is at most 16 * 256: fifteen
// dependent products of microseconds each are all launch latency one by one, so a cluster of blocks keeps the matrix in shared
// memory and does everything.  Block c holds 256 columns of Y as fp16 pairs; its layout (blocks of 64 columns, rows of 128 bytes,
// swizzled) is at once the K-major operand of Y Y^T and the MN-major second factor of P Y.  The blocks' shares of the gram matrix are added
// up in block order, a slice of rows to each block, over distributed shared memory; A^2 and P are small and formed by every block.
// Five steps took 84 us with a launch per product and take 28 us for 100 x 130; 100 x 4000 160 us as tiles of one launch (one SM goes over all of
// the longer side) and 63 us here.
constexpr int kSmallThreads = 512;
constexpr uint32_t kSmallSide = 128, kSmallCols = 256, kSmallCluster = 16;
constexpr uint32_t kSmallGroups = kSmallSide * kSmallCols / 8 / kSmallThreads;
constexpr uint32_t kSmallHi = 0, kSmallLo = 65536, kSmallGram = 131072, kSmallPoly = kSmallGram + 32768, kSmallBytes = 196608;

struct SmallArgs {
    OrthoArgs a;
    uint32_t m, n, tall, blocks;                 // blocks of the cluster
    uint32_t align, vec_u, vec_m;
    Waits waits;
};

// where 16-byte chunk `chunk` of row r of a 64-column block lies
__device__ __forceinline__ uint32_t swizzled(uint32_t r, uint32_t chunk) { return r * 128 + ((chunk ^ (r & 7)) << 4); }
__device__ __forceinline__ uint32_t map_to(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// what rounding to fp16 leaves of values
__device__ __forceinline__ void leave_low(float (&v)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async;" ::: "memory"); }
// 32 values of a row as fp16 into a swizzled matrix of 64-column blocks of 128 rows
__device__ __forceinline__ void put32(uint8_t* base, uint32_t r, uint32_t col, const float (&v)[32]) {
    uint8_t* block = base + (col >> 6) * 16384;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 q;
        q.x = pack16(v[8 * i], v[8 * i + 1], false);
        q.y = pack16(v[8 * i + 2], v[8 * i + 3], false);
        q.z = pack16(v[8 * i + 4], v[8 * i + 5], false);
        q.w = pack16(v[8 * i + 6], v[8 * i + 7], false);
        *(uint4*)(block + swizzled(r, ((col & 63) >> 3) + i)) = q;
    }
}

// PRECISE: A's second matrix lies where P lies otherwise, and P's pair takes the places of A's, element by element.
template <bool PRECISE>
__global__ void __launch_bounds__(kSmallThreads, 1) k_ortho_small(const __grid_constant__ SmallArgs s) {
    constexpr uint32_t kGramLo = kSmallPoly, kP = PRECISE ? kSmallGram : kSmallPoly, kPLo = kSmallPoly;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_mem;
    __shared__ uint32_t tmem_slot;
    __shared__ double sums[kSmallThreads / 32], shares[kSmallCluster];
    const OrthoArgs& a = s.a;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, S = s.blocks;
    const uint32_t rank = S > 1 ? cluster_rank() : 0, batch = blockIdx.x / S;
    const uint32_t base32 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base = smem_raw + (base32 - smem_u32(smem_raw));
    const uint32_t bar = smem_u32(&bar_mem);
    if (tid == 0) {
        mbar_init(bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) tmem_alloc<1>(smem_u32(&tmem_slot), 512);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *(volatile uint32_t*)&tmem_slot, tmem_sq = tmem + 128, tmem_x = tmem + 256;
    chain_acquire();

    // columns first .. first + width of Y are this block's; in memory they are columns (wide) or rows (tall) of the update
    const uint32_t first = rank * kSmallCols, width = s.n > first ? min(s.n - first, kSmallCols) : 0;
    // what the products go over, in whole steps of 16 (the same in every block of the cluster): beyond Y's rows and columns up to there is
    // zero, what lies further out is never read
    const uint32_t m16 = (s.m + 15) / 16 * 16, w16 = (min(s.n, kSmallCols) + 15) / 16 * 16, blocks64 = (w16 + 63) / 64;
    const uint64_t at_u = batch * a.stride_update, at_m = batch * a.stride_momentum;
    // element (i, j) of this block's part: i along the shorter side
    auto offset = [&](uint64_t ld, uint32_t i, uint32_t j) { return s.tall ? (uint64_t)(first + j) * ld + i : (uint64_t)i * ld + first + j; };
    // groups of eight neighbours of a row in memory, at most eight groups a thread, held in registers from the norm to the matrix
    const uint32_t fast = s.tall ? s.m : width, slow = s.tall ? width : s.m;
    const uint32_t per = max((fast + 7) / 8, 1u), groups = fast ? per * slow : 0;         // the cluster's last blocks may have no columns
    float u[kSmallGroups][8];
    double sum = 0;
    auto place = [&](uint32_t g, uint32_t& y, uint32_t& x) {
        const uint32_t q = g * kSmallThreads + tid;
        y = q / per;
        x = (q - y * per) * 8;
        return q < groups;
    };
#pragma unroll
    for (uint32_t g = 0; g < kSmallGroups; ++g) {
        uint32_t y, x;
        const bool live = place(g, y, x);
        if (live) load8(a.update, a.type, at_u + (s.tall ? offset(a.ld_update, x, y) : offset(a.ld_update, y, x)), fast - x, s.vec_u, u[g]);
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) u[g][k] = 0.0f;
    }
    if (a.momentum) {
#pragma unroll
        for (uint32_t g = 0; g < kSmallGroups; ++g) {
            uint32_t y, x;
            if (!place(g, y, x)) continue;
            const uint64_t at = at_m + (s.tall ? offset(a.ld_momentum, x, y) : offset(a.ld_momentum, y, x));
            float m[8];
            load8(a.momentum, SK_F32, at, fast - x, s.vec_m, m);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                m[k] = a.beta * m[k] + u[g][k];
                u[g][k] = a.nesterov ? u[g][k] + a.beta * m[k] : m[k];
            }
            if (s.vec_m) {
                *(float4*)(a.momentum + at) = make_float4(m[0], m[1], m[2], m[3]);
                *(float4*)(a.momentum + at + 4) = make_float4(m[4], m[5], m[6], m[7]);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (x + k < fast) a.momentum[at + k] = m[k];
            }
        }
    }
#pragma unroll
    for (uint32_t g = 0; g < kSmallGroups; ++g) {
        float part = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) part += u[g][k] * u[g][k];
        if (part > 1e-30f && part < 1e30f) sum += (double)part;      // the eight squares are well inside the 32-bit range
        else
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += (double)u[g][k] * (double)u[g][k];
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sums[warp] = sum;
    for (uint32_t q = tid; q < blocks64 * 1024; q += kSmallThreads) {
        ((uint4*)(base + kSmallHi))[q] = make_uint4(0, 0, 0, 0);
        ((uint4*)(base + kSmallLo))[q] = make_uint4(0, 0, 0, 0);
    }
    if (S > 1) cluster_sync_all();               // every block of the cluster has started
    __syncthreads();
    if (tid < S) {                               // this block's share into slot `rank` of every block
        double t = 0;
        for (int i = 0; i < kSmallThreads / 32; ++i) t += sums[i];
        asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(S > 1 ? map_to(smem_u32(&shares[rank]), tid) : smem_u32(&shares[0])), "d"(t) : "memory");
    }
    if (S > 1) cluster_sync_all();
    __syncthreads();
    sum = 0;
    for (uint32_t i = 0; i < S; ++i) sum += shares[i];
    const Scale scale = scale_of(sum, a.eps, false);
    const bool pair = PRECISE || a.steps > 2;
#pragma unroll
    for (uint32_t g = 0; g < kSmallGroups; ++g) {
        uint32_t y, x;
        if (!place(g, y, x)) continue;
        if (!s.tall) {                           // eight columns of a row: one 16-byte chunk
            uint32_t h[4], l[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p = u[g][2 * k] * scale.first * scale.second, r = u[g][2 * k + 1] * scale.first * scale.second;
                const __half2 both = __floats2half2_rn(p, r);
                const float2 f = __half22float2(both);
                h[k] = *(const uint32_t*)&both;
                l[k] = pack16(p - f.x, r - f.y, false);
            }
            const uint32_t at = (x >> 6) * 16384 + swizzled(y, (x & 63) >> 3);
            *(uint4*)(base + kSmallHi + at) = make_uint4(h[0], h[1], h[2], h[3]);
            if (pair) *(uint4*)(base + kSmallLo + at) = make_uint4(l[0], l[1], l[2], l[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (x + k >= fast) break;
                const float p = u[g][k] * scale.first * scale.second;
                const __half h = __float2half_rn(p);
                const uint32_t at = (y >> 6) * 16384 + swizzled(x + k, (y & 63) >> 3) + (y & 7) * 2;
                *(__half*)(base + kSmallHi + at) = h;
                if (pair) *(__half*)(base + kSmallLo + at) = __float2half_rn(p - __half2float(h));
            }
        }
    }

    // fp32 sums, fp16 operands, M = 128
    const uint32_t idesc = (1u << 4) | (8u << 24), idesc_m = idesc | (m16 / 8 << 17), idesc_x = idesc | (1u << 16) | (w16 / 8 << 17);
    const uint32_t quarter = warp & 3, part = warp >> 2, row = quarter * 32 + lane, lanes = (quarter * 32) << 16;     // part: of the columns
    uint32_t phase = 0;
    // The products of one phase issued by one thread, waited for by all.  A thread whose wait has run out issues nothing and waits for no products
    // any more; it still takes part in the barriers of the block and the cluster.
    bool ok = true;
    auto run = [&](auto issue) {
        fence_async();
        __syncthreads();
        if (tid == 0 && ok) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            issue();
            mma_commit<1>(bar);
        }
        if (ok) ok = mbar_wait(bar, phase, s.waits);
        phase ^= 1;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        __syncwarp();
    };
    // every thread has read what it needs of the accumulators before the next products overwrite them
    auto read_done = [&] { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); };

    for (int step = 0; step < a.steps; ++step) {
        const bool two = PRECISE || step < a.steps - 2;
        run([&] {                                // Y Y^T, this block's columns
            for (uint32_t k = 0; k < w16 / 16; ++k) {
                const uint64_t d = smem_desc(base32 + kSmallHi + (k >> 2) * 16384, false) + 2 * (k & 3);
                mma_f16<1>(tmem, d, d, idesc_m, k != 0);
                if (PRECISE) {
                    const uint64_t low = smem_desc(base32 + kSmallLo + (k >> 2) * 16384, false) + 2 * (k & 3);
                    mma_f16<1>(tmem, d, low, idesc_m, 1);
                    mma_f16<1>(tmem, low, d, idesc_m, 1);
                }
            }
        });
        const uint32_t col = part * 32;
        const bool mine = quarter * 32 < s.m && col < m16;       // this warp's rows and columns of the square matrices
        float v[32];
        if (mine) tmem_load32(tmem + col + lanes, v);
        if (S == 1) {
            if (mine) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= kUnscale;
                put32(base + kSmallGram, row, col, v);
                if (PRECISE) {
                    leave_low(v);
                    put32(base + kGramLo, row, col, v);
                }
            }
        } else {
            if (mine) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *(float4*)(base + kSmallGram + row * 512 + (((col >> 2) + i) ^ (row & 7)) * 16) =
                        make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
            read_done();
            cluster_sync_all();                  // everybody's share is there
            const uint32_t each = 128 / S, total4 = each * 32;           // rows of this block, in float4s: up to four a thread
            float4 t[4];
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                t[q] = make_float4(0, 0, 0, 0);
                const uint32_t item = q * kSmallThreads + tid;
                if (item >= total4) continue;
                const uint32_t r = rank * each + (item >> 5), c4 = item & 31;
                const uint32_t local = base32 + kSmallGram + r * 512 + (c4 ^ (r & 7)) * 16;
                for (uint32_t k = 0; k < S; ++k) {
                    float4 f;
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(f.x), "=f"(f.y), "=f"(f.z), "=f"(f.w) : "r"(map_to(local, k)) : "memory");
                    t[q].x += f.x; t[q].y += f.y; t[q].z += f.z; t[q].w += f.w;
                }
            }
            cluster_sync_all();                  // everybody has read: the space becomes A and P
#pragma unroll
            for (uint32_t q = 0; q < 4; ++q) {
                const uint32_t item = q * kSmallThreads + tid;
                if (item >= total4) continue;
                const uint32_t r = rank * each + (item >> 5), c4 = item & 31;
                const uint32_t local = base32 + kSmallGram + (c4 >> 4) * 16384 + swizzled(r, (c4 & 15) >> 1) + (c4 & 1) * 8;
                const uint32_t lo = pack16(t[q].x * kUnscale, t[q].y * kUnscale, false), hi = pack16(t[q].z * kUnscale, t[q].w * kUnscale, false);
                for (uint32_t k = 0; k < S; ++k) asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(map_to(local, k)), "r"(lo), "r"(hi) : "memory");
                if (PRECISE) {
                    const float2 f = __half22float2(*(const __half2*)&lo), g = __half22float2(*(const __half2*)&hi);
                    const uint32_t lo2 = pack16(t[q].x * kUnscale - f.x, t[q].y * kUnscale - f.y, false),
                                   hi2 = pack16(t[q].z * kUnscale - g.x, t[q].w * kUnscale - g.y, false);
                    for (uint32_t k = 0; k < S; ++k)
                        asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(map_to(local + kGramLo - kSmallGram, k)), "r"(lo2), "r"(hi2) : "memory");
                }
            }
            fence_async();
            cluster_sync_all();
        }
        read_done();
        run([&] {                                // A^2
            for (uint32_t k = 0; k < m16 / 16; ++k) {
                const uint64_t d = smem_desc(base32 + kSmallGram + (k >> 2) * 16384, false) + 2 * (k & 3);
                mma_f16<1>(tmem_sq, d, d, idesc_m, k != 0);
                if (PRECISE) {
                    const uint64_t low = smem_desc(base32 + kGramLo + (k >> 2) * 16384, false) + 2 * (k & 3);
                    mma_f16<1>(tmem_sq, d, low, idesc_m, 1);
                    mma_f16<1>(tmem_sq, low, d, idesc_m, 1);
                }
            }
        });
        if (mine) {
            tmem_load32(tmem_sq + col + lanes, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint4 w = *(const uint4*)(base + kSmallGram + (col >> 6) * 16384 + swizzled(row, ((col & 63) >> 3) + i));
                const uint32_t g[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float2 f = __half22float2(*(const __half2*)&g[k]);
                    v[8 * i + 2 * k] = a.coefficient[1] * f.x + a.coefficient[2] * kUnscale * v[8 * i + 2 * k];
                    v[8 * i + 2 * k + 1] = a.coefficient[1] * f.y + a.coefficient[2] * kUnscale * v[8 * i + 2 * k + 1];
                }
                if (PRECISE) {
                    const uint4 x = *(const uint4*)(base + kGramLo + (col >> 6) * 16384 + swizzled(row, ((col & 63) >> 3) + i));
                    const uint32_t l[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 f = __half22float2(*(const __half2*)&l[k]);
                        v[8 * i + 2 * k] += a.coefficient[1] * f.x;
                        v[8 * i + 2 * k + 1] += a.coefficient[1] * f.y;
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i == row) v[i] += a.coefficient[0] * kScale;
            put32(base + kP, row, col, v);
            if (PRECISE) {
                leave_low(v);
                put32(base + kPLo, row, col, v);
            }
        }
        read_done();
        run([&] {                                // P Y, with both matrices of the pair while there are two
            for (uint32_t which = 0; which < (two ? 2u : 1u); ++which)
                for (uint32_t k = 0; k < m16 / 16; ++k)
                    mma_f16<1>(tmem_x, smem_desc(base32 + kP + (k >> 2) * 16384, false) + 2 * (k & 3),
                               smem_desc(base32 + (which ? kSmallLo : kSmallHi), true, 16384) + 128 * k, idesc_x, (which | k) != 0);
            if (PRECISE)
                for (uint32_t k = 0; k < m16 / 16; ++k)
                    mma_f16<1>(tmem_x, smem_desc(base32 + kPLo + (k >> 2) * 16384, false) + 2 * (k & 3), smem_desc(base32 + kSmallHi, true, 16384) + 128 * k,
                               idesc_x, 1);
        });
        const bool last = step + 1 == a.steps, next_two = PRECISE || step + 1 < a.steps - 2;
#pragma unroll 1
        for (uint32_t col = quarter * 32 < s.m ? part * 32 : w16; col < w16; col += 32 * (kSmallThreads / 128)) {
            __syncwarp();
            tmem_load32(tmem_x + col + lanes, v);
            if (!last) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= kUnscale;
                put32(base + kSmallHi, row, col, v);
                if (next_two) {
                    leave_low(v);
                    put32(base + kSmallLo, row, col, v);
                }
                continue;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= kUnscale * kUnscale;
            const uint32_t row0 = quarter * 32;
            if (col >= width) continue;
            uint16_t* out = (uint16_t*)a.out + batch * a.stride_out;
            if (!s.tall) {
                store_tile32(out + first, a.out_type, a.ld_out, row0, min(s.m - row0, 32u), col, width, v, s.align,
                             base32 + kSmallGram + warp * kStageWords * 4, false, true);
            } else if (row < s.m) {              // the lanes' rows are the output's neighbouring columns
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (col + i < width) store_as(out, a.out_type, (uint64_t)(first + col + i) * a.ld_out + row, v[i]);
            }
        }
        read_done();
    }
    __syncthreads();
    if (S > 1) cluster_sync_all();               // nobody leaves while its shared memory may be read
    if (warp == 0) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        tmem_free<1>(tmem, 512);
    }
}

bool is_small(const OrthoArgs& a) {
    const uint64_t m = a.rows < a.cols ? a.rows : a.cols, n = a.rows < a.cols ? a.cols : a.rows;
    return m <= kSmallSide && n <= kSmallCluster * kSmallCols;
}
cudaError_t launch_small(const OrthoArgs& a, uint32_t align, const OpDevice& dev, cudaStream_t st) {
    SmallArgs s{a};
    s.tall = a.rows > a.cols;
    s.m = (uint32_t)(s.tall ? a.cols : a.rows);
    s.n = (uint32_t)(s.tall ? a.rows : a.cols);
    s.blocks = 1;
    while (s.blocks * kSmallCols < s.n) s.blocks *= 2;
    s.align = align;
    const uint64_t fast = a.cols;
    auto vec8 = [&](const void* p, uint64_t ld, uint64_t stride, uint32_t size) {
        return fast % 8 == 0 && (uintptr_t)p % 16 == 0 && ld * size % 16 == 0 && (a.batch == 1 || stride * size % 16 == 0);
    };
    s.vec_u = vec8(a.update, a.ld_update, a.stride_update, type_size(a.type));
    s.vec_m = a.momentum && vec8(a.momentum, a.ld_momentum, a.stride_momentum, 4);
    s.waits = dev.waits();
    constexpr int kSmem = (int)kSmallBytes + 1024;
    auto kernel = a.out_type == SK_F16 ? k_ortho_small<true> : k_ortho_small<false>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e == cudaSuccess && s.blocks > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)a.batch * s.blocks);
    cfg.blockDim = dim3(kSmallThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = s.blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = s.blocks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, s);
}

}  // namespace

template <bool SLICED, bool PRECISE>
cudaError_t launch_chain(bool wide, const ChainShape& p, const ChainLow& low, const ChainArgs& ea, uint32_t units, cudaStream_t st) {
    using Plan = ChainPlan<SLICED, PRECISE>;
    using Epi = ChainEpi<SLICED, PRECISE>;
    Plan plan{};
    static_cast<ChainShape&>(plan) = p;
    if constexpr (PRECISE) static_cast<ChainLow&>(plan) = low;
    auto launch = wide ? launch_plan<2, 256, Plan, Epi> : launch_plan<1, 128, Plan, Epi>;
    return launch(false, plan, ea, units, st);
}

uint64_t orthogonalize_workspace(const OrthoArgs& a) { return is_small(a) ? 0 : layout_of(a).total; }

int launch_orthogonalize(const OrthoArgs& a, const OpDevice& dev, uint32_t withhold_ms, cudaStream_t st) {
    const uint32_t align_rows = row_alignment(a.out, a.ld_out, a.out_type), align_batch = row_alignment(a.out, a.stride_out, a.out_type);
    const uint32_t align = a.batch > 1 && align_batch < align_rows ? align_batch : align_rows;
    if (is_small(a)) {
        SK_OP_CUDA(launch_small(a, align, dev, st));
        return SK_OK;
    }
    const OrthoLayout l = layout_of(a);
    uint8_t* ws = (uint8_t*)a.workspace;
    double* partial = (double*)(ws + l.off_partial);
    __half* x[2] = {(__half*)(ws + l.off_x[0]), (__half*)(ws + l.off_x[1])};
    __half* lo[2] = {(__half*)(ws + l.off_lo), (__half*)(ws + l.off_lo + round_up(a.batch * l.x_elems * 2, 256))};
    __half* gram = (__half*)(ws + l.off_a);
    __half* poly = (__half*)(ws + l.off_p);
    const bool tall = a.rows > a.cols;
    const uint32_t batch = (uint32_t)a.batch, m = l.m;
    // two 16-bit matrices for X in all but the last two steps, and one where that is exact
    const bool exact = a.type != SK_F32 && !a.momentum, precise = a.out_type == SK_F16;
    auto split = [&](int step) { return (precise || step < a.steps - 2) && !(step == 0 && exact); };

    const uint32_t blocks = (uint32_t)((a.rows * ((a.cols + 7) / 8) + 255) / 256);
    const uint32_t most = (uint32_t)(round_up((uint64_t)dev.sm_count * 8, batch) / batch), limit = most < kNormBlocks ? most : kNormBlocks;
    SquareArgs sq{a, partial, (float*)(ws + l.off_factor), blocks < limit ? blocks : limit};
    auto vec8 = [&](const void* p, uint64_t ld, uint64_t stride, uint32_t size) {
        return a.cols % 8 == 0 && (uintptr_t)p % 16 == 0 && ld * size % 16 == 0 && (batch == 1 || stride * size % 16 == 0);
    };
    sq.vec_u = vec8(a.update, a.ld_update, a.stride_update, type_size(a.type));
    sq.vec_m = a.momentum && vec8(a.momentum, a.ld_momentum, a.stride_momentum, 4);
    sq.hi = x[0];
    sq.lo = split(0) ? lo[0] : nullptr;
    sq.ld = l.ld_x;
    sq.stride = l.x_elems;
    sq.exact = exact;
    sq.count = (uint32_t*)(ws + l.off_count);
    SK_OP_CUDA(launch_kernel(true, k_ortho_square, dim3(sq.blocks, batch), 256, 0, st, sq));
    SK_OP_CUDA(launch_kernel(true, k_ortho_scale, dim3(sq.blocks, batch), 256, 0, st, sq));

    ChainArgs ea{};
    ea.gram = gram;
    ea.poly = poly;
    ea.gram_lo = (__half*)(ws + l.off_a_lo);
    ea.poly_lo = (__half*)(ws + l.off_p_lo);
    for (int i = 0; i < 2; ++i) { ea.hi[i] = x[i]; ea.lo[i] = lo[i]; }
    ea.a_stride = l.a_elems;
    ea.x_stride = l.x_elems;
    ea.ld_a = l.ld_a;
    ea.ld_x = l.ld_x;
    ea.a = a.coefficient[0];
    ea.b = a.coefficient[1];
    ea.c = a.coefficient[2];
    ea.factor = sq.factor;
    ea.out = a.out;
    ea.out_stride = a.stride_out;
    ea.ld_out = a.ld_out;
    ea.out_type = a.out_type;
    ea.align = align;
    ea.steps = (uint32_t)a.steps;

    ChainShape p{};
    ChainLow low{};
    bool ok = true;
    for (int i = 0; i < 2; ++i) {
        const Operand g{x[i], a.rows, a.cols, l.ld_x, l.x_elems, batch, tall}, h{x[i], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall},
            o{lo[i], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall};
        ok = ok && encode_operand(&p.gram_x[i], g, false, g.mn ? 64 : 128) && encode_operand(&p.apply_hi[i], h, false, h.mn ? 64 : 128) &&
             encode_operand(&p.apply_lo[i], o, false, o.mn ? 64 : 128);
        if (precise) {
            const Operand gl{lo[i], a.rows, a.cols, l.ld_x, l.x_elems, batch, tall};
            ok = ok && encode_operand(&low.gram_xlo[i], gl, false, gl.mn ? 64 : 128);
        }
    }
    const Operand oa{gram, m, m, l.ld_a, l.a_elems, batch, false}, op{poly, m, m, l.ld_a, l.a_elems, batch, false};
    ok = ok && encode_operand(&p.gram, oa, false, 128) && encode_operand(&p.poly, op, false, 128);
    if (precise) {
        const Operand al{ea.gram_lo, m, m, l.ld_a, l.a_elems, batch, false}, pl{ea.poly_lo, m, m, l.ld_a, l.a_elems, batch, false};
        ok = ok && encode_operand(&low.gram_lo, al, false, 128) && encode_operand(&low.poly_lo, pl, false, 128);
    }
    if (!ok) return set_error(SK_ECUDA, "sk_orthogonalize: a tensor map was refused");
    p.steps = (uint32_t)a.steps;
    p.exact = exact;
    p.tall = tall;
    p.batch = batch;
    p.m = m;
    p.rows = (uint32_t)a.rows;
    p.cols = (uint32_t)a.cols;
    p.k_poly = (m + kGemmK - 1) / kGemmK;
    p.k_gram = (uint32_t)(((tall ? a.rows : a.cols) + kGemmK - 1) / kGemmK);
    p.count = sq.count;
    p.waits = dev.waits();
    const ChainTiles c = chain_tiles(a, precise);
    const uint32_t tile = c.wide ? 256 : 128, slots = (uint32_t)dev.sm_count / (c.wide ? 2 : 1);
    p.side = (m + tile - 1) / tile;
    p.square = p.side * (p.side + 1) / 2;
    p.tiles_m = (p.rows + tile - 1) / tile;
    p.tiles_n = (p.cols + tile - 1) / tile;
    p.apply = p.tiles_m * p.tiles_n;
    p.slices = c.slices;
    p.k_slice = (p.k_gram + c.slices - 1) / c.slices;
    if (c.slices > 1) {
        ea.slices = (float*)(ws + l.off_slices);
        ea.slice_stride = batch * l.a_elems;
        ea.slice_count = c.slices;
        ea.join_cols = tile / ChainEpi<true, false>::kWarps;
    }
    p.signals = (c.wide ? 2 : 1) * ChainEpi<true, false>::kWarps;
    if ((uint64_t)a.steps * batch * ((c.slices > 1 ? 1ull + c.slices + kJoinParts : 2ull) * p.square + p.apply) * p.signals >= (1ull << 32))
        return set_error(SK_EINVAL, "sk_orthogonalize: batch * rows * cols is too large for one call");
    if (withhold_ms) {                           // every wait asks for more than the tiles' warps ever count
        ++p.signals;
        p.waits.limit_ms = withhold_ms;
    }
    const uint32_t most_tiles = batch * (p.square * p.slices > p.apply ? p.square * p.slices : p.apply), units = most_tiles < slots ? most_tiles : slots;
    auto launch = c.slices > 1 ? precise ? launch_chain<true, true> : launch_chain<true, false> : precise ? launch_chain<false, true> : launch_chain<false, false>;
    SK_OP_CUDA(launch(c.wide, p, low, ea, units, st));
    return SK_OK;
}

}  // namespace sk
