// Layer norm over the last axis, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) r w + b
//   h = (x - mu) r, g = dy w:  dx = r (g - mean(g) - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: forward reads x and writes y once, backward reads x and dy and writes dx once.  A row belongs to 8 or 32
// lanes of a warp or to a block, every thread to fixed columns.  What keeps the memory busy is a ring of rows in
// shared memory that each thread fills for itself with asynchronous copies (its own columns only, so no barrier guards
// it): the next rows travel while one is worked on, without holding registers.  Rows of odd lengths do so too, with accesses
// that begin before the row (Place); only matrices whose rows lie differently to the 16-byte boundary come element by element,
// 16-bit ones through registers.  The arithmetic is two values to an instruction (f32x2): with one the kernels are bound by
// issue (bf16 rows then take as long as fp32 ones).  Measured: 32768 x 4096 bf16 90 us forward (5.9 TB/s), 141 us backward (5.7);
// 32768 x 4096 fp32 166 and 244 us (6.5, 6.6 TB/s); weights read for every row from L1 instead of registers cost 274 us in the first.
//
// Statistics: a warp computes the mean of its part and the squares around that, and the parts are joined by the formula for
// the variance of a union: nothing cancels whatever the mean, and warps meet once per row.  In the backward pass the sums of
// dw and db stay in registers, and every block writes one partial row of them that a second, column-parallel kernel adds
// up in a fixed order (for few rows extra blocks form them instead): no atomics, the same bits every time.  All
// statistics and sums are 32-bit.
#include "sk_chain.cuh"
#include "sk_operators.h"

#include <atomic>
#include <type_traits>

namespace sk {
namespace {

constexpr int kDepth = 3;                        // rows of the ring
constexpr int kWarpThreads = 128;                // block of the kernels with several groups of lanes to a block

// ---- a thread's elements of a row: NV accesses of V neighbours, in NV * V / 2 pairs (of accesses where V is 1) ---------------
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

template <typename T, int V, int NV>
__device__ __forceinline__ void unpack(const Pack<T, V> (&p)[NV], F2 (&o)[NV * V / 2]) {
    if constexpr (V == 1) {
#pragma unroll
        for (int q = 0; q < NV / 2; ++q) o[q] = f2(to_float(p[2 * q].v[0]), to_float(p[2 * q + 1].v[0]));
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                F2& d = o[i * V / 2 + j];
                if constexpr (sizeof(T) == 4) {
                    d = f2(to_float(p[i].v[2 * j]), to_float(p[i].v[2 * j + 1]));
                } else {
                    const uint32_t w = ((const uint32_t*)&p[i])[j];
                    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                        d = f2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
                    } else {
                        const float2 f = __half22float2(*(const __half2*)&w);
                        d = f2(f.x, f.y);
                    }
                }
            }
    }
}
// Where a thread's accesses lie in the row.  SHIFT: the rows start off the 16-byte boundary; accesses stay on it and begin `shift` elements
// before the row, so the row's first and last one hold elements that are not the row's.  The shift is the same for all rows of a
// thread (they are a multiple of 16 bytes apart), and so its columns are.
template <int V, bool SHIFT>
struct Place {
    uint32_t t, tpr, cols, shift;
    __device__ __forceinline__ int col(int i) const { return (int)((i * tpr + t) * V) - (SHIFT ? (int)shift : 0); }
    __device__ __forceinline__ bool in(int i) const { return col(i) < (int)cols; }                       // any of it
    __device__ __forceinline__ bool whole(int i) const { return !SHIFT || (col(i) >= 0 && col(i) + V <= (int)cols); }
    __device__ __forceinline__ bool valid(int i, int j) const { return col(i) + j < (int)cols && (!SHIFT || col(i) + j >= 0); }
    // pair q with its elements beyond the row set to zero
    __device__ __forceinline__ F2 pair_only(int q, F2 d) const {
        const int i = V == 1 ? 2 * q : q / (V > 1 ? V / 2 : 1), j = V == 1 ? 0 : 2 * (q - i * (V / 2));
        const float2 f = parts(d);
        return f2(valid(i, j) ? f.x : 0.0f, (V == 1 ? valid(i + 1, 0) : valid(i, j + 1)) ? f.y : 0.0f);
    }
};
template <typename T, int V, int NV, bool SHIFT>
__device__ __forceinline__ void store(T* row, const F2 (&o)[NV * V / 2], const Place<V, SHIFT>& at) {
    if constexpr (V == 1) {
#pragma unroll
        for (int q = 0; q < NV / 2; ++q) {
            const float2 f = parts(o[q]);
            if (at.in(2 * q)) row[at.col(2 * q)] = from_float<T>(f.x);
            if (at.in(2 * q + 1)) row[at.col(2 * q + 1)] = from_float<T>(f.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Pack<T, V> p;
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                const float2 f = parts(o[i * V / 2 + j]);
                if constexpr (sizeof(T) == 4) {
                    p.v[2 * j] = from_float<T>(f.x);
                    p.v[2 * j + 1] = from_float<T>(f.y);
                } else {
                    ((uint32_t*)&p)[j] = pack16(f.x, f.y, std::is_same<T, __nv_bfloat16>::value);
                }
            }
            if (!at.in(i)) continue;
            if (at.whole(i)) {
                *(Pack<T, V>*)(row + at.col(i)) = p;
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (at.valid(i, j)) row[at.col(i) + j] = p.v[j];
            }
        }
    }
}
// The weights of pair q (`none` without a weight vector or beyond the row).
template <int V, bool SHIFT>
__device__ __forceinline__ F2 weights_of(const void* p, int type, float none, int q, const Place<V, SHIFT>& at) {
    const int i = V == 1 ? 2 * q : q / (V > 1 ? V / 2 : 1), j = V == 1 ? 0 : 2 * (q - i * (V / 2));
    if (!p) return f2(none, none);
    if (V > 1 && !SHIFT && type == SK_F32 && (uintptr_t)p % 8 == 0) {
        if (!at.in(i)) return f2(none, none);
        const float2 f = *(const float2*)((const float*)p + at.col(i) + j);
        return f2(f.x, f.y);
    }
    const int i2 = V == 1 ? i + 1 : i, j2 = V == 1 ? 0 : j + 1;
    return f2(at.valid(i, j) ? load_as(p, type, at.col(i) + j) : none, at.valid(i2, j2) ? load_as(p, type, at.col(i2) + j2) : none);
}

// ---- the rows on their way -------------------------------------------------------------------------------------------------
template <int BYTES>
__device__ __forceinline__ void copy_async(void* dst, const void* src, uint32_t bytes) {       // zeroes beyond `bytes`
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(d), "l"(src), "n"(BYTES), "r"(bytes) : "memory");
}

// A thread's columns of N matrices' rows.
template <typename T, int V, int NV, int N, bool SHIFT>
struct Rows {
    static constexpr bool kAsync = sizeof(T) * V >= 4;
    using P = Pack<T, V>;
    static constexpr uint32_t smem(uint32_t threads) { return kAsync ? kDepth * N * NV * threads * (uint32_t)sizeof(P) : 0; }
    const T* src[N];
    uint64_t ld[N], rows;
    Place<V, SHIFT> at;
    P* ring;                                     // [kDepth][N][NV][blockDim.x]
    P ahead[kAsync ? 1 : N][kAsync ? 1 : NV];
    const T* next[N];                            // the thread's first column of the row to ask for next
    uint64_t next_row;

    __device__ __forceinline__ P* slot(uint32_t s, int n, int i) const { return ring + ((s * N + n) * NV + i) * blockDim.x + threadIdx.x; }
    __device__ __forceinline__ void issue(uint64_t step, uint32_t s) {
        const bool live = next_row < rows;
#pragma unroll
        for (int n = 0; n < N; ++n) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const bool in = live && at.in(i);
                const T* p = next[n] + i * at.tpr * V;
                if constexpr (kAsync) {
                    uint32_t bytes = in ? (uint32_t)sizeof(P) : 0;
                    if constexpr (SHIFT) {
                        const int left = (int)at.cols - at.col(i);               // the row's end: no further
                        if (in && left < V) bytes = (uint32_t)left * sizeof(T);
                        if (i == 0 && in && p < src[n]) {                        // the matrix' start: the row's own elements one by one
                            P one;
#pragma unroll
                            for (int j = 0; j < V; ++j) one.v[j] = at.valid(0, j) ? p[j] : from_float<T>(0.0f);
                            *slot(s, n, 0) = one;
                            continue;
                        }
                    }
                    copy_async<(int)sizeof(P)>(slot(s, n, i), in ? p : (const T*)((uintptr_t)src[n] & ~(uintptr_t)15), bytes);
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) ahead[n][i].v[j] = from_float<T>(0.0f);
                    if (in) ahead[n][i] = *(const P*)p;
                }
            }
            next[n] += step * ld[n];
        }
        next_row += step;
        if constexpr (kAsync) asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ void start(uint64_t row, uint64_t step) {
        next_row = row;
#pragma unroll
        for (int n = 0; n < N; ++n) next[n] = src[n] + row * ld[n] + at.col(0);
        issue(step, 0);
        if constexpr (kAsync)
#pragma unroll
            for (int d = 1; d < kDepth - 1; ++d) issue(step, d);
    }
    // the row asked for longest ago, and the one kDepth - 1 (through registers: one) rows on asked for
    __device__ __forceinline__ void take(uint64_t step, uint32_t& s, P (&out)[N][NV]) {
        if constexpr (kAsync) {
            const uint32_t to = s == 0 ? kDepth - 1 : s - 1;
            issue(step, to);
            asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < NV; ++i) out[n][i] = *slot(s, n, i);
            if constexpr (SHIFT) {
                if (at.col(0) < 0) {                                             // what stands before the row
#pragma unroll
                    for (int n = 0; n < N; ++n)
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            if (!at.valid(0, j)) out[n][0].v[j] = from_float<T>(0.0f);
                }
            }
            s = s + 1 == kDepth ? 0 : s + 1;
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int i = 0; i < NV; ++i) out[n][i] = ahead[n][i];
            issue(step, 0);
        }
    }
};
// elements from the 16-byte boundary before a row to the row's start
template <typename T>
__device__ __forceinline__ uint32_t shift_of(const void* p, uint64_t ld, uint64_t row) {
    return (uint32_t)(((uintptr_t)p + row * ld * sizeof(T)) % 16 / sizeof(T));
}

template <int G>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = (G ? G : 32) / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// G lanes of a warp per row, or (G = 0) the block; threads per row * NV * V >= cols
template <typename T, int V, int NV, int G, int MAXT, int BLOCKS, bool SHIFT>
__global__ void __launch_bounds__(MAXT, BLOCKS) k_norm(const NormArgs a) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float2 warp_stats[2][32];
    constexpr int kQ = NV * V / 2;
    const uint32_t tpr = G ? G : blockDim.x, groups = blockDim.x / tpr, warps = blockDim.x >> 5;
    const uint64_t step = (uint64_t)gridDim.x * groups;
    uint64_t base = (uint64_t)blockIdx.x * groups, row = base + threadIdx.x / tpr;
    const Place<V, SHIFT> at{threadIdx.x % tpr, tpr, (uint32_t)a.cols, SHIFT ? shift_of<T>(a.x, a.ld_x, row) : 0};
    // columns of the row that the row's lanes, or warp `w` of the block, hold
    auto count_of = [&](uint32_t w) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int start = (int)((i * tpr + w * 32) * V) - (SHIFT ? (int)at.shift : 0), from = max(start, 0);
            const int to = min(start + (G ? G : 32) * V, (int)at.cols);
            n += max(to - from, 0);
        }
        return (float)n;
    };
    const uint32_t lane = threadIdx.x & 31;
    const float part = count_of(G ? 0 : threadIdx.x >> 5), part_inv = part > 0 ? 1.0f / part : 0.0f, inv = 1.0f / (float)at.cols;
    const float lane_n = G == 0 && lane < warps ? count_of(lane) : 0.0f, lane_inv = lane_n > 0 ? 1.0f / lane_n : 0.0f;   // of warp `lane`
    chain_acquire();
    F2 w[kQ], b[kQ];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        w[q] = weights_of<V, SHIFT>(a.weight, a.w_type, 1.0f, q, at);
        b[q] = weights_of<V, SHIFT>(a.bias, a.w_type, 0.0f, q, at);
    }
    Rows<T, V, NV, 1, SHIFT> in{{(const T*)a.x}, {a.ld_x}, a.rows, at, (Pack<T, V>*)ring};
    in.start(row, step);
    uint32_t slot = 0, turn = 0;
    for (; base < a.rows; base += step, row += step, turn ^= 1) {             // every lane stays in the loop
        Pack<T, V> x[1][NV];
        F2 v[kQ];
        in.take(step, slot, x);
        unpack<T, V, NV>(x[0], v);
        F2 s = f2(0, 0);
#pragma unroll
        for (int q = 0; q < kQ; ++q) s = s + v[q];
        float2 f = parts(s);
        float mean = lanes_sum<G>(f.x + f.y) * part_inv;
        s = f2(0, 0);
        F2 minus = f2(-mean, -mean);
        if constexpr (V == 1) {
#pragma unroll
            for (int q = 0; q < kQ; ++q) {
                const F2 d = at.pair_only(q, v[q] + minus);
                s = fma2(d, d, s);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!at.in(i)) continue;
                if (at.whole(i)) {
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) {
                        const F2 d = v[i * V / 2 + j] + minus;
                        s = fma2(d, d, s);
                    }
                } else {                                  // a row's first or last access
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) {
                        const F2 d = at.pair_only(i * V / 2 + j, v[i * V / 2 + j] + minus);
                        s = fma2(d, d, s);
                    }
                }
            }
        }
        f = parts(s);
        float squares = lanes_sum<G>(f.x + f.y);
        if constexpr (G == 0) {
            if ((threadIdx.x & 31) == 0) warp_stats[turn][threadIdx.x >> 5] = make_float2(mean * part, squares);
            __syncthreads();                              // two sets in turn: nobody is a whole row ahead of a reader
            const float2 q = lane < warps ? warp_stats[turn][lane] : make_float2(0, 0);       // a lane for every warp
            mean = lanes_sum<32>(q.x) * inv;
            const float d = q.x * lane_inv - mean;
            squares = lanes_sum<32>(q.y + d * d * lane_n);
        }
        const float rstd = rsqrtf(squares * inv + a.eps);
        if (G && row >= a.rows) continue;
        minus = f2(-mean, -mean);
        const F2 scale = f2(rstd, rstd);
#pragma unroll
        for (int q = 0; q < kQ; ++q) v[q] = fma2((v[q] + minus) * scale, w[q], b[q]);
        store<T, V, NV, SHIFT>((T*)a.y + row * a.ld_y, v, at);
        if (at.t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
    if constexpr (Rows<T, V, NV, 1, SHIFT>::kAsync) asm volatile("cp.async.wait_all;" ::: "memory");
}

// Sums of a row over a block's threads (the long-row kernels)
template <int N>
__device__ __forceinline__ void block_sum(float (&v)[N], float (*scratch)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = lanes_sum<32>(v[k]);
    const uint32_t warps = blockDim.x >> 5;
    __syncthreads();                                      // the previous sums have been read by everybody
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) scratch[threadIdx.x >> 5][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = scratch[0][k];
    for (uint32_t i = 1; i < warps; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += scratch[i][k];
}

// Rows longer than the register kernels hold: the block looks at the row three times, the later looks from L2.
constexpr int kLongThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_long(const NormArgs a) {
    __shared__ float scratch[32][1];
    chain_acquire();
    const float inv = 1.0f / (float)a.cols;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = (const T*)a.x + row * a.ld_x;
        T* y = (T*)a.y + row * a.ld_y;
        float sum[1] = {0}, sq[1] = {0};
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) sum[0] += to_float(x[c]);
        block_sum<1>(sum, scratch);
        const float mean = sum[0] * inv;
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float d = to_float(x[c]) - mean;
            sq[0] += d * d;
        }
        block_sum<1>(sq, scratch);
        const float rstd = rsqrtf(sq[0] * inv + a.eps);
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float w = a.weight ? load_as(a.weight, a.w_type, c) : 1.0f, b = a.bias ? load_as(a.bias, a.w_type, c) : 0.0f;
            y[c] = from_float<T>((to_float(x[c]) - mean) * rstd * w + b);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// dw and db of a slab of columns over all rows: for few rows, as extra blocks of the row kernel's launch.  They read x and dy a second time,
// from L2, and need neither partial rows nor a kernel after them.  A row of the slab is 32 bytes in two 16-byte accesses, or eight
// single elements where rows do not lie on 16-byte boundaries.
template <int V> struct Slab { static constexpr uint32_t kCols = V > 1 ? 2 * V : 8; };
template <typename T, int V>
__device__ void norm_columns(const NormBackwardArgs& a, uint32_t slab, float2 (*sums)[Slab<V>::kCols]) {
    constexpr uint32_t kCols = Slab<V>::kCols, kLanes = kCols / V;           // lanes to a row
    const uint32_t x = threadIdx.x % kLanes, y = threadIdx.x / kLanes, groups = blockDim.x / kLanes;
    const uint64_t c = (uint64_t)slab * kCols + x * V;
    float2 s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = make_float2(0, 0);
    if (c < a.cols) {                            // a multiple of V
        const T *px = (const T*)a.x + c, *pd = (const T*)a.dy + c;
#pragma unroll(V > 1 ? 4 : 8)
        for (uint32_t r = y; r < (uint32_t)a.rows; r += groups) {
            const Pack<T, V> dy = *(const Pack<T, V>*)(pd + r * a.ld_dy), in = *(const Pack<T, V>*)(px + r * a.ld_x);
            const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float d = to_float(dy.v[k]);
                s[k].x += d * ((to_float(in.v[k]) - mean) * rstd);
                s[k].y += d;
            }
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
#pragma unroll
        for (int o = kLanes; o < 32; o *= 2) {
            s[k].x += __shfl_xor_sync(0xffffffffu, s[k].x, o);
            s[k].y += __shfl_xor_sync(0xffffffffu, s[k].y, o);
        }
        if ((threadIdx.x & 31) < kLanes) sums[threadIdx.x >> 5][x * V + k] = s[k];
    }
    __syncthreads();
    const uint64_t col = (uint64_t)slab * kCols + threadIdx.x;
    if (threadIdx.x < kCols && col < a.cols) {
        float2 t = sums[0][threadIdx.x];
        for (uint32_t w = 1; w < (blockDim.x >> 5); ++w) {
            t.x += sums[w][threadIdx.x].x;
            t.y += sums[w][threadIdx.x].y;
        }
        if (a.dweight) store_as(a.dweight, a.dw_type, col, t.x);
        if (a.dbias) store_as(a.dbias, a.dw_type, col, t.y);
    }
}

template <typename T, int V, int NV, int G, int MAXT, int BLOCKS, bool SHIFT>
__global__ void __launch_bounds__(MAXT, BLOCKS) k_norm_backward(const NormBackwardArgs a) {
    extern __shared__ __align__(16) uint8_t ring[];
    __shared__ float2 warp_sums[2][32];
    __shared__ float gather[G ? kWarpThreads * NV * V : 1];
    constexpr int kQ = NV * V / 2;
    const uint32_t tpr = G ? G : blockDim.x, groups = blockDim.x / tpr, warps = blockDim.x >> 5;
    const uint64_t step = (uint64_t)(gridDim.x - a.slabs) * groups;
    uint64_t base = (uint64_t)blockIdx.x * groups, row = base + threadIdx.x / tpr;
    const Place<V, SHIFT> at{threadIdx.x % tpr, tpr, (uint32_t)a.cols, SHIFT ? shift_of<T>(a.x, a.ld_x, row) : 0};
    const float inv = 1.0f / (float)at.cols;
    chain_acquire();
    if (blockIdx.x >= gridDim.x - a.slabs) {
        constexpr int kV = SHIFT ? 1 : V;
        __shared__ float2 sums[MAXT / 32][Slab<kV>::kCols];
        norm_columns<T, kV>(a, blockIdx.x - (gridDim.x - a.slabs), sums);
        return;
    }
    F2 w[kQ], dw[kQ], db[kQ];
#pragma unroll
    for (int q = 0; q < kQ; ++q) {
        w[q] = weights_of<V, SHIFT>(a.weight, a.w_type, 1.0f, q, at);
        dw[q] = db[q] = f2(0, 0);
    }
    Rows<T, V, NV, 2, SHIFT> in{{(const T*)a.x, (const T*)a.dy}, {a.ld_x, a.ld_dy}, a.rows, at, (Pack<T, V>*)ring};
    in.start(row, step);
    uint32_t slot = 0, turn = 0;
    float next_mean = row < a.rows ? a.mean[row] : 0.0f, next_rstd = row < a.rows ? a.rstd[row] : 0.0f;
    for (; base < a.rows; base += step, row += step, turn ^= 1) {             // every lane stays in the loop
        Pack<T, V> v[2][NV];
        in.take(step, slot, v);
        const float mean = next_mean, rstd = next_rstd;
        const bool more = row + step < a.rows;
        next_mean = more ? a.mean[row + step] : 0.0f;
        next_rstd = more ? a.rstd[row + step] : 0.0f;
        const F2 minus = f2(-mean, -mean), scale = f2(rstd, rstd);
        F2 h[kQ], g[kQ], s1 = f2(0, 0), s2 = f2(0, 0);
        unpack<T, V, NV>(v[0], h);
        unpack<T, V, NV>(v[1], g);
#pragma unroll
        for (int q = 0; q < kQ; ++q) {                    // beyond the row dy is zero, and so is every term
            h[q] = (h[q] + minus) * scale;
            dw[q] = fma2(g[q], h[q], dw[q]);
            db[q] = db[q] + g[q];
            g[q] = g[q] * w[q];
            s1 = s1 + g[q];
            s2 = fma2(g[q], h[q], s2);
        }
        if (!a.dx) continue;
        const float2 p1 = parts(s1), p2 = parts(s2);
        float m1 = lanes_sum<G>(p1.x + p1.y), m2 = lanes_sum<G>(p2.x + p2.y);
        if constexpr (G == 0) {
            if ((threadIdx.x & 31) == 0) warp_sums[turn][threadIdx.x >> 5] = make_float2(m1, m2);
            __syncthreads();                              // two sets in turn: nobody is a whole row ahead of a reader
            m1 = m2 = 0;
            for (uint32_t k = 0; k < warps; ++k) {
                m1 += warp_sums[turn][k].x;
                m2 += warp_sums[turn][k].y;
            }
        }
        if (G && row >= a.rows) continue;
        m1 *= -inv * rstd;
        m2 *= -inv * rstd;
#pragma unroll
        for (int q = 0; q < kQ; ++q) g[q] = fma2(g[q], scale, fma2(h[q], f2(m2, m2), f2(m1, m1)));
        store<T, V, NV, SHIFT>((T*)a.dx + row * a.ld_dx, g, at);
    }
    if constexpr (Rows<T, V, NV, 2, SHIFT>::kAsync) asm volatile("cp.async.wait_all;" ::: "memory");
    if (!a.partial) return;
    float* out = a.partial + (uint64_t)blockIdx.x * 2 * at.cols;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float mine[NV * V];
#pragma unroll
        for (int q = 0; q < kQ; ++q) {
            const float2 f = parts(which ? db[q] : dw[q]);
            mine[2 * q] = f.x;
            mine[2 * q + 1] = f.y;
        }
        if constexpr (G != 0) {                           // the block's rows share their columns: one sum of them
            const uint32_t width = G * NV * V;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < NV * V; ++k)
                if (at.valid(k / V, k % V)) gather[(threadIdx.x / G) * width + at.col(k / V) + k % V] = mine[k];
            __syncthreads();
            for (uint32_t c = threadIdx.x; c < at.cols; c += blockDim.x) {
                float sum = 0;
                for (uint32_t k = 0; k < groups; ++k) sum += gather[k * width + c];
                out[(uint64_t)which * at.cols + c] = sum;
            }
        } else {
#pragma unroll
            for (int k = 0; k < NV * V; ++k)
                if (at.valid(k / V, k % V)) out[(uint64_t)which * at.cols + at.col(k / V) + k % V] = mine[k];
        }
    }
}

// Long rows, backward: the sums of a block are kept in its partial row in memory (own columns only, so no races).
template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_backward_long(const NormBackwardArgs a) {
    __shared__ float scratch[32][2];
    chain_acquire();
    const float inv = 1.0f / (float)a.cols;
    float* part = a.partial ? a.partial + (uint64_t)blockIdx.x * 2 * a.cols : nullptr;
    bool fresh = true;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, fresh = false) {
        const T* x = (const T*)a.x + row * a.ld_x;
        const T* dy = (const T*)a.dy + row * a.ld_dy;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s[2] = {0, 0};
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float h = (to_float(x[c]) - mean) * rstd, d = to_float(dy[c]);
            const float g = a.weight ? d * load_as(a.weight, a.w_type, c) : d;
            s[0] += g;
            s[1] += g * h;
            if (part) {
                part[c] = (fresh ? 0.0f : part[c]) + d * h;
                part[a.cols + c] = (fresh ? 0.0f : part[a.cols + c]) + d;
            }
        }
        block_sum<2>(s, scratch);
        if (!a.dx) continue;
        T* dx = (T*)a.dx + row * a.ld_dx;
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float h = (to_float(x[c]) - mean) * rstd;
            const float g = to_float(dy[c]) * (a.weight ? load_as(a.weight, a.w_type, c) : 1.0f);
            dx[c] = from_float<T>(rstd * (g - s[0] * inv - h * (s[1] * inv)));
        }
    }
}

// Adds the blocks' partial rows: eight columns to a block, 32 threads a column, in a fixed order.
__global__ void __launch_bounds__(256) k_norm_sum(const float* partial, uint32_t blocks, uint32_t cols, void* dweight, void* dbias, int type) {
    __shared__ float s[8][8];
    const uint32_t x = threadIdx.x & 7, y = threadIdx.x >> 3;
    const uint64_t c = (uint64_t)blockIdx.x * 8 + x, width = 2ull * cols;    // over both sums
    chain_acquire();
    float v = 0;
    if (c < width) {
#pragma unroll 8
        for (uint32_t b = y; b < blocks; b += 32) v += partial[b * width + c];
    }
    v += __shfl_xor_sync(0xffffffffu, v, 8);
    v += __shfl_xor_sync(0xffffffffu, v, 16);
    if ((threadIdx.x & 31) < 8) s[threadIdx.x >> 5][x] = v;
    __syncthreads();
    if (threadIdx.x < 8 && c < width) {
        v = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) v += s[i][x];
        void* out = c < cols ? dweight : dbias;
        if (out) store_as(out, type, c < cols ? c : c - cols, v);
    }
}

// Lanes per row (0: the block), threads of the block, values per thread.  More values a thread spread what a row costs each
// thread whatever its share (sums over lanes, addresses) over more of them.
struct NormPlan { uint32_t lanes, threads, per; };
NormPlan plan_lanes(uint64_t cols, uint32_t most) {          // a row to 8 or 32 lanes of a warp
    if (cols <= 64) return {8, kWarpThreads, 8};
    for (uint32_t per = 8; per <= most; per *= 2)
        if (cols <= 32 * per) return {32, kWarpThreads, per};
    return {0, 0, 0};
}
NormPlan plan_block(uint64_t cols, uint32_t per, uint32_t most) {
    const uint64_t threads = round_up((cols + per - 1) / per, 32);
    return threads <= most ? NormPlan{0, (uint32_t)threads, per} : NormPlan{0, 0, 0};
}
// Blocks: as many as stay resident, rows dealt out evenly over them.
uint32_t norm_blocks(uint64_t rows, const NormPlan& p, int sm_count, uint32_t threads_per_sm) {
    const uint64_t threads = p.threads ? p.threads : kLongThreads, groups = p.lanes ? threads / p.lanes : 1;
    const uint64_t want = (rows + groups - 1) / groups;
    const uint64_t per_sm = threads_per_sm / threads < 1 ? 1 : threads_per_sm / threads < 24 ? threads_per_sm / threads : 24;
    const uint64_t most = (uint64_t)sm_count * per_sm;
    if (want <= most) return (uint32_t)(want ? want : 1);
    const uint64_t rounds = (want + most - 1) / most, even = round_up((want + rounds - 1) / rounds, 8);
    return (uint32_t)(even <= most ? even : most / 8 * 8);       // a multiple of eight: a thread's rows are whole 16-byte steps apart
}

// What a kernel may take of shared memory is a property of the kernel on a device, not of a launch, and calls of other row lengths may be
// on their way in other threads: it is set once, to the most that any of its launches takes.
template <auto kernel, uint32_t MOST, typename Args>
cudaError_t launch_rows(dim3 grid, uint32_t threads, uint32_t smem, cudaStream_t st, const Args& a) {
    if constexpr (MOST > 24 * 1024) {            // with the kernel's own arrays, perhaps beyond what needs no permission
        static std::atomic<bool> prepared[64];
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        if (device >= 64 || !prepared[device]) {
            e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST);
            if (e != cudaSuccess) return e;
            if (device < 64) prepared[device] = true;
        }
    }
    return launch_kernel(true, kernel, grid, threads, smem, st, a);
}

template <typename T, int V, bool SHIFT, int PER, int G, int MAXT, int BLOCKS>
cudaError_t run_norm(const NormArgs& a, const NormPlan& p, int sm_count, cudaStream_t st) {
    using In = Rows<T, V, PER / V, 1, SHIFT>;
    return launch_rows<k_norm<T, V, PER / V, G, MAXT, BLOCKS, SHIFT>, In::smem(MAXT)>(dim3(norm_blocks(a.rows, p, sm_count, MAXT * BLOCKS)), p.threads,
                                                                                      In::smem(p.threads), st, a);
}
template <typename T, int V, bool SHIFT>
int norm_typed(const NormArgs& a, int sm_count, cudaStream_t st) {
    constexpr uint32_t kMost = V > 1 ? 32 : 8;                   // values a lane holds; single elements would take too many registers
    const uint64_t cols = a.cols + (SHIFT ? V - 1 : 0);
    cudaError_t e;
    NormPlan p = plan_lanes(cols, kMost);
    if constexpr (V > 1) {
        if (p.per == 16 || p.per == 32 || (!p.threads && (p = plan_block(cols, 32, 256)).threads)) {
            if (p.per == 16) e = run_norm<T, V, SHIFT, 16, 32, kWarpThreads, 6>(a, p, sm_count, st);
            else if (p.lanes) e = run_norm<T, V, SHIFT, 32, 32, kWarpThreads, 4>(a, p, sm_count, st);
            else e = run_norm<T, V, SHIFT, 32, 0, 256, 2>(a, p, sm_count, st);
            SK_OP_CUDA(e);
            return SK_OK;
        }
    }
    if (p.lanes == 8) e = run_norm<T, V, SHIFT, 8, 8, kWarpThreads, 8>(a, p, sm_count, st);
    else if (p.lanes) e = run_norm<T, V, SHIFT, 8, 32, kWarpThreads, 8>(a, p, sm_count, st);
    else if ((p = plan_block(cols, 16, 256)).threads) e = run_norm<T, V, SHIFT, 16, 0, 256, 3>(a, p, sm_count, st);
    else if ((p = plan_block(cols, 16, 1024)).threads) e = run_norm<T, V, SHIFT, 16, 0, 1024, 1>(a, p, sm_count, st);
    else e = launch_rows<k_norm_long<T>, 0>(dim3(norm_blocks(a.rows, p, sm_count, 2048)), kLongThreads, 0, st, a);
    SK_OP_CUDA(e);
    return SK_OK;
}

// Few rows: dw and db come from extra blocks of the one launch, which saves partial rows, the second kernel, and some 3 us of the host's time.
// Up to 256 rows always (16 x 768 bf16 2.8 us against 6.4); where rows lie on 16-byte boundaries and have at most 16 KB, up to 1024:
// 512 x 768 bf16 3.9 us against 6.8, 1024 x 4096 10.4 and 18.7, fp32 512 x 768 5.4 and 5.7, 1024 x 4096 14.6 and 13.8; but 1024 x 8192 32.1 and 24.6,
// 2048 x 768 16.6 and 8.8.
// (8184 columns: with up to seven values before a row that a block's threads still hold; the kernel for longer rows has no extra blocks.)
constexpr uint64_t kSlabRows = 256, kSlabCols = 8184, kSlabRowsWide = 1024, kSlabBytesWide = 16384;
bool always_slabs(uint64_t rows, uint64_t cols) { return rows <= kSlabRows && cols <= kSlabCols; }
// The plan decides how many partial rows there are, so the workspace's size needs it too.
// wide16: 16-bit rows by 16-byte accesses, of which a lane holds three before warps share a row (16384 x 768 bf16: 17.5 us, 21.2 with
// two warps a row; fp32 rows, as many bytes in flight, are at the memory's rate either way).
NormPlan plan_backward(uint64_t cols, bool wide16) {
    NormPlan p = plan_lanes(cols, 16);
    if (!p.threads && wide16 && cols <= 768) p = {32, kWarpThreads, 24};
    if (!p.threads) p = plan_block(cols, 16, 512);
    return p;
}
uint32_t backward_blocks(uint64_t rows, const NormPlan& p, int sm_count) { return norm_blocks(rows, p, sm_count, p.per == 8 ? 768 : p.per == 24 ? 384 : 512); }
template <typename T, int V, bool SHIFT, int PER, int G, int MAXT, int BLOCKS>
cudaError_t run_backward(const NormBackwardArgs& a, const NormPlan& p, uint32_t blocks, cudaStream_t st) {
    using In = Rows<T, V, PER / V, 2, SHIFT>;
    return launch_rows<k_norm_backward<T, V, PER / V, G, MAXT, BLOCKS, SHIFT>, In::smem(MAXT)>(dim3(blocks), p.threads, In::smem(p.threads), st, a);
}
template <typename T, int V, bool SHIFT>
int norm_backward_typed(NormBackwardArgs a, int sm_count, cudaStream_t st) {
    constexpr bool kWide16 = V == 8, kWhole = V > 1 && !SHIFT;
    if ((a.dweight || a.dbias) && (always_slabs(a.rows, a.cols) || (kWhole && a.rows <= kSlabRowsWide && a.cols * sizeof(T) <= kSlabBytesWide))) {
        constexpr uint32_t kCols = Slab<SHIFT ? 1 : V>::kCols;
        a.slabs = (uint32_t)((a.cols + kCols - 1) / kCols);
        a.partial = nullptr;
    }
    const NormPlan p = plan_backward(a.cols + (SHIFT ? V - 1 : 0), kWide16);
    const uint32_t row_blocks = backward_blocks(a.rows, p, sm_count);
    auto run = [&](uint32_t blocks) {
        if constexpr (kWide16) {
            if (p.per == 24) return run_backward<T, V, SHIFT, 24, 32, kWarpThreads, 3>(a, p, blocks, st);
        }
        if (p.lanes == 8) return run_backward<T, V, SHIFT, 8, 8, kWarpThreads, 6>(a, p, blocks, st);
        if (p.lanes == 32 && p.per == 8) return run_backward<T, V, SHIFT, 8, 32, kWarpThreads, 6>(a, p, blocks, st);
        if (p.lanes == 32) return run_backward<T, V, SHIFT, 16, 32, kWarpThreads, 4>(a, p, blocks, st);
        if (p.threads) return run_backward<T, V, SHIFT, 16, 0, 512, 1>(a, p, blocks, st);
        return launch_rows<k_norm_backward_long<T>, 0>(dim3(blocks), kLongThreads, 0, st, a);
    };
    if (a.slabs && (!a.dx || a.dx == a.dy || a.dx == a.x)) {         // in place the extra blocks would read what the others write: they go first
        SK_OP_CUDA(run(a.slabs));
        if (!a.dx) return SK_OK;
        a.slabs = 0;
    }
    cudaError_t e = run(row_blocks + a.slabs);
    SK_OP_CUDA(e);
    if (a.partial) {
        e = launch_kernel(true, k_norm_sum, dim3((uint32_t)((2 * a.cols + 7) / 8)), 256, 0, st, a.partial, row_blocks, (uint32_t)a.cols, a.dweight, a.dbias,
                          a.dw_type);
        SK_OP_CUDA(e);
    }
    return SK_OK;
}

// How the rows of up to three matrices are accessed together: 2, whole 16-byte accesses; 1, 16-byte accesses that begin before the
// row (the matrices' rows lie alike to the boundary); 0, single elements.  The first and the last access of a row cost more where they are
// not whole, which short rows do not win back: 65536 x 221 bf16 took 34 us so and takes 24 us by elements (backward 37, 28), 16384 x 4097
// 83 and 184 (156, 409).
struct Placed { const void* p; uint64_t ld; };
int access_of(uint64_t cols, uint32_t size, Placed x, Placed y, Placed z) {
    const uint64_t v = 16 / size;
    bool whole = cols % v == 0, alike = true;
    for (const Placed& m : {x, y, z}) {
        if (!m.p) continue;
        whole = whole && m.ld % v == 0 && (uintptr_t)m.p % 16 == 0;
        alike = alike && m.ld % v == x.ld % v && (uintptr_t)m.p % 16 == (uintptr_t)x.p % 16;
    }
    return whole ? 2 : alike && cols > 256 ? 1 : 0;
}
template <typename T>
int norm_placed(const NormArgs& a, int sm_count, cudaStream_t st) {
    constexpr int kV = 16 / sizeof(T);
    const int access = access_of(a.cols, sizeof(T), {a.x, a.ld_x}, {a.y, a.ld_y}, {nullptr, 0});
    return access == 2 ? norm_typed<T, kV, false>(a, sm_count, st) : access == 1 ? norm_typed<T, kV, true>(a, sm_count, st) : norm_typed<T, 1, false>(a, sm_count, st);
}
template <typename T>
int norm_backward_placed(const NormBackwardArgs& a, int sm_count, cudaStream_t st) {
    constexpr int kV = 16 / sizeof(T);
    const int access = access_of(a.cols, sizeof(T), {a.x, a.ld_x}, {a.dy, a.ld_dy}, {a.dx, a.ld_dx});
    return access == 2   ? norm_backward_typed<T, kV, false>(a, sm_count, st)
           : access == 1 ? norm_backward_typed<T, kV, true>(a, sm_count, st)
                         : norm_backward_typed<T, 1, false>(a, sm_count, st);
}

}  // namespace

int launch_norm(const NormArgs& a, int sm_count, cudaStream_t st) {
    return a.type == SK_F32 ? norm_placed<float>(a, sm_count, st) : a.type == SK_BF16 ? norm_placed<__nv_bfloat16>(a, sm_count, st) : norm_placed<__half>(a, sm_count, st);
}

int launch_norm_backward(const NormBackwardArgs& a, int sm_count, cudaStream_t st) {
    return a.type == SK_F32    ? norm_backward_placed<float>(a, sm_count, st)
           : a.type == SK_BF16 ? norm_backward_placed<__nv_bfloat16>(a, sm_count, st)
                               : norm_backward_placed<__half>(a, sm_count, st);
}

uint64_t norm_backward_workspace(uint64_t rows, uint64_t cols, int sm_count) {
    if (always_slabs(rows, cols)) return 0;
    uint32_t most = 0;                           // the rows' alignment decides between the plans: room for any
    for (uint64_t extra : {0, 3, 7})
        for (bool wide16 : {false, true}) {
            const uint32_t blocks = backward_blocks(rows, plan_backward(cols + extra, wide16), sm_count);
            most = blocks > most ? blocks : most;
        }
    return (uint64_t)most * 2 * cols * sizeof(float);
}

}  // namespace sk
