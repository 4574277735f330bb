// Layer norm over the last axis, forward and backward.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), y = (x - mu) r w + b
//   h = (x - mu) r, g = dy w:  dx = r (g - mean(g) - h mean(g h)),  dw = sum over rows of dy h,  db = sum over rows of dy
//
// Bound by memory: forward reads x and writes y once, backward reads x and dy and writes dx once.  A group of threads
// (a warp for short rows, up to a block of 512 for long ones) holds a row in registers, so the second and third looks
// at it (variance around the computed mean; dx after the two means) cost no memory traffic.  Groups walk over the rows
// of a fixed grid; the weights stay in registers, and in the backward pass so do the sums of dw and db, of
// which every block writes one partial row that a second, column-parallel kernel adds up in a fixed order: no atomics,
// the same bits every time.  All statistics and sums are 32-bit.
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

template <typename T, int V>
struct alignas(sizeof(T) * V) Pack { T v[V]; };

template <int TPR>
__device__ __forceinline__ float group_sum(float v, float* scratch) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        __syncthreads();                                  // the previous sum has been read by everybody
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) v += scratch[i];
    }
    return v;
}
template <int TPR>
__device__ __forceinline__ float2 group_sum2(float2 v, float2* scratch) {
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
    }
    if constexpr (TPR > 32) {
        constexpr int kWarps = TPR / 32;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
        __syncthreads();
        v = make_float2(0, 0);
#pragma unroll
        for (int i = 0; i < kWarps; ++i) { v.x += scratch[i].x; v.y += scratch[i].y; }
    }
    return v;
}

// TPR threads per row (32, or the whole block), NV accesses of V elements per thread; TPR * NV * V >= cols.
template <typename T, int V, int NV, int TPR>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) k_norm(const NormArgs a) {
    __shared__ float scratch[TPR / 32];
    constexpr int kGroups = TPR < 128 ? 128 / TPR : 1;
    const uint32_t t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const uint32_t cols = (uint32_t)a.cols;
    chain_acquire();
    float w[NV * V], b[NV * V];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = (i * TPR + t) * V + j;
            w[i * V + j] = c < cols && a.weight ? load_as(a.weight, a.w_type, c) : 1.0f;
            b[i * V + j] = c < cols && a.bias ? load_as(a.bias, a.w_type, c) : 0.0f;
        }
    const float inv = 1.0f / (float)cols;
    for (uint64_t row = (uint64_t)blockIdx.x * kGroups + group; row < a.rows; row += (uint64_t)gridDim.x * kGroups) {
        const T* x = (const T*)a.x + row * a.ld_x;
        Pack<T, V> p[NV];
        float sum = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (i * TPR + t) * V;
            if (c < cols) p[i] = *(const Pack<T, V>*)(x + c);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) p[i].v[j] = from_float<T>(0.0f);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) sum += to_float(p[i].v[j]);
        const float mean = group_sum<TPR>(sum, scratch) * inv;
        float sq = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_float(p[i].v[j]) - mean;
                if ((i * TPR + t) * V < cols) sq += d * d;
            }
        const float rstd = rsqrtf(group_sum<TPR>(sq, scratch) * inv + a.eps);
        T* y = (T*)a.y + row * a.ld_y;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (i * TPR + t) * V;
            Pack<T, V> o;
#pragma unroll
            for (int j = 0; j < V; ++j) o.v[j] = from_float<T>((to_float(p[i].v[j]) - mean) * rstd * w[i * V + j] + b[i * V + j]);
            if (c < cols) *(Pack<T, V>*)(y + c) = o;
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// Rows longer than the register kernels hold: the block looks at the row three times, the later looks from L2.
constexpr int kLongThreads = 512;
template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_long(const NormArgs a) {
    __shared__ float scratch[kLongThreads / 32];
    chain_acquire();
    const float inv = 1.0f / (float)a.cols;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = (const T*)a.x + row * a.ld_x;
        T* y = (T*)a.y + row * a.ld_y;
        float sum = 0, sq = 0;
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) sum += to_float(x[c]);
        const float mean = group_sum<kLongThreads>(sum, scratch) * inv;
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float d = to_float(x[c]) - mean;
            sq += d * d;
        }
        const float rstd = rsqrtf(group_sum<kLongThreads>(sq, scratch) * inv + a.eps);
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

template <typename T, int V, int NV, int TPR>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) k_norm_backward(const NormBackwardArgs a) {
    constexpr int kGroups = TPR < 128 ? 128 / TPR : 1;
    constexpr int kPer = NV * V;
    __shared__ float2 scratch[TPR / 32];
    __shared__ float gather[kGroups > 1 ? kGroups : 1][kGroups > 1 ? TPR * V : 1];
    const uint32_t t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const uint32_t cols = (uint32_t)a.cols;
    chain_acquire();
    float w[kPer], dw[kPer], db[kPer];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const uint32_t c = (i * TPR + t) * V + j;
            w[i * V + j] = c < cols && a.weight ? load_as(a.weight, a.w_type, c) : 1.0f;
            dw[i * V + j] = db[i * V + j] = 0.0f;
        }
    const float inv = 1.0f / (float)cols;
    for (uint64_t row = (uint64_t)blockIdx.x * kGroups + group; row < a.rows; row += (uint64_t)gridDim.x * kGroups) {
        const T* x = (const T*)a.x + row * a.ld_x;
        const T* dy = (const T*)a.dy + row * a.ld_dy;
        Pack<T, V> px[NV], pd[NV];
        const float mean = a.mean[row], rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (i * TPR + t) * V;
            if (c < cols) {
                px[i] = *(const Pack<T, V>*)(x + c);
                pd[i] = *(const Pack<T, V>*)(dy + c);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { px[i].v[j] = from_float<T>(mean); pd[i].v[j] = from_float<T>(0.0f); }
            }
        }
        float2 s = make_float2(0, 0);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int q = i * V + j;
                const float h = (to_float(px[i].v[j]) - mean) * rstd, d = to_float(pd[i].v[j]), g = d * w[q];
                s.x += g;
                s.y += g * h;
                dw[q] += d * h;
                db[q] += d;
            }
        if (!a.dx) continue;
        s = group_sum2<TPR>(s, scratch);
        const float m1 = s.x * inv, m2 = s.y * inv;
        T* dx = (T*)a.dx + row * a.ld_dx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t c = (i * TPR + t) * V;
            Pack<T, V> o;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float h = (to_float(px[i].v[j]) - mean) * rstd, g = to_float(pd[i].v[j]) * w[i * V + j];
                o.v[j] = from_float<T>(rstd * (g - m1 - h * m2));
            }
            if (c < cols) *(Pack<T, V>*)(dx + c) = o;
        }
    }
    if (!a.partial) return;
    float* out = a.partial + (uint64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if constexpr (kGroups > 1) {
                __syncthreads();
#pragma unroll
                for (int j = 0; j < V; ++j) gather[group][t * V + j] = which ? db[i * V + j] : dw[i * V + j];
                __syncthreads();
                for (uint32_t q = threadIdx.x; q < TPR * V; q += blockDim.x) {
                    const uint32_t c = i * TPR * V + q;
                    float v = 0;
#pragma unroll
                    for (int k = 0; k < kGroups; ++k) v += gather[k][q];
                    if (c < cols) out[(uint64_t)which * cols + c] = v;
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const uint32_t c = (i * TPR + t) * V + j;
                    if (c < cols) out[(uint64_t)which * cols + c] = which ? db[i * V + j] : dw[i * V + j];
                }
            }
        }
}

// Long rows, backward: the sums of a block are kept in its partial row in memory (own columns only, so no races).
template <typename T>
__global__ void __launch_bounds__(kLongThreads) k_norm_backward_long(const NormBackwardArgs a) {
    __shared__ float2 scratch[kLongThreads / 32];
    chain_acquire();
    const float inv = 1.0f / (float)a.cols;
    float* part = a.partial ? a.partial + (uint64_t)blockIdx.x * 2 * a.cols : nullptr;
    bool fresh = true;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x, fresh = false) {
        const T* x = (const T*)a.x + row * a.ld_x;
        const T* dy = (const T*)a.dy + row * a.ld_dy;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float2 s = make_float2(0, 0);
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float h = (to_float(x[c]) - mean) * rstd, d = to_float(dy[c]);
            const float g = a.weight ? d * load_as(a.weight, a.w_type, c) : d;
            s.x += g;
            s.y += g * h;
            if (part) {
                part[c] = (fresh ? 0.0f : part[c]) + d * h;
                part[a.cols + c] = (fresh ? 0.0f : part[a.cols + c]) + d;
            }
        }
        s = group_sum2<kLongThreads>(s, scratch);
        if (!a.dx) continue;
        T* dx = (T*)a.dx + row * a.ld_dx;
        for (uint64_t c = threadIdx.x; c < a.cols; c += kLongThreads) {
            const float h = (to_float(x[c]) - mean) * rstd;
            const float g = to_float(dy[c]) * (a.weight ? load_as(a.weight, a.w_type, c) : 1.0f);
            dx[c] = from_float<T>(rstd * (g - s.x * inv - h * (s.y * inv)));
        }
    }
}

// Adds the blocks' partial rows, in block order within each of the eight rows of threads, these in order.
__global__ void __launch_bounds__(256) k_norm_sum(const float* partial, uint32_t blocks, uint32_t cols, void* dweight, void* dbias, int type) {
    __shared__ float s[8][33];
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const uint64_t c = (uint64_t)blockIdx.x * 32 + x;            // over both sums: 2 * cols columns
    chain_acquire();
    float v = 0;
    if (c < 2ull * cols)
        for (uint32_t b = y; b < blocks; b += 8) v += partial[(uint64_t)b * 2 * cols + c];
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && c < 2ull * cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) v += s[i][x];
        void* out = c < cols ? dweight : dbias;
        if (out) store_as(out, type, c < cols ? c : c - cols, v);
    }
}

// threads per row and values per thread by the row's length; cap = values a thread may hold
struct NormPlan { uint32_t tpr, per; };
NormPlan plan_norm(uint64_t cols) {
    if (cols <= 256) return {32, 8};
    if (cols <= 1024) return {32, 32};
    if (cols <= 4096) return {128, 32};
    if (cols <= 16384) return {512, 32};
    return {0, 0};
}
NormPlan plan_backward(uint64_t cols) {
    if (cols <= 256) return {32, 8};
    if (cols <= 1024) return {128, 8};
    if (cols <= 2048) return {128, 16};
    if (cols <= 8192) return {512, 16};
    return {0, 0};
}
uint32_t backward_blocks(uint64_t rows, uint64_t cols, int sm_count) {
    const NormPlan p = plan_backward(cols);
    const uint64_t groups = p.tpr == 32 ? 4 : 1;
    const uint64_t want = (rows + groups - 1) / groups, most = (uint64_t)sm_count * (p.tpr == 512 || !p.tpr ? 2 : 4);
    return (uint32_t)(want < most ? (want ? want : 1) : most);
}

template <typename T, int V>
int norm_typed(const NormArgs& a, int sm_count, cudaStream_t st) {
    const NormPlan p = plan_norm(a.cols);
    const uint64_t groups = p.tpr == 32 ? 4 : 1;
    const uint64_t want = (a.rows + groups - 1) / groups, most = (uint64_t)sm_count * (p.tpr == 512 || !p.tpr ? 4 : 12);
    const dim3 grid((uint32_t)(want < most ? want : most));
    cudaError_t e;
    if (p.tpr == 32 && p.per == 8) e = launch_kernel(true, k_norm<T, V, 8 / V, 32>, grid, 128, 0, st, a);
    else if (p.tpr == 32) e = launch_kernel(true, k_norm<T, V, 32 / V, 32>, grid, 128, 0, st, a);
    else if (p.tpr == 128) e = launch_kernel(true, k_norm<T, V, 32 / V, 128>, grid, 128, 0, st, a);
    else if (p.tpr == 512) e = launch_kernel(true, k_norm<T, V, 32 / V, 512>, grid, 512, 0, st, a);
    else e = launch_kernel(true, k_norm_long<T>, grid, kLongThreads, 0, st, a);
    SK_OP_CUDA(e);
    return SK_OK;
}
template <typename T, int V>
int norm_backward_typed(const NormBackwardArgs& a, int sm_count, cudaStream_t st) {
    const NormPlan p = plan_backward(a.cols);
    const uint32_t blocks = backward_blocks(a.rows, a.cols, sm_count);
    const dim3 grid(blocks);
    cudaError_t e;
    if (p.tpr == 32) e = launch_kernel(true, k_norm_backward<T, V, 8 / V, 32>, grid, 128, 0, st, a);
    else if (p.tpr == 128 && p.per == 8) e = launch_kernel(true, k_norm_backward<T, V, 8 / V, 128>, grid, 128, 0, st, a);
    else if (p.tpr == 128) e = launch_kernel(true, k_norm_backward<T, V, 16 / V, 128>, grid, 128, 0, st, a);
    else if (p.tpr == 512) e = launch_kernel(true, k_norm_backward<T, V, 16 / V, 512>, grid, 512, 0, st, a);
    else e = launch_kernel(true, k_norm_backward_long<T>, grid, kLongThreads, 0, st, a);
    SK_OP_CUDA(e);
    if (a.partial) {
        e = launch_kernel(true, k_norm_sum, dim3((uint32_t)((2 * a.cols + 31) / 32)), 256, 0, st, a.partial, blocks, (uint32_t)a.cols,
                          a.dweight, a.dbias, a.dw_type);
        SK_OP_CUDA(e);
    }
    return SK_OK;
}
bool aligned16(const void* p, uint64_t ld, uint32_t size) { return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0; }

}  // namespace

int launch_norm(const NormArgs& a, int sm_count, cudaStream_t st) {
    const uint32_t size = type_size(a.type);
    // 128-bit accesses where every row of x and y starts and ends on a 16-byte boundary, single elements elsewhere
    const bool vec = a.cols * size % 16 == 0 && aligned16(a.x, a.ld_x, size) && aligned16(a.y, a.ld_y, size);
    if (a.type == SK_F32) return vec ? norm_typed<float, 4>(a, sm_count, st) : norm_typed<float, 1>(a, sm_count, st);
    if (a.type == SK_BF16) return vec ? norm_typed<__nv_bfloat16, 8>(a, sm_count, st) : norm_typed<__nv_bfloat16, 1>(a, sm_count, st);
    return vec ? norm_typed<__half, 8>(a, sm_count, st) : norm_typed<__half, 1>(a, sm_count, st);
}

int launch_norm_backward(const NormBackwardArgs& a, int sm_count, cudaStream_t st) {
    const uint32_t size = type_size(a.type);
    const bool vec = a.cols * size % 16 == 0 && aligned16(a.x, a.ld_x, size) && aligned16(a.dy, a.ld_dy, size) &&
                     (!a.dx || aligned16(a.dx, a.ld_dx, size));
    if (a.type == SK_F32) return vec ? norm_backward_typed<float, 4>(a, sm_count, st) : norm_backward_typed<float, 1>(a, sm_count, st);
    if (a.type == SK_BF16)
        return vec ? norm_backward_typed<__nv_bfloat16, 8>(a, sm_count, st) : norm_backward_typed<__nv_bfloat16, 1>(a, sm_count, st);
    return vec ? norm_backward_typed<__half, 8>(a, sm_count, st) : norm_backward_typed<__half, 1>(a, sm_count, st);
}

uint64_t norm_backward_workspace(uint64_t rows, uint64_t cols, int sm_count) {
    return (uint64_t)backward_blocks(rows, cols, sm_count) * 2 * cols * sizeof(float);
}

}  // namespace sk
