// Dropout from a counter: whether value i stays is a function of the seed and i, so that nothing is stored for the backward pass.
//
//   K = stream(seed, 1), u = stream(K, i div 4 + 1) (splitmix64, the library's own generator), f = bits 16 (i mod 4) .. + 15 of u
//   y_i = residual_i + (f >= below ? x_i 65536 / (65536 - below) : 0),  below = p 65536, rounded
//
// One draw serves four values, so that the generator (some twenty integer instructions) stays behind the memory traffic: with 32 bits a value it would take
// about as long as reading and writing 16-bit values does.  What is lost is the resolution of p, 2^-16; the factor is that of the rounded p, so
// that the mean is kept exactly.  Bound by HBM: every value is read once and written once. 32768 x 4096 bf16 with a residual (805 MB) 116 us, 6.9 TB/s; rows twice as far apart at the
// same rate; rows off the 16-byte boundary 2.4 TB/s (bf16) and 4.9 (fp32): a draw's values to a thread, by single accesses.
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ULL;
__device__ __forceinline__ uint64_t mix(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ULL;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBULL;
    return z ^ (z >> 31);
}
__device__ __forceinline__ uint64_t key_of(const DropoutArgs& a) { return mix((a.seed_at ? *a.seed_at : a.seed) + kGamma); }
// four draws of 16 bits: for the values 4 q .. 4 q + 3
__device__ __forceinline__ uint64_t draws(uint64_t key, uint64_t q) { return mix(key + (q + 1) * kGamma); }
__device__ __forceinline__ uint32_t field(uint64_t u, uint32_t i) { return (uint32_t)(u >> (16 * i)) & 0xFFFFu; }

__device__ __forceinline__ float one(float x, float r, bool stays, float scale) { return stays ? fmaf(x, scale, r) : r; }

// 16 bytes of a type
template <typename T> struct Vec { static constexpr uint32_t kN = 16 / sizeof(T); };

template <typename T, bool RES>
__device__ __forceinline__ void apply(const DropoutArgs& a, uint64_t key, uint64_t first, const uint4& x, const uint4& r, uint4& y) {
    constexpr uint32_t N = Vec<T>::kN;
    const T *px = (const T*)&x, *pr = (const T*)&r;
    T* py = (T*)&y;
#pragma unroll
    for (uint32_t q = 0; q < N / 4; ++q) {
        const uint64_t u = draws(key, first / 4 + q);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            py[4 * q + i] = from_float<T>(one(to_float(px[4 * q + i]), RES ? to_float(pr[4 * q + i]) : 0.0f, field(u, i) >= a.below, a.scale));
    }
}

// Values in whole 16-byte accesses: one run of them, or (ROWS) rows of a whole number of accesses, any number of accesses apart. kEach of them to a thread on their way at once.
constexpr uint32_t kDropThreads = 256, kEach = 4;
template <typename T, bool RES, bool ROWS>
__global__ void __launch_bounds__(kDropThreads) k_dropout_flat(const __grid_constant__ DropoutArgs a, uint64_t n) {
    constexpr uint32_t N = Vec<T>::kN;
    chain_acquire();
    const uint64_t key = key_of(a), vectors = n / N, v0 = (uint64_t)blockIdx.x * (kDropThreads * kEach) + threadIdx.x;
    const uint4 *x = (const uint4*)a.x, *res = (const uint4*)a.residual;
    uint4* y = (uint4*)a.y;
    uint4 vx[kEach], vr[kEach];
    uint64_t row[ROWS ? kEach : 1], col[ROWS ? kEach : 1];
    auto at = [&](uint32_t e, uint64_t v, uint64_t ld) { return ROWS ? row[ROWS ? e : 0] * (ld / N) + col[ROWS ? e : 0] : v; };
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
        const uint64_t v = v0 + e * kDropThreads;
        if (v < vectors) {
            if constexpr (ROWS) {
                const uint64_t each = a.cols / N;
                row[e] = vectors >> 32 ? v / each : (uint32_t)v / (uint32_t)each;
                col[e] = v - row[e] * each;
            }
            vx[e] = x[at(e, v, a.ld_x)];
            if (RES) vr[e] = res[at(e, v, a.ld_residual)];
        }
    }
#pragma unroll
    for (uint32_t e = 0; e < kEach; ++e) {
        const uint64_t v = v0 + e * kDropThreads;
        if (v < vectors) {
            uint4 out;
            apply<T, RES>(a, key, v * N, vx[e], vr[e], out);
            y[at(e, v, a.ld_y)] = out;
        }
    }
    if (ROWS) return;
    const uint64_t i = vectors * N + threadIdx.x;                // what is left of a last vector
    if (blockIdx.x == 0 && i < n) {
        const float r = RES ? to_float(((const T*)a.residual)[i]) : 0.0f;
        ((T*)a.y)[i] = from_float<T>(one(to_float(((const T*)a.x)[i]), r, field(draws(key, i / 4), i % 4) >= a.below, a.scale));
    }
}

// Rows any distance apart, any alignment: a thread takes the four values of a draw.
template <typename T, bool RES>
__global__ void __launch_bounds__(kDropThreads) k_dropout_rows(const __grid_constant__ DropoutArgs a, uint64_t n) {
    chain_acquire();
    const uint64_t key = key_of(a), step = (uint64_t)gridDim.x * kDropThreads;
    const T *x = (const T*)a.x, *res = (const T*)a.residual;
    T* y = (T*)a.y;
    for (uint64_t q = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x; q * 4 < n; q += step) {
        const uint64_t u = draws(key, q);
        uint64_t row = q * 4 / a.cols, col = q * 4 - row * a.cols;
        float vx[4], vr[4];
        uint64_t at[4];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            if (q * 4 + i < n) {
                vx[i] = to_float(x[row * a.ld_x + col]);
                vr[i] = RES ? to_float(res[row * a.ld_residual + col]) : 0.0f;
                at[i] = row * a.ld_y + col;
            }
            if (++col == a.cols) { col = 0; ++row; }
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (q * 4 + i < n) y[at[i]] = from_float<T>(one(vx[i], vr[i], field(u, i) >= a.below, a.scale));
    }
}

template <typename T, bool RES>
int launch(const DropoutArgs& a, int sm_count, cudaStream_t st) {
    const uint64_t n = a.rows * a.cols;
    const bool dense = a.rows == 1 || (a.ld_x == a.cols && a.ld_y == a.cols && (!RES || a.ld_residual == a.cols));
    const bool aligned = ((uintptr_t)a.x | (uintptr_t)a.y | (RES ? (uintptr_t)a.residual : 0)) % 16 == 0;
    const bool whole = (a.cols | a.ld_x | a.ld_y | (RES ? a.ld_residual : 0)) % Vec<T>::kN == 0;
    const uint64_t vectors = n / Vec<T>::kN, vectors_each = kDropThreads * kEach, blocks = (vectors + vectors_each - 1) / vectors_each;
    if (aligned && (dense || whole) && blocks < (1ull << 31)) {
        auto kernel = dense ? k_dropout_flat<T, RES, false> : k_dropout_flat<T, RES, true>;
        SK_OP_CUDA(launch_kernel(true, kernel, dim3(blocks ? (uint32_t)blocks : 1), kDropThreads, 0, st, a, n));
        return SK_OK;
    }
    const uint64_t want = (n + 4 * kDropThreads - 1) / (4 * kDropThreads), most = (uint64_t)sm_count * 32;
    SK_OP_CUDA(launch_kernel(true, k_dropout_rows<T, RES>, dim3((uint32_t)(want < most ? want : most)), kDropThreads, 0, st, a, n));
    return SK_OK;
}

}  // namespace

int launch_dropout(const DropoutArgs& a, int sm_count, cudaStream_t st) {
    if (a.type == SK_F32) return a.residual ? launch<float, true>(a, sm_count, st) : launch<float, false>(a, sm_count, st);
    if (a.type == SK_BF16) return a.residual ? launch<__nv_bfloat16, true>(a, sm_count, st) : launch<__nv_bfloat16, false>(a, sm_count, st);
    return a.residual ? launch<__half, true>(a, sm_count, st) : launch<__half, false>(a, sm_count, st);
}

}  // namespace sk
