// Declarations shared by the operators' files (layer norm, linear cross entropy, orthogonalised updates).  Not installed.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "../../include/sketched_amsgrad.h"

namespace sk {

// records a message for sk_last_error() and returns `code` (defined with the handle's entry points)
int set_error(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

#define SK_OP_CUDA(...)                                                                                        \
    do {                                                                                                       \
        cudaError_t err__ = (__VA_ARGS__);                                                                     \
        if (err__ != cudaSuccess)                                                                              \
            return sk::set_error(SK_ECUDA, "%s:%d: %s", __func__, __LINE__, cudaGetErrorString(err__));        \
    } while (0)

// Where a wait inside a kernel that runs out is counted, and after how long it does.  Thirty seconds: a tile over K = 2^31, the longest
// wait that any call can mean, takes up to eighteen; of the largest matrices in practice, below one.
constexpr uint32_t kWaitLimitMs = 30000;
struct Waits {
    uint32_t* status;
    uint32_t limit_ms;
};
// What the operators know about the current device; resolved once per device.
struct OpDevice {
    int sm_count = 0;
    uint32_t* status = nullptr;      // count of waits that ran out (a static of the library)
    Waits waits() const { return {status, kWaitLimitMs}; }
};
int op_device(OpDevice* out);        // SK_OK or an error with its message

inline uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }
inline bool type_ok(int t) { return t == SK_F32 || t == SK_BF16 || t == SK_F16; }
inline uint32_t type_size(int t) { return t == SK_F32 ? 4 : 2; }

// ---- element types on the device ------------------------------------------------------------------------------------
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// element i of an array whose type is known at run time only
__device__ __forceinline__ float load_as(const void* p, int type, uint64_t i) {
    if (type == SK_F32) return ((const float*)p)[i];
    if (type == SK_BF16) return __bfloat162float(((const __nv_bfloat16*)p)[i]);
    return __half2float(((const __half*)p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int type, uint64_t i, float v) {
    if (type == SK_F32) ((float*)p)[i] = v;
    else if (type == SK_BF16) ((__nv_bfloat16*)p)[i] = __float2bfloat16_rn(v);
    else ((__half*)p)[i] = __float2half_rn(v);
}
// two values rounded to 16 bits each, the first in the low half
__device__ __forceinline__ uint32_t pack16(float a, float b, bool bf16) {
    if (bf16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *(const uint32_t*)&h;
    }
    const __half2 h = __floats2half2_rn(a, b);
    return *(const uint32_t*)&h;
}
__device__ __forceinline__ void store32b(void* p, const uint32_t* r) {       // 32 bytes at a 32-byte boundary
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void load32b(const void* p, uint32_t* r) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),
                 "=r"(r[6]), "=r"(r[7]) : "l"(p) : "memory");
}

// ---- pairs of 32-bit values ---------------------------------------------------------------------------------------------
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float x, float y) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float2 parts(F2 a) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ F2 operator+(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 operator*(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
    F2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// What is known of an output's rows: the largest of 16, 4 and 2 bytes that every row starts on
inline uint32_t row_alignment(const void* p, uint64_t ld, int type) {
    const uint64_t bits = (uintptr_t)p | ld * type_size(type);
    return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

__device__ __forceinline__ void store_shared16(uint32_t at, uint4 q) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w) : "memory");
}
__device__ __forceinline__ void store_shared2(uint32_t at, uint32_t low) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((uint16_t)low) : "memory"); }
__device__ __forceinline__ uint4 load_shared16(uint32_t at) {
    uint4 q;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(at) : "memory");
    return q;
}
// A warp's staging area: 32 rows of 128 bytes, 16-byte chunks swizzled.  The key differs within any eight neighbouring rows, and within
// the four pairs of rows (2 i, 2 i + 1) + 0, 8, 16, 24 that a reader of columns takes.
__device__ __forceinline__ uint32_t staged(uint32_t stage, uint32_t r, uint32_t chunk) {
    return stage + r * 128 + ((chunk ^ ((r ^ ((r >> 3) << 1)) & 7)) << 4);
}

// A warp's rows of an output tile, 32 columns at a time: the lane's row (row0 + lane; rows of the 32 exist), v = its columns
// col .. col + 31 (those below limit exist; col is a multiple of 32).  The values pass through 4 KB of the warp's shared memory (stage, its shared
// address), so that neighbouring lanes write neighbouring addresses: whole 128-byte lines, two calls of 16-bit values
// together (pair; last: no second one follows).  All lanes take part.
__device__ __forceinline__ void store_tile32(void* out, int type, uint64_t ld, uint64_t row0, uint32_t rows, uint32_t col, uint32_t limit,
                                             const float (&v)[32], uint32_t align, uint32_t stage, bool pair, bool last) {
    const bool wide = type == SK_F32;            // 32 columns are whole lines already
    const uint32_t lane = threadIdx.x & 31, second = pair && !wide ? (col >> 5) & 1 : 0;
    if (!second) __syncwarp();                   // what was staged before has been read
    if (wide) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            store_shared16(staged(stage, lane, i), make_uint4(__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]),
                                                              __float_as_uint(v[4 * i + 3])));
    } else {
        uint32_t h[16];
        if (type == SK_BF16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = pack16(v[2 * i], v[2 * i + 1], true);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) h[i] = pack16(v[2 * i], v[2 * i + 1], false);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) store_shared16(staged(stage, lane, 4 * second + i), make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]));
        if (pair && !second && !last) return;    // the other half of the lines follows
    }
    __syncwarp();
    const uint32_t size = wide ? 4 : 2, first = col - 32 * second;
    const uint32_t bytes = min(limit - first, 32 * (second + 1)) * size;         // of every row (a whole one may have more than 32 bits can say)
    uint8_t* o = (uint8_t*)out + (row0 * ld + first) * size;
    const uint64_t step = ld * size;
    if (align >= 16 && bytes % 16 == 0) {        // eight lanes a row, all eight loads before the stores
        const uint32_t c = lane & 7, r0 = lane >> 3;
        if (c * 16 < bytes) {
            uint4 q[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) q[i] = load_shared16(staged(stage, r0 + 4 * i, c));
            uint8_t* p = o + r0 * step + c * 16;
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i)
                if (r0 + 4 * i < rows) *(uint4*)(p + 4 * i * step) = q[i];
        }
    } else if (align >= 4) {                     // a row after the other, eight at a time
        if (lane * 4 < bytes) {
            const bool whole = lane * 4 + 4 <= bytes;
            for (uint32_t r = 0; r < rows; r += 8) {
                uint32_t w[8];
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(staged(stage, r + i, lane >> 2) + (lane & 3) * 4) : "memory");
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (r + i < rows) {
                        if (whole) *(uint32_t*)(o + (r + i) * step + lane * 4) = w[i];
                        else *(uint16_t*)(o + (r + i) * step + lane * 4) = (uint16_t)w[i];
                    }
            }
        }
    } else {
        for (uint32_t r = 0; r < rows; r += 8) {
#pragma unroll
            for (uint32_t c = lane; c < 64; c += 32) {
                if (c * 2 >= bytes) break;
                uint16_t w[8];
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i) asm volatile("ld.shared.b16 %0, [%1];" : "=h"(w[i]) : "r"(staged(stage, r + i, c >> 3) + (c & 7) * 2) : "memory");
#pragma unroll
                for (uint32_t i = 0; i < 8; ++i)
                    if (r + i < rows) *(uint16_t*)(o + (r + i) * step + c * 2) = w[i];
            }
        }
    }
}

// ---- launchers ---------------------------------------------------------------------------------------------------------
struct NormArgs {
    const void *x, *weight, *bias;
    void* y;
    float *mean, *rstd;
    uint64_t rows, cols, ld_x, ld_y;
    int type, w_type;
    float eps;
};
struct NormBackwardArgs {
    const void *dy, *x, *weight;
    const float *mean, *rstd;
    void *dx, *dweight, *dbias;
    float* partial;                  // [blocks][2][cols], or null where extra blocks form the sums over the rows
    uint32_t slabs;                  // such blocks, set by the launcher
    uint64_t rows, cols, ld_dy, ld_x, ld_dx;
    int type, w_type, dw_type;
};
int launch_norm(const NormArgs& a, int sm_count, cudaStream_t st);
int launch_norm_backward(const NormBackwardArgs& a, int sm_count, cudaStream_t st);
uint64_t norm_backward_workspace(uint64_t rows, uint64_t cols, int sm_count);

// hidden (tokens x width) times vocabulary matrix (vocab x width), both of one 16-bit type
struct HeadArgs {
    const void *hidden, *weight;
    const int64_t* targets;
    uint64_t tokens, vocab, width, ld_hidden, ld_weight;
    int type;
    float *loss, *lse;               // forward: out; backward: lse in
    const float* dloss;              // backward only, from here on
    void *dhidden, *dweight;         // either may be null
    uint64_t ld_dhidden, ld_dweight;
    int dhidden_type, dweight_type;
    void* workspace;
};
int launch_head(const HeadArgs& a, const OpDevice& dev, cudaStream_t st);
int launch_head_backward(const HeadArgs& a, const OpDevice& dev, cudaStream_t st);
uint64_t head_workspace(const HeadArgs& a);
uint64_t head_backward_workspace(const HeadArgs& a);

struct OrthoArgs {
    const void* update;              // batch x rows x cols
    float* momentum;                 // same shape, or null
    void* out;
    uint64_t batch, rows, cols;
    uint64_t ld_update, stride_update, ld_momentum, stride_momentum, ld_out, stride_out;
    int type, out_type;
    int nesterov, steps;
    float beta, eps;
    float coefficient[3];
    void* workspace;
};
// Products grouped by expert: rows offsets[g] .. offsets[g + 1] of x with matrix g (out x width), all of one 16-bit type
constexpr uint32_t kMaxGroups = 2048;
struct GroupedArgs {
    const void *x, *weight;
    const int64_t* offsets;          // groups + 1
    uint64_t rows, groups, width, out;
    uint64_t ld_x, ld_weight, stride_weight;
    int type, fill;                  // fill: rows of no group become zero in y or dx
    void* y;                         // forward: rows x out
    uint64_t ld_y;
    const void* dy;                  // backward only, from here on
    void *dx, *dweight;              // either may be null
    uint64_t ld_dy, ld_dx, ld_dweight, stride_dweight;
    int dweight_type;
    void* workspace;
    uint32_t withhold_ms;            // not zero in tests, see sk_test_operators_wait
    Waits waits(const OpDevice& dev) const { return {dev.status, withhold_ms ? withhold_ms : kWaitLimitMs}; }
};
int launch_grouped(GroupedArgs a, const OpDevice& dev, cudaStream_t st);
int launch_grouped_backward(GroupedArgs a, const OpDevice& dev, cudaStream_t st);
uint64_t grouped_workspace(const GroupedArgs& a, bool backward);

struct SortArgs {
    const void* experts;             // n int64, or int32
    uint64_t n;
    uint32_t groups;
    int wide;                        // 64-bit
    int64_t *order, *places, *offsets;       // either of the first two may be null
    uint32_t* workspace;
};
int launch_sort(const SortArgs& a, int sm_count, cudaStream_t st);
uint64_t sort_workspace(uint64_t n, uint32_t groups, int sm_count);

struct DropoutArgs {
    const void *x, *residual;        // residual may be null
    void* y;
    uint64_t rows, cols, ld_x, ld_residual, ld_y;
    int type;
    uint64_t seed;
    const uint64_t* seed_at;         // on the device, or null
    uint32_t below;                  // a 16-bit number below this drops the value
    float scale;
};
int launch_dropout(const DropoutArgs& a, int sm_count, cudaStream_t st);

struct PolicyArgs {
    const float *nll, *old_nll, *advantages, *reference;
    const int64_t *targets, *offsets;        // either may be null
    uint64_t tokens, sequences;
    int advantage_of_sequences, average_sequences;
    double log_high, log_low;        // of the ratio's bounds
    float border_high, border_low;   // the same, rounded
    float high, low, kl;
    float *result, *norm;            // forward: out
    const float* dloss;              // backward: may be null
    float* dnll;
    float4* workspace;
};
int launch_policy(PolicyArgs a, cudaStream_t st);
int launch_policy_backward(const PolicyArgs& a, cudaStream_t st);
uint64_t policy_workspace(uint64_t tokens, uint64_t sequences);

// withhold_ms: not zero in tests, see sk_test_operators_wait
int launch_orthogonalize(const OrthoArgs& a, const OpDevice& dev, uint32_t withhold_ms, cudaStream_t st);
uint64_t orthogonalize_workspace(const OrthoArgs& a);

}  // namespace sk
