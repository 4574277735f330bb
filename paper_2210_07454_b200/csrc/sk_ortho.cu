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
//
// No operand is transposed: for a tall matrix (rows > cols) the same kernels take X in the other major
// (A = X^T X, X <- X P).
#include "sk_gemm.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr float kScale = 4096.0f, kUnscale = 1.0f / 4096.0f;     // 2^12
constexpr uint32_t kPadCols = 32;                                // leading dimensions: whole 32-column chunks

// A = X X^T, tiles on and below the diagonal, mirrored
struct GramEpi {
    struct Args { __half* out; uint64_t stride; uint32_t ld; const float* factor; };
    const Args& a;
    const GemmGroup& g;
    __half* out;
    uint32_t row, row0;                          // the lane's, the warp's first
    uint32_t* stage;
    bool mirror;
    float scale = kUnscale;
    __device__ GramEpi(const Args& a_, const GemmGroup& g_, const TileAt& at, uint32_t row_, uint32_t, uint32_t, uint32_t* stage_)
        : a(a_), g(g_), out(a_.out + at.b * a_.stride), row(row_), row0(row_ - (threadIdx.x & 31)), stage(stage_), mirror(at.m != at.n) {
        if (a.factor) scale *= a.factor[at.b] * a.factor[at.b];
    }
    __device__ void put(uint32_t col, float (&v)[32]) {
        if (row0 >= g.M) return;
        const uint32_t rows = g.M - row0 < 32 ? g.M - row0 : 32;
        store_block32(out, SK_F16, a.ld, row0, rows, col, 32, v, 32, stage, kStageRow);
        if (!mirror) return;
        // the block transposed: a lane's values are a column of it; four lanes write a row of the mirror image
        const uint32_t lane = threadIdx.x & 31, c = lane & 3;
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 32; ++i) ((__half*)(stage + i * kStageRow))[lane] = __float2half_rn(v[i]);
        __syncwarp();
#pragma unroll
        for (uint32_t r = lane >> 2; r < 32; r += 8)
            if (col + r < g.N) *(uint4*)(out + (uint64_t)(col + r) * a.ld + row0 + 8 * c) = *(const uint4*)(stage + r * kStageRow + 4 * c);
    }
    __device__ void chunk(uint32_t col, float (&v)[32]) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= scale;
        put(col, v);
    }
    __device__ void end() {}
};

// P = a I + b A + c A^2, likewise
struct PolyEpi {
    struct Args { GramEpi::Args o; const __half* gram; float a, b, c; };
    const Args& p;
    GramEpi e;
    const __half* gram;
    __device__ PolyEpi(const Args& a_, const GemmGroup& g_, const TileAt& at, uint32_t row_, uint32_t c0, uint32_t half, uint32_t* stage_)
        : p(a_), e(a_.o, g_, at, row_, c0, half, stage_), gram(a_.gram + at.b * a_.o.stride) {}
    __device__ void chunk(uint32_t col, float (&v)[32]) {
        if (e.row < e.g.M) {
            uint32_t r[16];
            const __half* src = gram + (uint64_t)e.row * p.o.ld + col;
            load32b(src, r);
            load32b(src + 16, r + 8);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = __half22float2(*(const __half2*)&r[i]);
                v[2 * i] = p.b * f.x + p.c * kUnscale * v[2 * i];
                v[2 * i + 1] = p.b * f.y + p.c * kUnscale * v[2 * i + 1];
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i == e.row) v[i] += p.a * kScale;
        }
        e.put(col, v);
    }
    __device__ void end() {}
};

// X <- P X: one fp16 matrix, or two whose sum it is; the last step writes the result in the caller's type and layout
struct ApplyEpi {
    struct Args { __half *hi, *lo; void* out; uint64_t stride; uint64_t ld; int type; uint32_t align; const float* factor; };
    const Args& a;
    const GemmGroup& g;
    uint64_t first;
    uint32_t row0, rows;
    uint32_t* stage;
    float scale = kUnscale;
    __device__ ApplyEpi(const Args& a_, const GemmGroup& g_, const TileAt& at, uint32_t row_, uint32_t, uint32_t, uint32_t* stage_)
        : a(a_), g(g_), first(at.b * a_.stride), row0(row_ - (threadIdx.x & 31)), stage(stage_) {
        rows = row0 >= g.M ? 0 : g.M - row0 < 32 ? g.M - row0 : 32;
        if (a.factor) scale *= a.factor[at.b];
        if (a.out) scale *= kUnscale;
    }
    __device__ void chunk(uint32_t col, float (&v)[32]) {
        if (!rows) return;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= scale;
        if (a.out) {
            store_block32((uint16_t*)a.out + first, a.type, a.ld, row0, rows, col, g.N - col, v, a.align, stage, kStageRow);
            return;
        }
        store_block32(a.hi + first, SK_F16, a.ld, row0, rows, col, 32, v, 32, stage, kStageRow);
        if (a.lo) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
            store_block32(a.lo + first, SK_F16, a.ld, row0, rows, col, 32, v, 32, stage, kStageRow);
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

struct SquareArgs {
    OrthoArgs a;
    double* partial;                             // [batch][kNormBlocks]
    float* factor;                               // [batch]: X = factor * (the matrix that is stored)
    uint32_t blocks, vec_u, vec_m;
    __half *hi, *lo;
    uint32_t ld;
    uint64_t stride;
    uint32_t exact;                              // U is the 16-bit update itself: stored exactly, times a power of two
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
    __shared__ float s_scale;
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
        const double scale = (double)kScale / (sqrt(sum) + (double)a.eps);
        int e = 0;
        double rest = 1.0;
        if (s.exact && scale > 1e-30 && scale < 1e30) {
            rest = frexp(scale, &e) * 2.0;                           // scale = rest * 2^(e-1), rest in [1, 2)
            s_scale = (float)ldexp(1.0, e - 1);
        } else {
            s_scale = (float)scale;
        }
        if (blockIdx.x == 0) s.factor[b] = (float)rest;
    }
    __syncthreads();
    const float scale = s_scale;
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
            const float x = u[2 * i] * scale, y = u[2 * i + 1] * scale;
            const __half2 p = __floats2half2_rn(x, y);
            const float2 f = __half22float2(p);
            h[i] = *(const uint32_t*)&p;
            l[i] = pack16(x - f.x, y - f.y, false);
        }
        const uint64_t at = b * s.stride + (uint64_t)row * s.ld + col;   // ld is a multiple of 32: whole groups fit
        *(uint4*)(s.hi + at) = make_uint4(h[0], h[1], h[2], h[3]);
        if (s.lo) *(uint4*)(s.lo + at) = make_uint4(l[0], l[1], l[2], l[3]);
    }
}

struct OrthoLayout {
    uint32_t ld_x, ld_a, m;
    uint64_t x_elems, a_elems;                   // per matrix
    uint64_t off_partial, off_factor, off_x[2], off_lo, off_a, off_p, total;
};
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
    l.off_x[0] = take(a.batch * l.x_elems * 2);
    l.off_x[1] = take(a.batch * l.x_elems * 2);
    l.off_lo = take(2 * round_up(a.batch * l.x_elems * 2, 256));
    l.off_a = take(a.batch * l.a_elems * 2);
    l.off_p = take(a.batch * l.a_elems * 2);
    l.total = at;
    return l;
}

}  // namespace

uint64_t orthogonalize_workspace(const OrthoArgs& a) { return layout_of(a).total; }

int launch_orthogonalize(const OrthoArgs& a, const OpDevice& dev, cudaStream_t st) {
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
    const bool exact = a.type != SK_F32 && !a.momentum;
    auto split = [&](int step) { return step < a.steps - 2 && !(step == 0 && exact); };

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
    SK_OP_CUDA(launch_kernel(true, k_ortho_square, dim3(sq.blocks, batch), 256, 0, st, sq));
    SK_OP_CUDA(launch_kernel(true, k_ortho_scale, dim3(sq.blocks, batch), 256, 0, st, sq));

    GemmGroup square{};
    square.M = square.N = m;
    square.batch = batch;
    square.symmetric = 1;
    GemmGroup apply = square;
    apply.symmetric = 0;
    apply.M = (uint32_t)a.rows;
    apply.N = (uint32_t)a.cols;
    const Operand oa{gram, m, m, l.ld_a, l.a_elems, batch, false}, op{poly, m, m, l.ld_a, l.a_elems, batch, false};
    const uint32_t align_rows = row_alignment(a.out, a.ld_out, a.out_type), align_batch = row_alignment(a.out, a.stride_out, a.out_type);
    const uint32_t align = batch > 1 && align_batch < align_rows ? align_batch : align_rows;
    for (int s = 0; s < a.steps; ++s) {
        const int from = s & 1, to = from ^ 1;
        const Operand ox{x[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, tall};
        SK_OP_CUDA(launch_product<GramEpi>(true, ox, ox, nullptr, nullptr, square, dev.status, {gram, l.a_elems, l.ld_a, s == 0 ? sq.factor : nullptr}, dev.sm_count, st));
        PolyEpi::Args pa{{poly, l.a_elems, l.ld_a, nullptr}, gram, a.coefficient[0], a.coefficient[1], a.coefficient[2]};
        SK_OP_CUDA(launch_product<PolyEpi>(true, oa, oa, nullptr, nullptr, square, dev.status, pa, dev.sm_count, st));
        ApplyEpi::Args ea{};
        ea.factor = s == 0 ? sq.factor : nullptr;
        if (s + 1 < a.steps) {
            ea.hi = x[to];
            ea.lo = split(s + 1) ? lo[to] : nullptr;
            ea.stride = l.x_elems;
            ea.ld = l.ld_x;
        } else {
            ea.out = a.out;
            ea.stride = a.stride_out;
            ea.ld = a.ld_out;
            ea.type = a.out_type;
            ea.align = align;
        }
        // X stored with its columns contiguous is the K-major first factor of X P, and the MN-major second factor of P X
        const Operand xh{x[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall}, xl{lo[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall};
        const bool two = split(s);
        if (tall) SK_OP_CUDA(launch_product<ApplyEpi>(true, xh, op, two ? &xl : nullptr, two ? &op : nullptr, apply, dev.status, ea, dev.sm_count, st));
        else SK_OP_CUDA(launch_product<ApplyEpi>(true, op, xh, two ? &op : nullptr, two ? &xl : nullptr, apply, dev.status, ea, dev.sm_count, st));
    }
    return SK_OK;
}

}  // namespace sk
