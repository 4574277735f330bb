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
    struct Args { __half* out; uint64_t stride; uint32_t ld; };
    const Args& a;
    const GemmShape& g;
    __half* out;
    uint32_t row;
    bool mirror;
    __device__ GramEpi(const Args& a_, const GemmShape& g_, const TileAt& at, uint32_t row_, uint32_t, uint32_t)
        : a(a_), g(g_), out(a_.out + at.b * a_.stride), row(row_), mirror(at.m != at.n) {}
    __device__ void put(uint32_t col, float (&v)[32]) {
        if (row >= g.M) return;
        store_row32(out, SK_F16, (uint64_t)row * a.ld + col, v, 32, true);
        if (mirror) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col + i < g.N) out[(uint64_t)(col + i) * a.ld + row] = __float2half_rn(v[i]);
        }
    }
    __device__ void chunk(uint32_t col, float (&v)[32]) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= kUnscale;
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
    __device__ PolyEpi(const Args& a_, const GemmShape& g_, const TileAt& at, uint32_t row_, uint32_t c0, uint32_t half)
        : p(a_), e(a_.o, g_, at, row_, c0, half), gram(a_.gram + at.b * a_.o.stride) {}
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
    struct Args { __half *hi, *lo; void* out; uint64_t stride; uint64_t ld; int type; uint32_t vec; };
    const Args& a;
    const GemmShape& g;
    uint64_t at0;
    uint32_t row;
    __device__ ApplyEpi(const Args& a_, const GemmShape& g_, const TileAt& at, uint32_t row_, uint32_t, uint32_t)
        : a(a_), g(g_), at0(at.b * a_.stride + (uint64_t)row_ * a_.ld), row(row_) {}
    __device__ void chunk(uint32_t col, float (&v)[32]) {
        if (row >= g.M) return;
        if (a.out) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= kUnscale * kUnscale;
            store_row32(a.out, a.type, at0 + col, v, g.N - col, a.vec);
            return;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= kUnscale;
        store_row32(a.hi, SK_F16, at0 + col, v, 32, true);
        if (a.lo) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] -= __half2float(__float2half_rn(v[i]));
            store_row32(a.lo, SK_F16, at0 + col, v, 32, true);
        }
    }
    __device__ void end() {}
};

// ---- the normalised matrix ------------------------------------------------------------------------------------------
constexpr uint32_t kNormBlocks = 64;             // most partial sums of squares per matrix

// Sums of squares of U per block, in 64 bits (an update in fp32 may have squares beyond its range); updates the momentum.
__global__ void __launch_bounds__(256) k_ortho_square(const OrthoArgs a, double* partial) {
    __shared__ double s[8];
    chain_acquire();
    const uint32_t b = blockIdx.y, groups = ((uint32_t)a.cols + 7) / 8;
    const uint64_t total = a.rows * groups;
    double sum = 0;
    for (uint64_t q = (uint64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (uint64_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)q / groups, col = ((uint32_t)q - row * groups) * 8;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (col + i >= a.cols) break;
            float u = load_as(a.update, a.type, b * a.stride_update + row * a.ld_update + col + i);
            if (a.momentum) {
                float* m = a.momentum + b * a.stride_momentum + row * a.ld_momentum + col + i;
                const float next = a.beta * *m + u;
                *m = next;
                u = a.nesterov ? u + a.beta * next : next;
            }
            sum += (double)u * (double)u;
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) sum += s[i];
        partial[(uint64_t)b * kNormBlocks + blockIdx.x] = sum;
    }
}

__global__ void __launch_bounds__(256) k_ortho_scale(const OrthoArgs a, const double* partial, uint32_t blocks, __half* hi, __half* lo,
                                                     uint32_t ld, uint64_t stride) {
    __shared__ float s_factor;
    chain_acquire();
    const uint32_t b = blockIdx.y, groups = ((uint32_t)a.cols + 7) / 8;
    if (threadIdx.x == 0) {
        double sum = 0;
        for (uint32_t i = 0; i < blocks; ++i) sum += partial[(uint64_t)b * kNormBlocks + i];
        s_factor = (float)(1.0 / (sqrt(sum) + (double)a.eps));
    }
    __syncthreads();
    const float factor = s_factor;
    const uint64_t total = a.rows * groups;
    for (uint64_t q = (uint64_t)blockIdx.x * 256 + threadIdx.x; q < total; q += (uint64_t)gridDim.x * 256) {
        const uint32_t row = (uint32_t)q / groups, col = ((uint32_t)q - row * groups) * 8;
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) {
            if (col + i >= a.cols) break;
            float u = load_as(a.update, a.type, b * a.stride_update + row * a.ld_update + col + i);
            if (a.momentum) {
                const float m = a.momentum[b * a.stride_momentum + row * a.ld_momentum + col + i];
                u = a.nesterov ? u + a.beta * m : m;
            }
            const float x = u * factor * kScale;
            const __half h = __float2half_rn(x);
            const uint64_t at = b * stride + (uint64_t)row * ld + col + i;
            hi[at] = h;
            if (lo) lo[at] = __float2half_rn(x - __half2float(h));
        }
    }
}

struct OrthoLayout {
    uint32_t ld_x, ld_a, m;
    uint64_t x_elems, a_elems;                   // per matrix
    uint64_t off_partial, off_x[2], off_lo, off_a, off_p, total;
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
    // two 16-bit matrices for X in all but the last two steps
    auto split = [&](int step) { return step < a.steps - 2; };

    const uint64_t groups = a.rows * ((a.cols + 7) / 8);
    uint32_t blocks = (uint32_t)((groups + 255) / 256);
    uint32_t few = blocks < kNormBlocks ? blocks : kNormBlocks;
    SK_OP_CUDA(launch_kernel(true, k_ortho_square, dim3(few, batch), 256, 0, st, a, partial));
    const uint32_t most = (uint32_t)dev.sm_count * 8;
    SK_OP_CUDA(launch_kernel(true, k_ortho_scale, dim3(blocks < most ? blocks : most, batch), 256, 0, st, a, partial, few, x[0],
                             split(0) ? lo[0] : nullptr, l.ld_x, l.x_elems));

    GemmShape square{};
    square.M = square.N = m;
    square.batch = batch;
    square.symmetric = 1;
    square.status = dev.status;
    GemmShape apply = square;
    apply.symmetric = 0;
    apply.M = (uint32_t)a.rows;
    apply.N = (uint32_t)a.cols;
    const Operand oa{gram, m, m, l.ld_a, l.a_elems, batch, false}, op{poly, m, m, l.ld_a, l.a_elems, batch, false};
    const bool vec = (uintptr_t)a.out % 32 == 0 && a.ld_out * type_size(a.out_type) % 32 == 0 && a.stride_out * type_size(a.out_type) % 32 == 0;
    for (int s = 0; s < a.steps; ++s) {
        const int from = s & 1, to = from ^ 1;
        const Operand ox{x[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, tall};
        SK_OP_CUDA(launch_product<GramEpi>(true, ox, ox, nullptr, nullptr, square, {gram, l.a_elems, l.ld_a}, dev.sm_count, st));
        PolyEpi::Args pa{{poly, l.a_elems, l.ld_a}, gram, a.coefficient[0], a.coefficient[1], a.coefficient[2]};
        SK_OP_CUDA(launch_product<PolyEpi>(true, oa, oa, nullptr, nullptr, square, pa, dev.sm_count, st));
        ApplyEpi::Args ea{};
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
            ea.vec = vec;
        }
        // X stored with its columns contiguous is the K-major first factor of X P, and the MN-major second factor of P X
        const Operand xh{x[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall}, xl{lo[from], a.rows, a.cols, l.ld_x, l.x_elems, batch, !tall};
        const bool two = split(s);
        if (tall) SK_OP_CUDA(launch_product<ApplyEpi>(true, xh, op, two ? &xl : nullptr, two ? &op : nullptr, apply, ea, dev.sm_count, st));
        else SK_OP_CUDA(launch_product<ApplyEpi>(true, op, xh, two ? &op : nullptr, two ? &xl : nullptr, apply, ea, dev.sm_count, st));
    }
    return SK_OK;
}

}  // namespace sk
