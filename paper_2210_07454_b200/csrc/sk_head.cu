// Softmax cross entropy of a linear head over a large vocabulary, without keeping the logits.
//
//   z = hidden W^T;  lse_i = log sum_v exp z_iv;  loss_i = lse_i - z_i,target(i)
//   G_iv = dloss_i (exp(z_iv - lse_i) - [v = target(i)]);  dhidden = G W,  dW = G^T hidden
//
// Forward: one product whose epilogue keeps, per row and half tile, the maximum and the sum of exponentials relative to
// it (32 bits), and the target's logit; a small kernel joins the pieces.  The logits never leave the SM.
// Backward: the vocabulary is taken in pieces.  A product recomputes a piece's logits and its epilogue writes the piece of G (in the
// inputs' 16-bit type, the operand type of the two products that follow); then dW's rows of the piece and the piece's share
// of dhidden, which is added up in 32 bits over the pieces.  Bound by the tensor cores (2 T V D flops forward, 4 backward plus 2
// for the recomputation); for few tokens by reading W.
//
// For few tokens the rounding of G shows in the gradients: one entry of a row, the target's, is much larger than the others, and its error is not
// averaged away (1 x 3941 x 1024 bf16: 2.7e-3 for an output whose own rounding is 1.7e-3).  Up to kPairTokens tokens G is therefore the sum of two 16-bit
// matrices, one below the other, and so are the hidden states twice: dW sums over twice the rows, and the rows of dhidden are added up in
// pairs.  The rows fit one tile either way, and W is read no more often (8 x 50257 x 768 64.3 -> 66.4 us, 64 tokens 68 -> 73).  For more tokens that would double the products; there the rounding of
// G adds some 35 % to the error of the output's own (41 % at most, were every entry rounded by itself).
//
// A row whose target is negative takes no part: loss 0, gradient 0.  A target >= vocab gives a loss of NaN and no gradient.
#include "sk_gemm.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float exp2_fast(float x) {          // 2^x, 2 ulp
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// per (half tile, row): maximum of the logits and the sum of exp(z - maximum)
template <bool PARTS>
struct StatsEpi {
    static constexpr int kWarps = 8, kWords = kStageWords;
    static constexpr bool kParts = PARTS;
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) { return true; }
    struct Args { float2* part; float* at_target; const int64_t* targets; };
    const Args& a;
    const TileJob& t;
    uint32_t row, slot;
    int64_t target;
    float top = -INFINITY, sum = 0;
    __device__ StatsEpi(const Args& a_, const TileJob& t_, uint32_t row_, uint32_t half, uint32_t)
        : a(a_), t(t_), row(row_), slot(t_.n * 2 + half) { target = row < t.M ? a.targets[row] : -1; }
    __device__ void chunk(uint32_t col, float (&v)[32], bool) {
        const uint32_t valid = t.N - col;
        const uint64_t d = (uint64_t)(target - (int64_t)col);
        if (d < 32 && d < valid) {
            float z = v[0];
#pragma unroll
            for (int i = 1; i < 32; ++i) z = d == (uint64_t)i ? v[i] : z;
            a.at_target[row] = z;
        }
        if (valid < 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = (uint32_t)i < valid ? v[i] : -INFINITY;
        }
        float m = v[0];
#pragma unroll
        for (int i = 1; i < 32; ++i) m = fmaxf(m, v[i]);
        if (m > top) {
            sum *= exp2_fast((top - m) * kLog2e);
            top = m;
        }
        // the difference first: it is exact near the maximum, whatever the logits' size
        const float off = top == -INFINITY ? 0.0f : top;
        const F2 minus = f2(-off, -off), log2e = f2(kLog2e, kLog2e);
        F2 s = f2(0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 e = parts((f2(v[2 * i], v[2 * i + 1]) + minus) * log2e);
            s = s + f2(exp2_fast(e.x), exp2_fast(e.y));
        }
        const float2 both = parts(s);
        sum += both.x + both.y;
    }
    __device__ void end() {
        if (row < t.M) a.part[(uint64_t)slot * t.M + row] = make_float2(top, sum);
    }
};

// Joins the pieces: eight rows to a block, 64 threads a row; first the maximum over the pieces, then the sum relative to it.
constexpr int kJoinThreads = 512;
__global__ void __launch_bounds__(kJoinThreads) k_head_join(const float2* part, const float* at_target, const int64_t* targets, uint32_t tokens,
                                                            uint64_t vocab, uint32_t slots, float* loss, float* lse) {
    __shared__ float s[kJoinThreads / 32][8];
    chain_acquire();
    const uint32_t x = threadIdx.x & 7, y = threadIdx.x >> 3, warp = threadIdx.x >> 5, row = blockIdx.x * 8 + x;
    const bool live = row < tokens;
    const float2* p = part + row;
    float top = -INFINITY;
    if (live) {
#pragma unroll 4
        for (uint32_t q = y; q < slots; q += kJoinThreads / 8) top = fmaxf(top, p[(uint64_t)q * tokens].x);
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
    if ((threadIdx.x & 31) < 8) s[warp][x] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kJoinThreads / 32; ++i) top = fmaxf(top, s[i][x]);
    float sum = 0;
    if (live) {
#pragma unroll 4
        for (uint32_t q = y; q < slots; q += kJoinThreads / 8) {
            const float2 f = p[(uint64_t)q * tokens];
            if (f.y != 0.0f) sum += f.y * (f.x == top ? 1.0f : expf(f.x - top));      // 0: nothing above minus infinity
        }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 8);
    sum += __shfl_xor_sync(0xffffffffu, sum, 16);
    __syncthreads();
    if ((threadIdx.x & 31) < 8) s[warp][x] = sum;
    __syncthreads();
    if (y == 0 && live) {
        sum = 0;
#pragma unroll
        for (int i = 0; i < kJoinThreads / 32; ++i) sum += s[i][x];
        const float log_sum = logf(sum);
        const int64_t t = targets[row];
        if (lse) lse[row] = top + log_sum;
        // the difference of two logits first: of a confident token it is small, and exact
        if (loss) loss[row] = t < 0 ? 0.0f : t >= (int64_t)vocab ? NAN : (top - at_target[row]) + log_sum;
    }
}

// G's piece.  PAIR: as the sum of two matrices, the second's lines through an area of their own.
template <bool PAIR>
struct GradEpi {
    static constexpr int kWarps = 8, kWords = (PAIR ? 2 : 1) * kStageWords;
    static constexpr bool kParts = false;
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) { return true; }
    struct Args {
        uint16_t *out, *low;                     // low: the second matrix
        uint64_t ld;
        const float *lse, *dloss, *factor;
        const int64_t* targets;
        uint64_t vocab;
        uint32_t first;
    };
    const Args& a;
    const TileJob& t;
    uint32_t row0, rows;
    uint32_t stage;
    float off = 0, scale = 0;
    int64_t target = -1;
    __device__ GradEpi(const Args& a_, const TileJob& t_, uint32_t row, uint32_t, uint32_t stage_)
        : a(a_), t(t_), row0(row - (threadIdx.x & 31)), stage(stage_) {
        rows = row0 >= t.M ? 0 : t.M - row0 < 32 ? t.M - row0 : 32;
        if (row < t.M) {
            const int64_t v = a.targets[row];
            if (v >= 0 && v < (int64_t)a.vocab) {
                target = v - (int64_t)a.first;
                scale = a.dloss[row] * *a.factor;
                off = a.lse[row];
            }
        }
    }
    __device__ void chunk(uint32_t col, float (&v)[32], bool last) {
        if (!rows) return;
        const uint64_t d = (uint64_t)(target - (int64_t)col);
        if (scale != 0.0f) {
            const F2 minus = f2(-off, -off), log2e = f2(kLog2e, kLog2e), by = f2(scale, scale);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 e = parts((f2(v[2 * i], v[2 * i + 1]) + minus) * log2e);
                v[2 * i] = exp2_fast(e.x);
                v[2 * i + 1] = exp2_fast(e.y);
            }
            if (d < 32) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] -= d == (uint64_t)i ? 1.0f : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 g = parts(f2(v[2 * i], v[2 * i + 1]) * by);
                v[2 * i] = g.x;
                v[2 * i + 1] = g.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.0f;
        }
        __syncwarp();
        store_tile32(a.out, t.bf16 ? SK_BF16 : SK_F16, a.ld, row0, rows, col, (uint32_t)a.ld, v, 16, stage, true, last);
        if constexpr (PAIR) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] -= t.bf16 ? __bfloat162float(__float2bfloat16_rn(v[i])) : __half2float(__float2half_rn(v[i]));
            store_tile32(a.low, t.bf16 ? SK_BF16 : SK_F16, a.ld, row0, rows, col, (uint32_t)a.ld, v, 16, stage + kStageWords * 4, true, last);
        }
    }
    __device__ void end() {}
};

// One of two products, by the group: rows of dW, or a share of dhidden.  Shares of more than one piece or slice are added up in 32
// bits, a slice of K in a matrix of its own (`sum`, one after the other), and joined by k_head_sum.
struct OutEpi {
    static constexpr int kWarps = 8, kWords = kStageWords;
    static constexpr bool kParts = false;
    template <class Plan> __device__ bool begin(const Plan&, uint32_t) { return true; }
    struct One { void* out; float* sum; uint64_t ld, sum_stride; int type; uint32_t align, add; };
    struct Args { One o[2]; const float* factor; };
    const One& a;
    const TileJob& t;
    float* sum;
    uint32_t row0, rows;
    uint32_t stage;
    float scale;
    __device__ OutEpi(const Args& a_, const TileJob& t_, uint32_t row, uint32_t, uint32_t stage_)
        : a(a_.o[t_.kind]), t(t_), sum(a.sum ? a.sum + t_.slice * a.sum_stride : nullptr), row0(row - (threadIdx.x & 31)), stage(stage_),
          scale(1.0f / *a_.factor) {
        rows = row0 >= t.M ? 0 : t.M - row0 < 32 ? t.M - row0 : 32;
    }
    __device__ void chunk(uint32_t col, float (&v)[32], bool last) {
        if (!rows) return;
        if (!sum) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= scale;
            store_tile32(a.out, a.type, a.ld, row0, rows, col, t.N, v, a.align, stage, true, last);
            return;
        }
        const uint32_t lane = threadIdx.x & 31;
        if (a.add && lane < rows) {
            const float* s = sum + (uint64_t)(row0 + lane) * a.ld + col;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                uint32_t r[8];
                load32b(s + 8 * q, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * q + i] += __uint_as_float(r[i]);
            }
        }
        __syncwarp();
        store_tile32(sum, SK_F32, a.ld, row0, rows, col, (uint32_t)a.ld, v, 16, stage, false, last);
    }
    __device__ void end() {}
};

// dhidden from its shares, slices in order, and with `second` the other half of the sum as far behind each
__global__ void __launch_bounds__(256) k_head_sum(const float* sum, uint32_t slices, uint64_t stride, uint64_t second, uint64_t ld_sum, uint64_t rows,
                                                  uint32_t cols, const float* factor, void* out, uint64_t ld, int type) {
    chain_acquire();
    const float scale = 1.0f / *factor;
    const uint32_t groups = (cols + 3) / 4;
    const uint64_t total = rows * groups;
    for (uint64_t q = blockIdx.x * 256ull + threadIdx.x; q < total; q += gridDim.x * 256ull) {
        const uint64_t row = q / groups;
        const uint32_t col = (uint32_t)(q - row * groups) * 4;
        const float* p = sum + row * ld_sum + col;               // ld_sum is a multiple of 32
        float4 v = *(const float4*)p, u = second ? *(const float4*)(p + second) : make_float4(0, 0, 0, 0);
#pragma unroll 4
        for (uint32_t s = 1; s < slices; ++s) {                  // several slices' loads on their way at once
            const float4 w = *(const float4*)(p + s * stride);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
            if (second) {
                const float4 x = *(const float4*)(p + second + s * stride);
                u.x += x.x; u.y += x.y; u.z += x.z; u.w += x.w;
            }
        }
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;          // small against the first: added last
        const float f[4] = {v.x * scale, v.y * scale, v.z * scale, v.w * scale};
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (col + i < cols) store_as(out, type, row * ld + col + i, f[i]);
    }
}

// Rows copied to a leading dimension that TMA can address, up to two matrices in one launch; with targets, the rows that
// take no part become zero.  The backward pass always takes the hidden states through this: in dW a token without a target is multiplied
// by zeros, and whatever its row holds (padding may hold infinities or NaN) must not survive that.
struct PackArgs {
    struct One { const uint16_t* src; uint16_t* dst; uint64_t ld, rows, distinct; const int64_t* targets; uint32_t ld_dst; } m[2];    // rows: `distinct` ones over again
    uint64_t vocab;
    uint32_t cols, first_blocks;                 // blocks of the first matrix
    uint32_t copy_blocks;                        // of all matrices
    const float* dloss;                          // with a factor: one block more
    float* factor;
    float most;                                  // of |dloss| times the factor
};
// What G is multiplied by before it is rounded; the products divide by it again.  It brings the largest |dloss| to a power of two: 1, or 2^14 for fp16, so
// that small probabilities stay above fp16's smallest values.  A target's entry of G is dloss (p - 1), about -dloss, and in a mean it is the same for
// all tokens: this way its rounding is nothing (-1 is exact), where it would be the same error in all of them, up to 2^-8 of the gradients in bf16.
__device__ void head_factor(const float* dloss, const int64_t* targets, uint64_t tokens, uint64_t vocab, float most, float* factor) {
    __shared__ float s[8];
    float m = 0;
    for (uint64_t i = threadIdx.x; i < tokens; i += 256)
        if (targets[i] >= 0 && targets[i] < (int64_t)vocab) m = fmaxf(m, fabsf(dloss[i]));
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 8; ++i) m = fmaxf(m, s[i]);
        *factor = m > 0 && isfinite(m) ? fminf(fmaxf(most / m, 0x1p-100f), 0x1p100f) : 1.0f;
    }
}
// A thread copies eight neighbours: eight loads on their way at once whatever the alignment, one 16-byte store.
__global__ void __launch_bounds__(256) k_head_pack(const __grid_constant__ PackArgs a) {
    chain_acquire();
    if (blockIdx.x >= a.copy_blocks) {
        head_factor(a.dloss, a.m[0].targets, a.m[0].distinct, a.vocab, a.most, a.factor);
        return;
    }
    const uint32_t which = blockIdx.x >= a.first_blocks;
    const PackArgs::One& m = a.m[which];
    const uint32_t groups = m.ld_dst / 8, block = which ? blockIdx.x - a.first_blocks : blockIdx.x;
    const uint64_t total = m.rows * groups, step = (uint64_t)(which ? a.copy_blocks - a.first_blocks : a.first_blocks) * 256;
    const bool vec = (uintptr_t)m.src % 16 == 0 && m.ld % 8 == 0, half = (uintptr_t)m.src % 8 == 0 && m.ld % 4 == 0;
    for (uint64_t q = block * 256ull + threadIdx.x; q < total; q += step) {
        const uint64_t r = q / groups;
        const uint32_t c = (uint32_t)(q - r * groups) * 8;
        const uint64_t from = r < m.distinct ? r : r - m.distinct;
        const bool live = !m.targets || (m.targets[from] >= 0 && m.targets[from] < (int64_t)a.vocab);
        const uint16_t* s = m.src + from * m.ld + c;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (live && c + 8 <= a.cols && vec) {
            v = *(const uint4*)s;
        } else if (live && c + 8 <= a.cols && half) {
            const uint2 x = *(const uint2*)s, y = *(const uint2*)(s + 4);
            v = make_uint4(x.x, x.y, y.x, y.y);
        } else if (live) {
            uint32_t e[8];
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) e[i] = c + i < a.cols ? s[i] : 0;
            v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
        }
        *(uint4*)(m.dst + r * m.ld_dst + c) = v;
    }
}

// Stages of K to an accumulation of the logits in the forward pass.  The loss of a few tokens is the difference of two logits, and nothing averages
// what they are off: up to 16 tokens take 256 values (1 x 2424 fp16: error of the loss 2.5e-5 in one accumulation, 8e-7 so; 8 x 50257 x 768 takes
// 25.9 us for 24.2, with 128 values 27.5).  Over more tokens 1024 values keep it below 7e-7 (in one accumulation 1e-6 to 2.3e-6 at widths of 1500 to
// 3800; 4096 x 32000 x 4096 takes 832 us for 797, 2048 x 50257 x 2048 some 2 % more).
uint32_t logit_part(uint64_t tokens) { return tokens <= 16 ? 4 : 16; }

bool addressable(const void* p, uint64_t ld) { return (uintptr_t)p % 16 == 0 && ld % 8 == 0; }

struct HeadLayout {
    bool pack_h, pack_w;
    uint64_t ld_h, ld_w, off_h, off_w, off_part, off_target, off_factor, off_g, ld_g, off_sum, ld_sum, sum_stride, piece, total;
    uint32_t slices;                             // of the vocabulary's pieces in the product that gives dhidden
    uint64_t rows;                               // of G: one or two for a token
    bool wide;                                   // tiles of the two gradient products
};
// columns of the vocabulary per piece: G's piece is to stay below this size
constexpr uint64_t kPieceBytes = 512ull << 20;
constexpr uint64_t kPairTokens = 64;             // G a pair: both halves' rows fit a tile of 128

// The product that gives dhidden has few tiles and a long K (a piece of the vocabulary), the one that gives dW many short ones; they run
// in one launch.  K is split where one tile of the first would last longer than about half of an even share of all the work.
// (n: columns of a whole piece.)
constexpr uint32_t kPlanSms = 148;               // the plan, and with it the workspace, is made for a B200
uint32_t slices_of(uint64_t tokens, uint64_t n, uint64_t width, bool wide) {
    if (n < tokens) return 1;
    const uint64_t tile = wide ? 256 : 128, units = kPlanSms / (wide ? 2 : 1);
    const uint64_t rows = (tokens + tile - 1) / tile, cols = (width + 255) / 256, vocab = (n + tile - 1) / tile;
    const uint64_t k0 = (n + kGemmK - 1) / kGemmK, k1 = (tokens + kGemmK - 1) / kGemmK;
    const uint64_t work = rows * cols * (k0 + kTileCost) + vocab * cols * (k1 + kTileCost);
    uint64_t s = 2 * k0 * units / work;
    if (s > k0 / 8) s = k0 / 8;                  // a slice is worth its epilogue
    if (s > 32) s = 32;
    if (s < 2) return 1;
    const uint64_t each = (k0 + s - 1) / s;
    return (uint32_t)((k0 + each - 1) / each);   // as many as the first piece really has: every one is written there
}

HeadLayout layout_of(const HeadArgs& a, bool backward) {
    HeadLayout l{};
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) { const uint64_t r = at; at += round_up(bytes, 256); return r; };
    l.pack_h = backward || !addressable(a.hidden, a.ld_hidden);
    l.pack_w = !addressable(a.weight, a.ld_weight);
    // Rows of whole 128-byte lines, as a tile's rows of 64 values are fetched: for the hidden states and G, which every tile reads (1000 x 32003 x 1000
    // backward: 186 us with rows that are multiples of 16 bytes, 181 with G in whole lines, 173 with both).  The weights' copy costs
    // more than that would save.
    l.ld_h = round_up(a.width, 64);
    l.ld_w = round_up(a.width, 8);
    l.rows = backward && a.tokens <= kPairTokens ? 2 * a.tokens : a.tokens;
    if (l.pack_h) l.off_h = take(l.rows * l.ld_h * 2);
    if (l.pack_w) l.off_w = take(a.vocab * l.ld_w * 2);
    if (!backward) {
        l.off_part = take(2 * ((a.vocab + 127) / 128) * a.tokens * sizeof(float2));
        l.off_target = take(a.tokens * 4);
    } else {
        l.off_factor = take(4);
        uint64_t pieces = (l.rows * a.vocab * 2 + kPieceBytes - 1) / kPieceBytes;
        l.piece = round_up((a.vocab + pieces - 1) / pieces, 256);
        l.ld_g = l.piece < round_up(a.vocab, 64) ? l.piece : round_up(a.vocab, 64);
        l.off_g = take(l.rows * l.ld_g * 2);
        l.ld_sum = round_up(a.width, 32);
        l.sum_stride = l.rows * l.ld_sum;
        l.wide = a.tokens > 128;
        l.slices = slices_of(a.tokens, l.piece < a.vocab ? l.piece : a.vocab, a.width, l.wide);
        if (a.dhidden && (l.piece < a.vocab || l.slices > 1 || l.rows > a.tokens)) l.off_sum = take(l.slices * l.sum_stride * 4);
    }
    l.total = at;
    return l;
}

// the operands as TMA can address them: packed copies where the caller's are not
int pack_operands(const HeadArgs& a, bool backward, const HeadLayout& l, const OpDevice& dev, const void** h, const void** w, uint64_t* ld_h, uint64_t* ld_w,
                  float* factor, cudaStream_t st) {
    uint8_t* ws = (uint8_t*)a.workspace;
    *h = a.hidden; *w = a.weight; *ld_h = a.ld_hidden; *ld_w = a.ld_weight;
    PackArgs p{};
    uint32_t n = 0, blocks[2] = {0, 0};
    auto add = [&](const void* src, uint64_t ld, uint64_t off, uint64_t ld_dst, uint64_t rows, uint64_t distinct, const int64_t* targets) {
        p.m[n] = {(const uint16_t*)src, (uint16_t*)(ws + off), ld, rows, distinct, targets, (uint32_t)ld_dst};
        const uint64_t want = (rows * (ld_dst / 8) + 255) / 256, most = (uint64_t)dev.sm_count * 16;
        blocks[n++] = (uint32_t)(want < most ? want : most);
    };
    if (l.pack_h) {
        add(a.hidden, a.ld_hidden, l.off_h, l.ld_h, l.rows, a.tokens, backward ? a.targets : nullptr);
        *h = ws + l.off_h; *ld_h = l.ld_h;
    }
    if (l.pack_w) {
        add(a.weight, a.ld_weight, l.off_w, l.ld_w, a.vocab, a.vocab, nullptr);
        *w = ws + l.off_w; *ld_w = l.ld_w;
    }
    if (!n) return SK_OK;
    p.vocab = a.vocab;
    p.cols = (uint32_t)a.width;
    p.first_blocks = blocks[0];
    p.copy_blocks = blocks[0] + blocks[1];
    p.dloss = a.dloss;
    p.factor = factor;
    p.most = a.type == SK_F16 ? 0x1p14f : 1.0f;
    SK_OP_CUDA(launch_kernel(true, k_head_pack, dim3(p.copy_blocks + (factor ? 1 : 0)), 256, 0, st, p));
    return SK_OK;
}

}  // namespace

uint64_t head_workspace(const HeadArgs& a) { return layout_of(a, false).total; }
uint64_t head_backward_workspace(const HeadArgs& a) { return layout_of(a, true).total; }

int launch_head(const HeadArgs& a, const OpDevice& dev, cudaStream_t st) {
    const HeadLayout l = layout_of(a, false);
    uint8_t* ws = (uint8_t*)a.workspace;
    const void *h, *w;
    uint64_t ld_h, ld_w;
    int rc = pack_operands(a, false, l, dev, &h, &w, &ld_h, &ld_w, nullptr, st);
    if (rc) return rc;
    GemmGroup g{};
    g.M = (uint32_t)a.tokens;
    g.N = (uint32_t)a.vocab;
    g.bf16 = a.type == SK_BF16;
    float2* part = (float2*)(ws + l.off_part);
    float* at_target = (float*)(ws + l.off_target);
    const Operand oh{h, a.tokens, a.width, ld_h, 0, 1, false}, ow{w, a.vocab, a.width, ld_w, 0, 1, false};
    const uint64_t stages = (a.width + kGemmK - 1) / kGemmK;
    const bool wide = wide_tiles(g.M, g.N, stages, dev.sm_count);
    g.part = logit_part(a.tokens);
    if (stages <= g.part) {
        const StatsEpi<false>::Args ea{part, at_target, a.targets};
        auto launch = wide ? launch_products<2, 256, StatsEpi<false>> : launch_products<1, 128, StatsEpi<false>>;
        SK_OP_CUDA(launch(true, oh, ow, g, 1, nullptr, nullptr, nullptr, dev.waits(), ea, dev.sm_count, st));
    } else {
        const StatsEpi<true>::Args ea{part, at_target, a.targets};
        auto launch = wide ? launch_products<2, 256, StatsEpi<true>> : launch_products<1, 128, StatsEpi<true>>;
        SK_OP_CUDA(launch(true, oh, ow, g, 1, nullptr, nullptr, nullptr, dev.waits(), ea, dev.sm_count, st));
    }
    const uint32_t tile = wide ? 256 : 128, slots = 2 * ((g.N + tile - 1) / tile);
    SK_OP_CUDA(launch_kernel(true, k_head_join, dim3((g.M + 7) / 8), kJoinThreads, 0, st, (const float2*)part, (const float*)at_target, a.targets, g.M,
                             a.vocab, slots, a.loss, a.lse));
    return SK_OK;
}

int launch_head_backward(const HeadArgs& a, const OpDevice& dev, cudaStream_t st) {
    const HeadLayout l = layout_of(a, true);
    uint8_t* ws = (uint8_t*)a.workspace;
    const void *h, *w;
    uint64_t ld_h, ld_w;
    float* factor = (float*)(ws + l.off_factor);
    int rc = pack_operands(a, true, l, dev, &h, &w, &ld_h, &ld_w, factor, st);
    if (rc) return rc;
    const uint32_t tokens = (uint32_t)a.tokens, width = (uint32_t)a.width;
    uint16_t* gbuf = (uint16_t*)(ws + l.off_g);
    float* sum = l.off_sum ? (float*)(ws + l.off_sum) : nullptr;
    for (uint64_t v0 = 0; v0 < a.vocab; v0 += l.piece) {
        const uint32_t n = (uint32_t)(a.vocab - v0 < l.piece ? a.vocab - v0 : l.piece);
        const uint16_t* wp = (const uint16_t*)w + v0 * ld_w;
        const Operand oh{h, a.tokens, a.width, ld_h, 0, 1, false}, ow{wp, n, a.width, ld_w, 0, 1, false};
        GemmGroup g{};
        g.bf16 = a.type == SK_BF16;
        g.M = tokens;
        g.N = n;
        if (l.rows > a.tokens) {                         // one tile high
            const GradEpi<true>::Args ga{gbuf, gbuf + a.tokens * l.ld_g, l.ld_g, a.lse, a.dloss, factor, a.targets, a.vocab, (uint32_t)v0};
            SK_OP_CUDA((launch_products<1, 128, GradEpi<true>>(true, oh, ow, g, 1, nullptr, nullptr, nullptr, dev.waits(), ga, dev.sm_count, st)));
        } else {
            const GradEpi<false>::Args ga{gbuf, nullptr, l.ld_g, a.lse, a.dloss, factor, a.targets, a.vocab, (uint32_t)v0};
            auto launch_g = wide_tiles(tokens, n, (a.width + kGemmK - 1) / kGemmK, dev.sm_count) ? launch_products<2, 256, GradEpi<false>>
                                                                                                  : launch_products<1, 128, GradEpi<false>>;
            SK_OP_CUDA(launch_g(true, oh, ow, g, 1, nullptr, nullptr, nullptr, dev.waits(), ga, dev.sm_count, st));
        }
        // dW[v] = sum over tokens of G[t][v] hidden[t]: both factors with their rows contiguous;
        // dhidden[t] += sum over the piece of G[t][v] W[v]
        const Operand gt{gbuf, l.rows, n, l.ld_g, 0, 1, true}, ht{h, l.rows, a.width, ld_h, 0, 1, true};
        const Operand og{gbuf, l.rows, n, l.ld_g, 0, 1, false}, wt{wp, n, a.width, ld_w, 0, 1, true};
        GemmGroup gw = g, gh = g;
        gw.M = n;
        gw.N = gh.N = width;
        gh.M = (uint32_t)l.rows;
        OutEpi::One one_w{}, one_h{};
        one_w.out = (uint8_t*)a.dweight + v0 * a.ld_dweight * type_size(a.dweight_type);
        one_w.ld = a.ld_dweight;
        one_w.type = a.dweight_type;
        one_w.align = row_alignment(one_w.out, one_w.ld, one_w.type);
        one_h.out = a.dhidden;
        one_h.type = a.dhidden_type;
        one_h.ld = sum ? l.ld_sum : a.ld_dhidden;
        one_h.sum = sum;
        one_h.sum_stride = l.sum_stride;
        one_h.add = v0 != 0;
        one_h.align = row_alignment(one_h.out, one_h.ld, one_h.type);
        const bool h_first = n >= tokens;                // the one with the longer K is the first
        const uint32_t split = h_first ? l.slices : 1;   // of dhidden's product, when it is the first
        OutEpi::Args ea{{h_first ? one_h : one_w, h_first ? one_w : one_h}, factor};
        auto launch = l.wide ? launch_products<2, 256, OutEpi> : launch_products<1, 256, OutEpi>;
        const bool both = a.dweight && a.dhidden, h_is_0 = both ? h_first : a.dhidden != nullptr;
        if (!both) ea.o[0] = h_is_0 ? one_h : one_w;
        SK_OP_CUDA(launch(true, h_is_0 ? og : gt, h_is_0 ? wt : ht, h_is_0 ? gh : gw, h_is_0 ? split : 1, h_is_0 ? &gt : &og, h_is_0 ? &ht : &wt,
                          both ? (h_is_0 ? &gw : &gh) : nullptr, dev.waits(), ea, dev.sm_count, st));
    }
    if (sum) {
        const uint64_t want = (a.tokens * ((width + 3) / 4) + 255) / 256, most = (uint64_t)dev.sm_count * 8;
        SK_OP_CUDA(launch_kernel(true, k_head_sum, dim3((uint32_t)(want < most ? want : most)), 256, 0, st, (const float*)sum, l.slices, l.sum_stride,
                                 l.rows > a.tokens ? a.tokens * l.ld_sum : 0, l.ld_sum, a.tokens, width, (const float*)factor, a.dhidden, a.ld_dhidden, a.dhidden_type));
    }
    return SK_OK;
}

}  // namespace sk
