// The clipped policy loss with a KL term over the tokens of ragged sequences, and its gradient.
//
//   d = old_nll - nll (the log of the ratio r = exp d);  A >= 0: s = A min(r, 1 + high);  A < 0: s = A max(r, 1 - low)
//   e = nll - reference_nll;  k = exp e - e - 1;  token loss = -s + kl k
//   loss = sum over the tokens that take part of norm token loss;  norm: one over their number, or one over the number of sequences that have
//   any and over their number in the sequence
//   d loss / d nll = norm ([not clipped] A r + kl (exp e - 1))
//
// What is clipped is decided as on d in 64 bits, where the difference of two 32-bit numbers is exact enough, so that the loss and its gradient, which are
// two calls, and anyone who computes the formula decide alike.  A = 0 gives 0 however far r or its bound is, beyond 32 bits too.
//
// Tokens are taken in chunks of kChunk by a block each.  A chunk adds up what it has of each sequence; a sequence that goes over several chunks has
// one sum where it begins (unless that is a chunk's first token) and one for each chunk whose first token is its own.  A second launch joins
// them, in order; a single chunk's block does so itself.  The same bits every time.  1003 tokens with their gradient 11 us, bound by latency; 1000003 19.2 us (28 MB, 4.3 at the copy
// rate): three launches, of which the large ones load in one wave of blocks and then compute, 143 instructions a token.
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint32_t kPolicyThreads = 256, kPerThread = 8, kChunk = kPolicyThreads * kPerThread;
constexpr uint32_t kPolicyJoin = 1024;               // threads of the second launch, at most

// exp(e) - e - 1 for |e| < 1, by its series, in which nothing cancels: the next term is 3e-9 of the sum at 1, 6e-9 at -1.
__device__ __forceinline__ float k_series(float e) {
    float s = 1.0f / 39916800;
    s = fmaf(s, e, 1.0f / 3628800);
    s = fmaf(s, e, 1.0f / 362880);
    s = fmaf(s, e, 1.0f / 40320);
    s = fmaf(s, e, 1.0f / 5040);
    s = fmaf(s, e, 1.0f / 720);
    s = fmaf(s, e, 1.0f / 120);
    s = fmaf(s, e, 1.0f / 24);
    s = fmaf(s, e, 1.0f / 6);
    s = fmaf(s, e, 0.5f);
    return s * (e * e);
}
// exp(e) - e - 1 and its derivative exp(e) - 1. From 1 on by exp, whose error is at most 3.8 and 1.6 times as large relative to the difference (at 1). The derivative is not
// formed from the value there: e, however large, would be subtracted and added again (-1 became 0 for e below -2^24, NaN for -inf). Beside exp(128), which overflows, e does
// not matter, and an infinite one would give inf - inf.
__device__ __forceinline__ float k_term(float e) { return fabsf(e) < 1.0f ? k_series(e) : expf(e) - fminf(e, 128.0f) - 1.0f; }
__device__ __forceinline__ float k_slope(float e) {
    float s = k_series(e) + e;
    if (!(fabsf(e) < 1.0f)) s = expf(e) - 1.0f;
    return s;
}

struct Token { float ratio, held, advantage; bool clipped; };        // held: the bound that takes the ratio's place
// The difference is rounded once, like the argument of exp; it says by itself what is clipped unless it lies within its rounding of the border. Ratios that may overflow, as rare,
// take the same branch: of an advantage of zero they leave nothing. (Asked for each product by itself, that took the gradient of 1000003 tokens from 8.1 to 8.6 us.)
__device__ __forceinline__ Token token_of(const PolicyArgs& a, float old_nll, float nll, float advantage) {
    const float d = old_nll - nll;
    Token v;
    v.ratio = expf(d);
    v.advantage = advantage;
    const bool up = advantage >= 0;
    const float border = up ? a.border_high : a.border_low;
    v.clipped = up ? d > border : d < border;
    v.held = up ? a.high : a.low;
    if (fabsf(d - border) <= 0x1p-21f * fabsf(border) || d > 88.0f) {
        const double exact = (double)old_nll - (double)nll;
        v.clipped = up ? exact > a.log_high : exact < a.log_low;
        if (advantage == 0 && d > 88.0f) v.ratio = v.held = 0.0f;
    }
    return v;
}

// The number of sequences that begin at or before token t, less one: the token's own (or, behind the last one's end, the number of sequences; before
// the first, -1).  By a whole warp: 32 probes at a time.
__device__ __forceinline__ int64_t sequence_of(const int64_t* offsets, int64_t count, int64_t t) {
    const int64_t lane = threadIdx.x & 31;
    int64_t low = 0, high = count;                   // offsets[i] <= t for all i < low, > t for all i >= high
    while (low < high) {
        const int64_t step = (high - low + 31) / 32, at = low + (lane + 1) * step - 1;       // the ends of 32 pieces
        const uint32_t under = __popc(__ballot_sync(0xffffffffu, at < high && offsets[at] <= t));
        const int64_t from = low + under * step;
        high = min(high, from + step - 1);
        low = min(from, high);
    }
    return low - 1;
}

// What a block knows of the sequences of its tokens, from the first token's to the last one's: where they begin, counted from its first token, if they
// are few; else they are looked up in the offsets.
constexpr uint32_t kHeld = 256;
struct Range {
    int64_t first, last;
    uint32_t count;                                  // of those that begin inside
    const uint32_t* begins;                          // null: too many
};
__device__ __forceinline__ Range range_of(const PolicyArgs& a, uint64_t c0, uint64_t c1) {
    __shared__ int64_t found[2];
    __shared__ uint32_t held[kHeld];
    if (!a.offsets) return {0, 0, 0, held};
    const uint32_t warp = threadIdx.x >> 5;
    if (warp < 2) {
        const int64_t s = sequence_of(a.offsets, (int64_t)a.sequences + 1, (int64_t)(warp ? c1 - 1 : c0));
        if ((threadIdx.x & 31) == 0) found[warp] = s;
    }
    __syncthreads();
    const int64_t first = found[0], last = max(found[1], first);         // offsets that decrease are no reason to look anywhere else
    if (last - first > (int64_t)kHeld) return {first, last, 0, nullptr};
    const uint32_t count = (uint32_t)(last - first);
    if (count) {
        for (uint32_t i = threadIdx.x; i < count; i += blockDim.x) held[i] = (uint32_t)max(a.offsets[first + 1 + i] - (int64_t)c0, (int64_t)0);
        __syncthreads();
    }
    return {first, last, count, held};
}
// of token c0 + at
__device__ __forceinline__ int64_t own_sequence(const PolicyArgs& a, const Range& r, uint64_t c0, uint32_t at) {
    if (!r.begins) {
        int64_t low = r.first + 1, high = r.last + 1;        // offsets[i] <= token for all i < low, > for all i >= high
        while (low < high) {
            const int64_t middle = (low + high) >> 1;
            if (a.offsets[middle] <= (int64_t)(c0 + at)) low = middle + 1;
            else high = middle;
        }
        return low - 1;
    }
    uint32_t low = 0, high = r.count;
    while (low < high) {
        const uint32_t middle = (low + high) >> 1;
        if (r.begins[middle] <= at) low = middle + 1;
        else high = middle;
    }
    return r.first + low;
}

// kN tokens of a thread, kPolicyThreads apart: everything is loaded before anything is computed, of tokens that take no part too.
template <uint32_t kN>
struct Tokens {
    float nll[kN], old_nll[kN], advantage[kN], reference[kN];
    uint32_t sequence[kN];
    uint32_t live;                                   // a bit each
    __device__ __forceinline__ void load(float (&v)[kN], const float* p, uint32_t rest) {
#pragma unroll
        for (uint32_t i = 0; i < kN; ++i) v[i] = i * kPolicyThreads < rest ? p[i * kPolicyThreads] : 0.0f;
    }
    __device__ __forceinline__ Tokens(const PolicyArgs& a, uint64_t c0, uint64_t c1) {
        const uint64_t t0 = c0 + threadIdx.x;
        const uint32_t rest = t0 < c1 ? (uint32_t)(c1 - t0) : 0;
        load(nll, a.nll + t0, rest);
        load(old_nll, a.old_nll + t0, rest);
        if (a.reference) load(reference, a.reference + t0, rest);
        if (!a.advantage_of_sequences) load(advantage, a.advantages + t0, rest);
        live = 0;
        const int64_t* targets = a.targets + (a.targets ? t0 : 0);
#pragma unroll
        for (uint32_t i = 0; i < kN; ++i)
            if (i * kPolicyThreads < rest && (!a.targets || targets[i * kPolicyThreads] >= 0)) live |= 1u << i;
    }
    __device__ __forceinline__ void place(const PolicyArgs& a, const Range& r, uint64_t c0) {
#pragma unroll
        for (uint32_t i = 0; i < kN; ++i) {
            const int64_t q = own_sequence(a, r, c0, i * kPolicyThreads + threadIdx.x);
            if (q < 0 || q >= (int64_t)a.sequences) live &= ~(1u << i);
            sequence[i] = live >> i & 1 ? (uint32_t)q : 0;
        }
        if (a.advantage_of_sequences) {
#pragma unroll
            for (uint32_t i = 0; i < kN; ++i) advantage[i] = a.advantages[sequence[i]];      // there is at least one sequence
        }
    }
};

// sums of a chunk in 32 bits, of chunks in 64
struct Sums { double loss, k, clipped, count; };
__device__ __forceinline__ void add(Sums& s, const Sums& o) { s.loss += o.loss; s.k += o.k; s.clipped += o.clipped; s.count += o.count; }
__device__ __forceinline__ void add(Sums& s, const float4& o) { s.loss += o.x; s.k += o.y; s.clipped += o.z; s.count += o.w; }
__device__ __forceinline__ void add(float4& s, const float4& o) { s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w; }
__device__ __forceinline__ Sums over(const Sums& s, int o) {
    return {__shfl_xor_sync(0xffffffffu, s.loss, o), __shfl_xor_sync(0xffffffffu, s.k, o), __shfl_xor_sync(0xffffffffu, s.clipped, o),
            __shfl_xor_sync(0xffffffffu, s.count, o)};
}
__device__ __forceinline__ float4 over(const float4& s, int o) {
    return make_float4(__shfl_xor_sync(0xffffffffu, s.x, o), __shfl_xor_sync(0xffffffffu, s.y, o), __shfl_xor_sync(0xffffffffu, s.z, o),
                       __shfl_xor_sync(0xffffffffu, s.w, o));
}
template <class T>
__device__ __forceinline__ void warp_sum(T& s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) add(s, over(s, o));
}
// over the block, to every thread
template <class T>
__device__ T block_sum(T s) {
    __shared__ T parts[kPolicyJoin / 32];
    warp_sum(s);
    __syncthreads();                                 // what was read before has been
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = s;
    __syncthreads();
    T r{};
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) add(r, parts[w]);
    return r;
}

// heads: chunks' sums (of all their tokens, or of their first token's sequence); starts: for each sequence the sum where it begins
__device__ void join(const PolicyArgs& a, uint32_t chunks, const float4* heads, const float4* starts) {
    if (!a.average_sequences) {
        Sums s{};
        for (uint32_t c = threadIdx.x; c < chunks; c += blockDim.x) add(s, heads[c]);
        s = block_sum(s);
        const double each = s.count > 0 ? 1.0 / s.count : 0.0;
        for (uint64_t q = threadIdx.x; q < a.sequences; q += blockDim.x) a.norm[q] = (float)each;
        if (threadIdx.x == 0) {
            a.result[0] = (float)(s.loss * each);
            a.result[1] = (float)(s.k * each);
            a.result[2] = (float)(s.clipped * each);
        }
        return;
    }
    const uint32_t lane = threadIdx.x & 31;
    Sums all{};                                      // of the sequences' means; count: of sequences
    for (uint64_t q0 = 0; q0 < a.sequences; q0 += blockDim.x) {
        const uint64_t q = q0 + threadIdx.x;
        int64_t from = 0, to = 0;
        if (q < a.sequences) {
            from = a.offsets ? max(a.offsets[q], (int64_t)0) : 0;
            to = a.offsets ? min(a.offsets[q + 1], (int64_t)a.tokens) : (int64_t)a.tokens;
        }
        Sums s{};
        uint32_t c0 = 0, c1 = 0;                     // chunks whose first token is the sequence's
        if (from < to) {
            c0 = (uint32_t)((from + kChunk - 1) / kChunk);
            c1 = (uint32_t)((to - 1) / kChunk) + 1;
            if (from % kChunk) add(s, starts[q]);
        }
        const bool is_long = c1 > c0 + 4;
        if (!is_long)
            for (uint32_t c = c0; c < c1; ++c) add(s, heads[c]);
        for (uint32_t who = __ballot_sync(0xffffffffu, is_long); who; who &= who - 1) {          // the whole warp for a long one
            const int l = __ffs(who) - 1;
            const uint32_t b = __shfl_sync(0xffffffffu, c0, l), e = __shfl_sync(0xffffffffu, c1, l);
            Sums p{};
            for (uint32_t c = b + lane; c < e; c += 32) add(p, heads[c]);
            warp_sum(p);
            if ((int)lane == l) add(s, p);
        }
        if (q < a.sequences) a.norm[q] = (float)s.count;         // for now: at most 2^24 are exact, see below
        if (s.count > 0) add(all, Sums{s.loss / s.count, s.k / s.count, s.clipped / s.count, 1.0});
    }
    all = block_sum(all);
    const double each = all.count > 0 ? 1.0 / all.count : 0.0;
    for (uint64_t q = threadIdx.x; q < a.sequences; q += blockDim.x) {
        const float count = a.norm[q];
        a.norm[q] = count > 0 ? (float)(each / count) : 0.0f;
    }
    if (threadIdx.x == 0) {
        a.result[0] = (float)(all.loss * each);
        a.result[1] = (float)(all.k * each);
        a.result[2] = (float)(all.clipped * each);
    }
}

// One chunk of few sequences keeps its sums to itself and needs no workspace.
constexpr uint32_t kOwnSums = 64;
__global__ void __launch_bounds__(kPolicyThreads, 4) k_policy(const __grid_constant__ PolicyArgs a) {
    __shared__ float4 of_token[kChunk], own[1 + kOwnSums];
    float4* const sums = a.workspace ? a.workspace : own;
    chain_acquire();
    const uint64_t c0 = (uint64_t)blockIdx.x * kChunk, c1 = min(c0 + kChunk, a.tokens);
    Tokens<kPerThread> t(a, c0, c1);
    const Range r = range_of(a, c0, c1);
    t.place(a, r, c0);
    float4 s = make_float4(0, 0, 0, 0);
#pragma unroll
    for (uint32_t i = 0; i < kPerThread; ++i) {
        float4 v = make_float4(0, 0, 0, 0);
        if (t.live >> i & 1) {
            const Token p = token_of(a, t.old_nll[i], t.nll[i], t.advantage[i]);
            v.x = -p.advantage * (p.clipped ? p.held : p.ratio);
            if (a.reference) {
                v.y = k_term(t.nll[i] - t.reference[i]);
                if (a.kl != 0) v.x += a.kl * v.y;
            }
            v.z = p.clipped;
            v.w = 1;
        }
        if (a.average_sequences) of_token[i * kPolicyThreads + threadIdx.x] = v;
        add(s, v);
    }
    const uint32_t chunks = gridDim.x;
    if (!a.average_sequences) {
        s = block_sum(s);
        if (threadIdx.x == 0) sums[blockIdx.x] = s;
    } else {
        __syncthreads();
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        uint32_t turn = warp;
        for (int64_t q0 = r.first; q0 <= r.last; q0 += 32) {                                     // a lane finds each one's tokens, the warps take turns adding up
            const int64_t q = q0 + lane;
            int64_t from = 0, to = 0;
            bool begins_here = false;
            if (q >= 0 && q <= r.last && q < (int64_t)a.sequences) {
                const int64_t begin = a.offsets ? a.offsets[q] : 0, end = a.offsets ? a.offsets[q + 1] : (int64_t)a.tokens;
                from = max(begin, (int64_t)c0);
                to = min(end, (int64_t)c1);
                begins_here = begin > (int64_t)c0;
            }
            const uint32_t first = (uint32_t)(from - (int64_t)c0), count = from < to ? (uint32_t)(to - from) : 0;
            for (uint32_t some = __ballot_sync(0xffffffffu, count > 0); some; some &= some - 1) {
                if (turn++ % (kPolicyThreads / 32)) continue;
                const int l = __ffs(some) - 1;
                const uint32_t f = __shfl_sync(0xffffffffu, first, l), n = __shfl_sync(0xffffffffu, count, l);
                float4 p = make_float4(0, 0, 0, 0);
                for (uint32_t i = lane; i < n; i += 32) add(p, of_token[f + i]);
                warp_sum(p);
                if ((int)lane == l) sums[begins_here ? chunks + q : blockIdx.x] = p;
            }
        }
    }
    if (chunks > 1) return;
    __syncthreads();
    join(a, 1, sums, sums + 1);
}

__global__ void __launch_bounds__(kPolicyJoin) k_policy_join(const __grid_constant__ PolicyArgs a, uint32_t chunks) {
    chain_acquire();
    join(a, chunks, a.workspace, a.workspace + chunks);
}

constexpr uint32_t kBackEach = 4;
__global__ void __launch_bounds__(kPolicyThreads) k_policy_backward(const __grid_constant__ PolicyArgs a) {
    chain_acquire();
    const uint64_t c0 = (uint64_t)blockIdx.x * (kPolicyThreads * kBackEach), c1 = min(c0 + kPolicyThreads * kBackEach, a.tokens);
    Tokens<kBackEach> t(a, c0, c1);
    const float dloss = a.dloss ? *a.dloss : 1.0f;
    const Range r = range_of(a, c0, c1);
    t.place(a, r, c0);
    float norm[kBackEach];
#pragma unroll
    for (uint32_t i = 0; i < kBackEach; ++i) norm[i] = a.norm[t.sequence[i]];
#pragma unroll
    for (uint32_t i = 0; i < kBackEach; ++i) {
        const uint64_t at = c0 + i * kPolicyThreads + threadIdx.x;
        float g = 0;
        if (t.live >> i & 1) {
            const Token p = token_of(a, t.old_nll[i], t.nll[i], t.advantage[i]);
            g = p.clipped ? 0.0f : p.advantage * p.ratio;
            if (a.reference && a.kl != 0) g += a.kl * k_slope(t.nll[i] - t.reference[i]);
            g *= dloss * norm[i];
        }
        if (at < c1) a.dnll[at] = g;
    }
}

uint64_t chunks_of(uint64_t tokens) { return (tokens + kChunk - 1) / kChunk; }

}  // namespace

uint64_t policy_workspace(uint64_t tokens, uint64_t sequences) {
    return tokens <= kChunk && sequences <= kOwnSums ? 0 : (chunks_of(tokens) + sequences) * sizeof(float4);
}

int launch_policy(PolicyArgs a, cudaStream_t st) {
    if (!policy_workspace(a.tokens, a.sequences)) a.workspace = nullptr;
    const uint32_t chunks = (uint32_t)chunks_of(a.tokens);
    SK_OP_CUDA(launch_kernel(true, k_policy, dim3(chunks), kPolicyThreads, 0, st, a));
    // a thread a sequence; sums over the chunks need few
    const uint32_t threads = a.average_sequences && a.sequences > kPolicyThreads ? kPolicyJoin : kPolicyThreads;
    if (chunks > 1) SK_OP_CUDA(launch_kernel(true, k_policy_join, dim3(1), threads, 0, st, a, chunks));
    return SK_OK;
}

int launch_policy_backward(const PolicyArgs& a, cudaStream_t st) {
    const uint64_t each = kPolicyThreads * kBackEach;
    SK_OP_CUDA(launch_kernel(true, k_policy_backward, dim3((uint32_t)((a.tokens + each - 1) / each)), kPolicyThreads, 0, st, a));
    return SK_OK;
}

}  // namespace sk
