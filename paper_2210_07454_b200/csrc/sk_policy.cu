// The clipped policy loss with a KL term over the tokens of ragged sequences, and its gradient.
//
//   d = old_nll - nll (the log of the ratio r = exp d);  A >= 0: s = A min(r, 1 + high);  A < 0: s = A max(r, 1 - low)
//   e = nll - reference_nll;  k = exp e - e - 1;  token loss = -s + kl k
//   loss = sum over the tokens that take part of norm token loss;  norm: one over their number, or one over the number of sequences that have
//   any and over their number in the sequence
//   d loss / d nll = norm ([not clipped] A r + kl (exp e - 1))
//
// What is clipped is decided on d in 64 bits, where the difference of two 32-bit numbers is exact enough, so that the loss and its gradient, which are two
// calls, and anyone who computes the formula decide alike.  A min(r, ...) instead of min(A r, ...): an infinite r with A = 0 is 0.
//
// Tokens are taken in chunks of kChunk by a block each.  A chunk adds up what it has of each sequence; a sequence that goes over several chunks has
// one sum where it begins (unless that is a chunk's first token) and one for each chunk whose first token is its own.  A second launch joins
// them, in order; a single chunk's block does so itself.  The same bits every time.  Bound by HBM for long rollouts, by latency for short ones.
#include "sk_chain.cuh"
#include "sk_operators.h"

namespace sk {
namespace {

constexpr uint32_t kPolicyThreads = 256, kPerThread = 8, kChunk = kPolicyThreads * kPerThread;
constexpr uint32_t kPolicyJoin = 1024;

// exp(e) - e - 1: near 0 the three cancel, and the series takes over
__device__ __forceinline__ float k_term(float e) {
    const float s = 1.0f + e * (1.0f / 3) * (1.0f + e * 0.25f * (1.0f + e * 0.2f * (1.0f + e * (1.0f / 6) * (1.0f + e * (1.0f / 7) * (1.0f + e * 0.125f)))));
    return fabsf(e) < 0.35f ? 0.5f * e * e * s : expm1f(e) - e;
}

struct Token { float ratio, advantage; bool clipped; };
__device__ __forceinline__ Token token_of(const PolicyArgs& a, uint64_t t, uint64_t sequence) {
    const double d = (double)a.old_nll[t] - (double)a.nll[t];
    Token v;
    v.ratio = expf((float)d);
    v.advantage = a.advantages[a.advantage_of_sequences ? sequence : t];
    v.clipped = v.advantage >= 0 ? d > a.log_high : d < a.log_low;
    return v;
}
__device__ __forceinline__ float drift_of(const PolicyArgs& a, uint64_t t) { return (float)((double)a.nll[t] - (double)a.reference[t]); }

// The number of sequences that begin at or before token t, of those from `low` on that begin before `high`; less one, the token's own (or, behind the
// last one's end, the number of sequences).
__device__ __forceinline__ int64_t sequence_of(const int64_t* offsets, int64_t low, int64_t high, int64_t t) {
    while (low < high) {                             // offsets[i] <= t for all i < low, > t for all i >= high
        const int64_t middle = (low + high) >> 1;
        if (offsets[middle] <= t) low = middle + 1;
        else high = middle;
    }
    return low - 1;
}

// the sequences of a chunk's first and last token
struct Range { int64_t first, last; };
__device__ __forceinline__ Range range_of(const PolicyArgs& a, uint64_t c0, uint64_t c1) {
    __shared__ int64_t found[2];
    if (!a.offsets) return {0, 0};
    if (threadIdx.x < 64 && (threadIdx.x & 31) == 0)
        found[threadIdx.x >> 5] = sequence_of(a.offsets, 0, (int64_t)a.sequences + 1, (int64_t)(threadIdx.x ? c1 - 1 : c0));
    __syncthreads();
    return {found[0], found[1]};
}
__device__ __forceinline__ int64_t own_sequence(const PolicyArgs& a, const Range& r, uint64_t t) {
    return r.first == r.last ? r.first : sequence_of(a.offsets, r.first + 1, r.last + 1, (int64_t)t);
}

struct Sums { double loss, k, clipped, count; };
__device__ __forceinline__ void add(Sums& s, const Sums& o) { s.loss += o.loss; s.k += o.k; s.clipped += o.clipped; s.count += o.count; }
__device__ __forceinline__ void add(Sums& s, const float4& o) { s.loss += o.x; s.k += o.y; s.clipped += o.z; s.count += o.w; }
__device__ __forceinline__ void warp_sum(Sums& s) {
#pragma unroll
    for (int o = 16; o; o >>= 1)
        add(s, Sums{__shfl_xor_sync(0xffffffffu, s.loss, o), __shfl_xor_sync(0xffffffffu, s.k, o), __shfl_xor_sync(0xffffffffu, s.clipped, o),
                    __shfl_xor_sync(0xffffffffu, s.count, o)});
}
// over the block, to every thread
__device__ Sums block_sum(Sums s) {
    __shared__ Sums parts[kPolicyJoin / 32];
    warp_sum(s);
    __syncthreads();                                 // what was read before has been
    if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = s;
    __syncthreads();
    Sums r{};
    for (uint32_t w = 0; w < blockDim.x / 32; ++w) add(r, parts[w]);
    return r;
}
__device__ __forceinline__ float4 narrow(const Sums& s) { return make_float4((float)s.loss, (float)s.k, (float)s.clipped, (float)s.count); }

// workspace: chunks' sums (of all their tokens, or of their first token's sequence), then for each sequence the sum where it begins
__device__ void join(const PolicyArgs& a, uint32_t chunks) {
    const float4 *heads = a.workspace, *starts = a.workspace + chunks;
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

__global__ void __launch_bounds__(kPolicyThreads) k_policy(const __grid_constant__ PolicyArgs a) {
    __shared__ float4 of_token[kChunk];
    chain_acquire();
    const uint64_t c0 = (uint64_t)blockIdx.x * kChunk, c1 = min(c0 + kChunk, a.tokens);
    const Range r = range_of(a, c0, c1);
    Sums s{};
    {
        float loss = 0, k = 0, clipped = 0, count = 0;
#pragma unroll
        for (uint32_t i = 0; i < kPerThread; ++i) {
            const uint32_t at = i * kPolicyThreads + threadIdx.x;
            const uint64_t t = c0 + at;
            float4 v = make_float4(0, 0, 0, 0);
            if (t < c1) {
                const int64_t q = own_sequence(a, r, t);
                if (q >= 0 && q < (int64_t)a.sequences && (!a.targets || a.targets[t] >= 0)) {
                    const Token p = token_of(a, t, (uint64_t)q);
                    v.x = -p.advantage * (p.clipped ? (p.advantage >= 0 ? a.high : a.low) : p.ratio);
                    if (a.reference) {
                        v.y = k_term(drift_of(a, t));
                        if (a.kl != 0) v.x += a.kl * v.y;
                    }
                    v.z = p.clipped;
                    v.w = 1;
                }
            }
            if (a.average_sequences) of_token[at] = v;
            loss += v.x; k += v.y; clipped += v.z; count += v.w;
        }
        s = Sums{loss, k, clipped, count};
    }
    const uint32_t chunks = gridDim.x;
    if (!a.average_sequences) {
        s = block_sum(s);
        if (threadIdx.x == 0) a.workspace[blockIdx.x] = narrow(s);
    } else {
        __syncthreads();
        const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        for (int64_t q = r.first + warp; q <= r.last; q += kPolicyThreads / 32) {
            if (q < 0 || q >= (int64_t)a.sequences) continue;
            const int64_t begin = a.offsets ? a.offsets[q] : 0, end = a.offsets ? a.offsets[q + 1] : (int64_t)a.tokens;
            const int64_t from = max(begin, (int64_t)c0), to = min(end, (int64_t)c1);
            if (from >= to) continue;
            Sums p{};
            for (int64_t t = from + lane; t < to; t += 32) add(p, of_token[t - c0]);
            warp_sum(p);
            if (lane == 0) a.workspace[begin <= (int64_t)c0 ? blockIdx.x : chunks + q] = narrow(p);
        }
    }
    if (chunks > 1) return;
    __syncthreads();
    join(a, 1);
}

__global__ void __launch_bounds__(kPolicyJoin) k_policy_join(const __grid_constant__ PolicyArgs a, uint32_t chunks) {
    chain_acquire();
    join(a, chunks);
}

constexpr uint32_t kBackEach = 4;
__global__ void __launch_bounds__(kPolicyThreads) k_policy_backward(const __grid_constant__ PolicyArgs a) {
    chain_acquire();
    const uint64_t c0 = (uint64_t)blockIdx.x * (kPolicyThreads * kBackEach), c1 = min(c0 + kPolicyThreads * kBackEach, a.tokens);
    const Range r = range_of(a, c0, c1);
    const float dloss = a.dloss ? *a.dloss : 1.0f;
#pragma unroll
    for (uint32_t i = 0; i < kBackEach; ++i) {
        const uint64_t t = c0 + i * kPolicyThreads + threadIdx.x;
        if (t >= c1) break;
        const int64_t q = own_sequence(a, r, t);
        float g = 0;
        if (q >= 0 && q < (int64_t)a.sequences && (!a.targets || a.targets[t] >= 0)) {
            const Token p = token_of(a, t, (uint64_t)q);
            g = p.clipped ? 0.0f : p.advantage * p.ratio;
            if (a.reference && a.kl != 0) g += a.kl * expm1f(drift_of(a, t));
            g *= dloss * a.norm[q];
        }
        a.dnll[t] = g;
    }
}

uint64_t chunks_of(uint64_t tokens) { return (tokens + kChunk - 1) / kChunk; }

}  // namespace

uint64_t policy_workspace(uint64_t tokens, uint64_t sequences) { return (chunks_of(tokens) + sequences) * sizeof(float4); }

int launch_policy(const PolicyArgs& a, cudaStream_t st) {
    const uint32_t chunks = (uint32_t)chunks_of(a.tokens);
    SK_OP_CUDA(launch_kernel(true, k_policy, dim3(chunks), kPolicyThreads, 0, st, a));
    if (chunks > 1) SK_OP_CUDA(launch_kernel(true, k_policy_join, dim3(1), kPolicyJoin, 0, st, a, chunks));
    return SK_OK;
}

int launch_policy_backward(const PolicyArgs& a, cudaStream_t st) {
    const uint64_t each = kPolicyThreads * kBackEach;
    SK_OP_CUDA(launch_kernel(true, k_policy_backward, dim3((uint32_t)((a.tokens + each - 1) / each)), kPolicyThreads, 0, st, a));
    return SK_OK;
}

}  // namespace sk
