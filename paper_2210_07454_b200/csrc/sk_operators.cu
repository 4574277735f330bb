// C entry points of the language-model operators: checks of arguments, what is known of the device, TMA descriptors.
#include "sk_operators.h"
#include "sk_gemm.cuh"

#include <atomic>
#include <cmath>

namespace sk {
namespace {

// How many waits inside kernels have run out on the device, ever, and how many of them have been reported.  Nothing is set back on the
// device, so a wait that runs out while another is being reported is not lost.
__device__ uint32_t g_op_status;
std::atomic<uint32_t> g_reported[64];

thread_local OpDevice t_devices[64];
thread_local uint32_t t_withhold_ms;             // of this thread's next call, see sk_test_operators_wait

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
std::atomic<EncodeFn> g_encode{nullptr};

}  // namespace

int op_device(OpDevice* out) {
    int d = 0;
    SK_OP_CUDA(cudaGetDevice(&d));
    if (d < 0 || d >= 64) return set_error(SK_EINVAL, "device %d: the operators know 64 devices", d);
    OpDevice& dev = t_devices[d];
    if (!dev.status) {
        if (!g_encode.load()) {
            void* fn = nullptr;
            cudaDriverEntryPointQueryResult found{};
            SK_OP_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found));
            if (found != cudaDriverEntryPointSuccess || !fn) return set_error(SK_ECUDA, "the driver has no cuTensorMapEncodeTiled");
            g_encode.store((EncodeFn)fn);
        }
        SK_OP_CUDA(cudaDeviceGetAttribute(&dev.sm_count, cudaDevAttrMultiProcessorCount, d));
        void* p = nullptr;
        SK_OP_CUDA(cudaGetSymbolAddress(&p, g_op_status));
        dev.status = (uint32_t*)p;
    }
    *out = dev;
    return SK_OK;
}

bool encode_operand(CUtensorMap* map, const Operand& o, bool bf16, uint32_t box_rows) {
    const cuuint64_t dims[3] = {o.cols, o.rows, o.batch};
    const cuuint64_t strides[2] = {o.ld * 2, (o.batch > 1 ? o.batch_stride : round_up(o.rows * o.ld, 8)) * 2};
    const cuuint32_t box[3] = {64, box_rows, 1}, elem[3] = {1, 1, 1};
    return g_encode.load()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(o.p), dims, strides, box,
                    elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

namespace {
bool misaligned(const void* p, int type) { return (uintptr_t)p % type_size(type) != 0; }
int check_workspace(const char* who, const void* ws, uint64_t have, uint64_t need) {
    if (need && !ws) return set_error(SK_EINVAL, "%s: null workspace (%llu bytes are needed)", who, (unsigned long long)need);
    if (have < need)
        return set_error(SK_EINVAL, "%s: a workspace of %llu bytes is needed, got %llu", who, (unsigned long long)need, (unsigned long long)have);
    if ((uintptr_t)ws % 256) return set_error(SK_EINVAL, "%s: the workspace must be 256-byte aligned", who);
    return SK_OK;
}
constexpr uint64_t kMaxExtent = 1ull << 31;
}  // namespace
}  // namespace sk

using namespace sk;

extern "C" {

int sk_layer_norm(const void* x, uint64_t ld_x, void* y, uint64_t ld_y, int type, uint64_t rows, uint64_t cols, const void* weight, const void* bias,
                  int weight_type, float eps, float* mean, float* rstd, void* stream) {
    const char* who = "sk_layer_norm";
    if (!type_ok(type) || !type_ok(weight_type)) return set_error(SK_EINVAL, "%s: unknown type", who);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(SK_EINVAL, "%s: eps must be finite and not negative", who);
    if (cols < 1 || cols >= kMaxExtent) return set_error(SK_EINVAL, "%s: cols must be in 1..2^31-1", who);
    if (rows >= (1ull << 40)) return set_error(SK_EINVAL, "%s: too many rows", who);
    if (rows == 0) return SK_OK;
    if (!x || !y) return set_error(SK_EINVAL, "%s: null argument", who);
    if (ld_x < cols || ld_y < cols) return set_error(SK_EINVAL, "%s: a leading dimension is below cols", who);
    if (rows > 1 && y == x && ld_y != ld_x) return set_error(SK_EINVAL, "%s: in place, the leading dimensions must be the same", who);
    if (misaligned(x, type) || misaligned(y, type) || misaligned(weight, weight_type) || misaligned(bias, weight_type) || misaligned(mean, SK_F32) ||
        misaligned(rstd, SK_F32))
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    const NormArgs a{x, weight, bias, y, mean, rstd, rows, cols, ld_x, ld_y, type, weight_type, eps};
    return launch_norm(a, dev.sm_count, (cudaStream_t)stream);
}

uint64_t sk_layer_norm_backward_workspace(uint64_t rows, uint64_t cols) {
    OpDevice dev;
    if (op_device(&dev) || cols < 1 || cols >= kMaxExtent) return 0;
    return norm_backward_workspace(rows, cols, dev.sm_count);
}

int sk_layer_norm_backward(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, void* dx, uint64_t ld_dx, int type, uint64_t rows, uint64_t cols,
                           const void* weight, int weight_type, const float* mean, const float* rstd, void* dweight, void* dbias, int dweight_type,
                           void* workspace, uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_layer_norm_backward";
    if (!type_ok(type) || !type_ok(weight_type) || !type_ok(dweight_type)) return set_error(SK_EINVAL, "%s: unknown type", who);
    if (cols < 1 || cols >= kMaxExtent) return set_error(SK_EINVAL, "%s: cols must be in 1..2^31-1", who);
    if (rows >= (1ull << 40)) return set_error(SK_EINVAL, "%s: too many rows", who);
    if (misaligned(dy, type) || misaligned(x, type) || misaligned(dx, type) || misaligned(weight, weight_type) || misaligned(mean, SK_F32) ||
        misaligned(rstd, SK_F32) || misaligned(dweight, dweight_type) || misaligned(dbias, dweight_type))
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (rows == 0) {                              // sums over no rows
        if (dweight) SK_OP_CUDA(cudaMemsetAsync(dweight, 0, cols * type_size(dweight_type), (cudaStream_t)stream));
        if (dbias) SK_OP_CUDA(cudaMemsetAsync(dbias, 0, cols * type_size(dweight_type), (cudaStream_t)stream));
        return SK_OK;
    }
    if (!dy || !x || !mean || !rstd) return set_error(SK_EINVAL, "%s: null argument", who);
    if (ld_dy < cols || ld_x < cols || (dx && ld_dx < cols)) return set_error(SK_EINVAL, "%s: a leading dimension is below cols", who);
    if (rows > 1 && ((dx == x && ld_dx != ld_x) || (dx == dy && ld_dx != ld_dy)))
        return set_error(SK_EINVAL, "%s: in place, the leading dimensions must be the same", who);
    if (!dx && !dweight && !dbias) return SK_OK;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    const bool sums = dweight || dbias;
    if (int rc = check_workspace(who, workspace, workspace_bytes, sums ? norm_backward_workspace(rows, cols, dev.sm_count) : 0)) return rc;
    const NormBackwardArgs a{dy, x, weight, mean, rstd, dx, dweight, dbias, sums ? (float*)workspace : nullptr, 0, rows, cols, ld_dy, ld_x, ld_dx,
                             type, weight_type, dweight_type};
    return launch_norm_backward(a, dev.sm_count, (cudaStream_t)stream);
}

static int head_checked(const char* who, const HeadArgs& a) {
    if (a.type != SK_BF16 && a.type != SK_F16) return set_error(SK_EINVAL, "%s: type must be SK_BF16 or SK_F16", who);
    if (a.vocab < 1 || a.vocab >= kMaxExtent || a.tokens >= kMaxExtent || a.width < 1 || a.width >= kMaxExtent)
        return set_error(SK_EINVAL, "%s: vocab and width must be in 1..2^31-1, tokens below 2^31", who);
    if (a.tokens && (!a.hidden || !a.weight || !a.targets)) return set_error(SK_EINVAL, "%s: null argument", who);
    if (a.ld_hidden < a.width || a.ld_weight < a.width) return set_error(SK_EINVAL, "%s: a leading dimension is below width", who);
    if (a.ld_hidden >= (1ull << 36) || a.ld_weight >= (1ull << 36)) return set_error(SK_EINVAL, "%s: a leading dimension is too large", who);
    if (misaligned(a.hidden, a.type) || misaligned(a.weight, a.type) || (uintptr_t)a.targets % 8 || misaligned(a.lse, SK_F32))
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    return SK_OK;
}

uint64_t sk_linear_cross_entropy_workspace(const void* hidden, uint64_t ld_hidden, const void* weight, uint64_t ld_weight, uint64_t tokens, uint64_t vocab,
                                           uint64_t width) {
    HeadArgs a{};
    a.hidden = hidden; a.ld_hidden = ld_hidden; a.weight = weight; a.ld_weight = ld_weight;
    a.tokens = tokens; a.vocab = vocab; a.width = width;
    return tokens && vocab ? head_workspace(a) : 0;
}

int sk_linear_cross_entropy(const void* hidden, uint64_t ld_hidden, const void* weight, uint64_t ld_weight, int type, uint64_t tokens, uint64_t vocab,
                            uint64_t width, const int64_t* targets, float* loss, float* lse, void* workspace, uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_linear_cross_entropy";
    HeadArgs a{};
    a.hidden = hidden; a.ld_hidden = ld_hidden; a.weight = weight; a.ld_weight = ld_weight;
    a.type = type; a.tokens = tokens; a.vocab = vocab; a.width = width;
    a.targets = targets; a.loss = loss; a.lse = lse; a.workspace = workspace;
    if (int rc = head_checked(who, a)) return rc;
    if (misaligned(loss, SK_F32)) return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (!tokens || (!loss && !lse)) return SK_OK;
    if (int rc = check_workspace(who, workspace, workspace_bytes, head_workspace(a))) return rc;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    return launch_head(a, dev, (cudaStream_t)stream);
}

uint64_t sk_linear_cross_entropy_backward_workspace(const void* hidden, uint64_t ld_hidden, const void* weight, uint64_t ld_weight, uint64_t tokens,
                                                    uint64_t vocab, uint64_t width) {
    HeadArgs a{};
    a.hidden = hidden; a.ld_hidden = ld_hidden; a.weight = weight; a.ld_weight = ld_weight;
    a.tokens = tokens; a.vocab = vocab; a.width = width;
    a.dhidden = a.dweight = &a;                   // as if both were wanted
    return tokens && vocab ? head_backward_workspace(a) : 0;
}

int sk_linear_cross_entropy_backward(const float* dloss, const void* hidden, uint64_t ld_hidden, const void* weight, uint64_t ld_weight, int type,
                                     uint64_t tokens, uint64_t vocab, uint64_t width, const int64_t* targets, const float* lse, void* dhidden,
                                     uint64_t ld_dhidden, int dhidden_type, void* dweight, uint64_t ld_dweight, int dweight_type, void* workspace,
                                     uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_linear_cross_entropy_backward";
    HeadArgs a{};
    a.hidden = hidden; a.ld_hidden = ld_hidden; a.weight = weight; a.ld_weight = ld_weight;
    a.type = type; a.tokens = tokens; a.vocab = vocab; a.width = width;
    a.targets = targets; a.lse = const_cast<float*>(lse); a.dloss = dloss; a.workspace = workspace;
    a.dhidden = dhidden; a.ld_dhidden = ld_dhidden; a.dhidden_type = dhidden_type;
    a.dweight = dweight; a.ld_dweight = ld_dweight; a.dweight_type = dweight_type;
    if (int rc = head_checked(who, a)) return rc;
    if (tokens && (!dloss || !lse)) return set_error(SK_EINVAL, "%s: null argument", who);
    if ((dhidden && dhidden_type != type && dhidden_type != SK_F32) || (dweight && dweight_type != type && dweight_type != SK_F32))
        return set_error(SK_EINVAL, "%s: the gradients' types must be the inputs' or SK_F32", who);
    if ((dhidden && ld_dhidden < width) || (dweight && ld_dweight < width)) return set_error(SK_EINVAL, "%s: a leading dimension is below width", who);
    if (misaligned(dloss, SK_F32) || (dhidden && misaligned(dhidden, dhidden_type)) || (dweight && misaligned(dweight, dweight_type)))
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (!tokens) {
        if (dweight) {
            const uint64_t size = type_size(dweight_type);
            SK_OP_CUDA(cudaMemset2DAsync(dweight, ld_dweight * size, 0, width * size, vocab, (cudaStream_t)stream));
        }
        return SK_OK;
    }
    if (!dhidden && !dweight) return SK_OK;
    if (dweight == weight || dhidden == weight) return set_error(SK_EINVAL, "%s: weight's memory cannot take a gradient in place", who);
    if (int rc = check_workspace(who, workspace, workspace_bytes, head_backward_workspace(a))) return rc;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    return launch_head_backward(a, dev, (cudaStream_t)stream);
}

uint64_t sk_orthogonalize_workspace(uint64_t batch, uint64_t rows, uint64_t cols) {
    if (!batch || !rows || !cols || batch > 65535 || rows > 65536 || cols > 65536) return 0;
    OrthoArgs a{};
    a.batch = batch; a.rows = rows; a.cols = cols;
    return orthogonalize_workspace(a);
}

int sk_orthogonalize(const void* update, uint64_t ld_update, uint64_t stride_update, int type, float* momentum, uint64_t ld_momentum,
                     uint64_t stride_momentum, float beta, int nesterov, void* out, uint64_t ld_out, uint64_t stride_out, int out_type, uint64_t batch,
                     uint64_t rows, uint64_t cols, int steps, const float* coefficients, float eps, void* workspace, uint64_t workspace_bytes,
                     void* stream) {
    const char* who = "sk_orthogonalize";
    if (!type_ok(type)) return set_error(SK_EINVAL, "%s: unknown type", who);
    if (out_type != SK_BF16 && out_type != SK_F16) return set_error(SK_EINVAL, "%s: out_type must be SK_BF16 or SK_F16", who);
    if (steps < 1 || steps > 32) return set_error(SK_EINVAL, "%s: steps must be in 1..32", who);
    if (batch > 65535 || rows > 65536 || cols > 65536) return set_error(SK_EINVAL, "%s: batch must be <= 65535, rows and cols <= 65536", who);
    if (!coefficients) return set_error(SK_EINVAL, "%s: null coefficients", who);
    if (!(std::fabs(coefficients[0]) + std::fabs(coefficients[1]) + std::fabs(coefficients[2]) < 15.0f))
        return set_error(SK_EINVAL, "%s: coefficients out of range (|a| + |b| + |c| must be below 15)", who);
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return set_error(SK_EINVAL, "%s: eps must be finite and not negative", who);
    if (momentum && !std::isfinite(beta)) return set_error(SK_EINVAL, "%s: beta must be finite", who);
    if (!batch || !rows || !cols) return SK_OK;
    if (!update || !out) return set_error(SK_EINVAL, "%s: null argument", who);
    if (ld_update < cols || ld_out < cols || (momentum && ld_momentum < cols)) return set_error(SK_EINVAL, "%s: a leading dimension is below cols", who);
    if (batch > 1 && (stride_out < (rows - 1) * ld_out + cols || (momentum && stride_momentum < (rows - 1) * ld_momentum + cols)))
        return set_error(SK_EINVAL, "%s: the matrices of an output overlap", who);
    if (misaligned(update, type) || misaligned(momentum, SK_F32) || misaligned(out, out_type))
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    OrthoArgs a{};
    a.update = update; a.ld_update = ld_update; a.stride_update = stride_update; a.type = type;
    a.momentum = momentum; a.ld_momentum = ld_momentum; a.stride_momentum = stride_momentum; a.beta = beta; a.nesterov = nesterov;
    a.out = out; a.ld_out = ld_out; a.stride_out = stride_out; a.out_type = out_type;
    a.batch = batch; a.rows = rows; a.cols = cols; a.steps = steps; a.eps = eps;
    for (int i = 0; i < 3; ++i) a.coefficient[i] = coefficients[i];
    a.workspace = workspace;
    if (int rc = check_workspace(who, workspace, workspace_bytes, orthogonalize_workspace(a))) return rc;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    const uint32_t withhold_ms = t_withhold_ms;
    t_withhold_ms = 0;
    return launch_orthogonalize(a, dev, withhold_ms, (cudaStream_t)stream);
}

int sk_test_operators_wait(uint32_t limit_ms) {
    if (limit_ms < 1 || limit_ms > 1000) return set_error(SK_EINVAL, "sk_test_operators_wait: limit_ms must be in 1..1000");
    t_withhold_ms = limit_ms;
    return SK_OK;
}

int sk_operators_sync(void* stream) {
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    int d = 0;
    SK_OP_CUDA(cudaGetDevice(&d));
    uint32_t count = 0;
    SK_OP_CUDA(cudaMemcpyAsync(&count, dev.status, 4, cudaMemcpyDeviceToHost, (cudaStream_t)stream));
    SK_OP_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
    uint32_t reported = g_reported[d].load();
    do {
        if ((int32_t)(count - reported) <= 0) return SK_OK;          // reported, or overtaken by a thread that read later
    } while (!g_reported[d].compare_exchange_weak(reported, count));
    return set_error(SK_EDEVICE, "%u waits inside operators' kernels ran out: their outputs are invalid", count - reported);
}

}  // extern "C"
