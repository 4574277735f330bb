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

bool encode_out(CUtensorMap* map, void* out, uint64_t batch, uint64_t rows, uint64_t cols, uint64_t ld, uint64_t stride, int type, uint32_t box_rows) {
    const uint64_t size = type_size(type);
    const cuuint64_t dims[3] = {cols, rows, batch}, strides[2] = {ld * size, stride * size};
    const cuuint32_t box[3] = {32, box_rows, 1}, elem[3] = {1, 1, 1};
    const CUtensorMapDataType t = type == SK_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : type == SK_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return g_encode.load()(map, t, 3, out, dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, type == SK_F32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                           CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
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
uint32_t take_withhold_ms() {
    const uint32_t ms = t_withhold_ms;
    t_withhold_ms = 0;
    return ms;
}
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
    return launch_orthogonalize(a, dev, take_withhold_ms(), (cudaStream_t)stream);
}

static int grouped_checked(const char* who, const GroupedArgs& a, bool backward) {
    if (a.type != SK_BF16 && a.type != SK_F16) return set_error(SK_EINVAL, "%s: type must be SK_BF16 or SK_F16", who);
    if (a.groups < 1 || a.groups > kMaxGroups) return set_error(SK_EINVAL, "%s: groups must be in 1..%u", who, kMaxGroups);
    if (a.rows > (1ull << 30)) return set_error(SK_EINVAL, "%s: rows must be <= 2^30", who);
    if (a.width < 1 || a.width > (1u << 20) || a.out < 1 || a.out > (1u << 20)) return set_error(SK_EINVAL, "%s: width and out must be in 1..2^20", who);
    const uint64_t tile_rows = a.rows / 128 + a.groups + 2, tw = a.width / 128 + 1, to = a.out / 128 + 1;
    if (tile_rows * (tw > to ? tw : to) >= kMaxExtent || a.groups * tw * to >= kMaxExtent) return set_error(SK_EINVAL, "%s: the product is too large", who);
    if (a.rows && (!a.x || !a.weight || !a.offsets || (backward && !a.dy))) return set_error(SK_EINVAL, "%s: null argument", who);
    if (a.ld_x < a.width || a.ld_weight < a.width || (backward && a.ld_dy < a.out)) return set_error(SK_EINVAL, "%s: a leading dimension is below the rows' length", who);
    if (a.ld_x >= (1ull << 36) || a.ld_weight >= (1ull << 36) || a.ld_dy >= (1ull << 36) || a.stride_weight >= (1ull << 38))
        return set_error(SK_EINVAL, "%s: a leading dimension or stride is too large", who);
    if (misaligned(a.x, a.type) || misaligned(a.weight, a.type) || misaligned(a.dy, a.type) || (uintptr_t)a.offsets % 8)
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    return SK_OK;
}

uint64_t sk_grouped_linear_workspace(const void* x, uint64_t ld_x, const void* weight, uint64_t ld_weight, uint64_t stride_weight, uint64_t rows,
                                     uint64_t groups, uint64_t width, uint64_t out, const void* y, uint64_t ld_y) {
    GroupedArgs a{};
    a.x = x; a.ld_x = ld_x; a.weight = weight; a.ld_weight = ld_weight; a.stride_weight = stride_weight;
    a.rows = rows; a.groups = groups; a.width = width; a.out = out;
    a.y = const_cast<void*>(y); a.ld_y = ld_y;
    return rows && groups && width && out ? grouped_workspace(a, false) : 0;
}

int sk_grouped_linear(const void* x, uint64_t ld_x, const void* weight, uint64_t ld_weight, uint64_t stride_weight, int type, uint64_t rows, uint64_t groups,
                      uint64_t width, uint64_t out, const int64_t* offsets, void* y, uint64_t ld_y, int fill, void* workspace, uint64_t workspace_bytes,
                      void* stream) {
    const char* who = "sk_grouped_linear";
    GroupedArgs a{};
    a.x = x; a.ld_x = ld_x; a.weight = weight; a.ld_weight = ld_weight; a.stride_weight = stride_weight;
    a.type = type; a.rows = rows; a.groups = groups; a.width = width; a.out = out; a.offsets = offsets; a.fill = fill;
    a.y = y; a.ld_y = ld_y; a.workspace = workspace;
    if (int rc = grouped_checked(who, a, false)) return rc;
    if (!rows) return SK_OK;
    if (!y) return set_error(SK_EINVAL, "%s: null argument", who);
    if (ld_y < out) return set_error(SK_EINVAL, "%s: a leading dimension is below the rows' length", who);
    if (misaligned(y, type)) return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (y == x || y == weight) return set_error(SK_EINVAL, "%s: the product cannot be written in place", who);
    if (int rc = check_workspace(who, workspace, workspace_bytes, grouped_workspace(a, false))) return rc;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    a.withhold_ms = take_withhold_ms();
    return launch_grouped(a, dev, (cudaStream_t)stream);
}

uint64_t sk_grouped_linear_backward_workspace(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_weight,
                                              uint64_t stride_weight, uint64_t rows, uint64_t groups, uint64_t width, uint64_t out, const void* dx,
                                              uint64_t ld_dx, const void* dweight, uint64_t ld_dweight, uint64_t stride_dweight, int dweight_type) {
    GroupedArgs a{};
    a.dy = dy; a.ld_dy = ld_dy; a.x = x; a.ld_x = ld_x; a.weight = weight; a.ld_weight = ld_weight; a.stride_weight = stride_weight;
    a.rows = rows; a.groups = groups; a.width = width; a.out = out;
    a.dx = const_cast<void*>(dx); a.ld_dx = ld_dx;
    a.dweight = const_cast<void*>(dweight); a.ld_dweight = ld_dweight; a.stride_dweight = stride_dweight; a.dweight_type = dweight_type;
    return rows && groups && width && out && type_ok(dweight_type) ? grouped_workspace(a, true) : 0;
}

int sk_grouped_linear_backward(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* weight, uint64_t ld_weight, uint64_t stride_weight,
                               int type, uint64_t rows, uint64_t groups, uint64_t width, uint64_t out, const int64_t* offsets, void* dx, uint64_t ld_dx,
                               int fill, void* dweight, uint64_t ld_dweight, uint64_t stride_dweight, int dweight_type, void* workspace,
                               uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_grouped_linear_backward";
    GroupedArgs a{};
    a.dy = dy; a.ld_dy = ld_dy; a.x = x; a.ld_x = ld_x; a.weight = weight; a.ld_weight = ld_weight; a.stride_weight = stride_weight;
    a.type = type; a.rows = rows; a.groups = groups; a.width = width; a.out = out; a.offsets = offsets; a.fill = fill;
    a.dx = dx; a.ld_dx = ld_dx; a.dweight = dweight; a.ld_dweight = ld_dweight; a.stride_dweight = stride_dweight; a.dweight_type = dweight_type;
    a.workspace = workspace;
    if (int rc = grouped_checked(who, a, true)) return rc;
    if (dweight && dweight_type != type && dweight_type != SK_F32) return set_error(SK_EINVAL, "%s: dweight's type must be the inputs' or SK_F32", who);
    if ((dx && ld_dx < width) || (dweight && ld_dweight < width)) return set_error(SK_EINVAL, "%s: a leading dimension is below the rows' length", who);
    if (dweight && groups > 1 && stride_dweight < (out - 1) * ld_dweight + width) return set_error(SK_EINVAL, "%s: the matrices of an output overlap", who);
    if (misaligned(dx, type) || (dweight && misaligned(dweight, dweight_type))) return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (!rows) {                                  // sums over no rows
        const uint64_t size = dweight ? type_size(dweight_type) : 0;
        const bool together = groups == 1 || stride_dweight == out * ld_dweight;
        for (uint64_t g = 0; dweight && g < (together ? 1 : groups); ++g)
            SK_OP_CUDA(cudaMemset2DAsync((uint8_t*)dweight + g * stride_dweight * size, ld_dweight * size, 0, width * size, together ? groups * out : out,
                                         (cudaStream_t)stream));
        return SK_OK;
    }
    if (!dx && !dweight) return SK_OK;
    if ((dx && (dx == dy || dx == x || dx == weight)) || (dweight && (dweight == dy || dweight == x || dweight == weight)))
        return set_error(SK_EINVAL, "%s: the gradients cannot be written in place", who);
    if (int rc = check_workspace(who, workspace, workspace_bytes, grouped_workspace(a, true))) return rc;
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    a.withhold_ms = take_withhold_ms();
    return launch_grouped_backward(a, dev, (cudaStream_t)stream);
}

uint64_t sk_sort_by_expert_workspace(uint64_t n, uint64_t groups) {
    OpDevice dev;
    if (!n || n >= kMaxExtent || groups < 1 || groups > kMaxGroups || op_device(&dev)) return 0;
    return sort_workspace(n, (uint32_t)groups, dev.sm_count);
}

int sk_sort_by_expert(const void* experts, int expert_bits, uint64_t n, uint64_t groups, int64_t* order, int64_t* places, int64_t* offsets, void* workspace,
                      uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_sort_by_expert";
    if (expert_bits != 32 && expert_bits != 64) return set_error(SK_EINVAL, "%s: expert_bits must be 32 or 64", who);
    if (groups < 1 || groups > kMaxGroups) return set_error(SK_EINVAL, "%s: groups must be in 1..%u", who, kMaxGroups);
    if (n >= kMaxExtent) return set_error(SK_EINVAL, "%s: n must be below 2^31", who);
    if (!offsets || (n && !experts)) return set_error(SK_EINVAL, "%s: null argument", who);
    if ((uintptr_t)experts % (expert_bits / 8) || (uintptr_t)order % 8 || (uintptr_t)places % 8 || (uintptr_t)offsets % 8)
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    if (n && (order == experts || places == experts || offsets == experts)) return set_error(SK_EINVAL, "%s: the experts cannot be sorted in place", who);
    if (!n) {
        SK_OP_CUDA(cudaMemsetAsync(offsets, 0, (groups + 1) * 8, (cudaStream_t)stream));
        return SK_OK;
    }
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    if (int rc = check_workspace(who, workspace, workspace_bytes, sort_workspace(n, (uint32_t)groups, dev.sm_count))) return rc;
    return launch_sort({experts, n, (uint32_t)groups, expert_bits == 64, order, places, offsets, (uint32_t*)workspace}, dev.sm_count, (cudaStream_t)stream);
}

int sk_dropout(const void* x, uint64_t ld_x, const void* residual, uint64_t ld_residual, void* y, uint64_t ld_y, int type, uint64_t rows, uint64_t cols,
               double p, uint64_t seed, const uint64_t* seed_at, void* stream) {
    const char* who = "sk_dropout";
    if (!type_ok(type)) return set_error(SK_EINVAL, "%s: unknown type", who);
    if (!(p >= 0.0 && p <= 1.0)) return set_error(SK_EINVAL, "%s: p must be in 0..1", who);
    if (cols >= (1ull << 40) || rows >= (1ull << 40) || rows * (cols >> 20) >= (1ull << 30)) return set_error(SK_EINVAL, "%s: too many values", who);
    if (!rows || !cols) return SK_OK;
    if (!x || !y) return set_error(SK_EINVAL, "%s: null argument", who);
    if (ld_x < cols || ld_y < cols || (residual && ld_residual < cols)) return set_error(SK_EINVAL, "%s: a leading dimension is below cols", who);
    if (rows > 1 && ((y == x && ld_y != ld_x) || (y == residual && ld_y != ld_residual)))
        return set_error(SK_EINVAL, "%s: in place, the leading dimensions must be the same", who);
    if (misaligned(x, type) || misaligned(residual, type) || misaligned(y, type) || (uintptr_t)seed_at % 8)
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    OpDevice dev;
    if (int rc = op_device(&dev)) return rc;
    const uint32_t below = (uint32_t)std::nearbyint(p * 65536.0);
    const float scale = below < 65536 ? (float)(65536.0 / (65536.0 - below)) : 0.0f;
    return launch_dropout({x, residual, y, rows, cols, ld_x, ld_residual, ld_y, type, seed, seed_at, below, scale}, dev.sm_count, (cudaStream_t)stream);
}

static int policy_checked(const char* who, const PolicyArgs& a, double clip_low, double clip_high) {
    if (a.tokens >= (1ull << 40) || a.sequences < 1 || a.sequences >= kMaxExtent) return set_error(SK_EINVAL, "%s: tokens must be below 2^40, sequences in 1..2^31-1", who);
    if (!a.offsets && a.sequences != 1) return set_error(SK_EINVAL, "%s: without offsets there is one sequence", who);
    if (!(clip_low >= 0 && clip_low <= 1) || !(clip_high >= 0)) return set_error(SK_EINVAL, "%s: clip_low must be in 0..1, clip_high not negative", who);
    if (!std::isfinite(a.kl)) return set_error(SK_EINVAL, "%s: kl must be finite", who);
    if (a.tokens && (!a.nll || !a.old_nll || !a.advantages)) return set_error(SK_EINVAL, "%s: null argument", who);
    if (a.kl != 0 && !a.reference && a.tokens) return set_error(SK_EINVAL, "%s: kl needs reference_nll", who);
    if (misaligned(a.nll, SK_F32) || misaligned(a.old_nll, SK_F32) || misaligned(a.advantages, SK_F32) || misaligned(a.reference, SK_F32) ||
        misaligned(a.result, SK_F32) || misaligned(a.norm, SK_F32) || misaligned(a.dloss, SK_F32) || misaligned(a.dnll, SK_F32) ||
        (uintptr_t)a.targets % 8 || (uintptr_t)a.offsets % 8)
        return set_error(SK_EINVAL, "%s: a pointer is not aligned to its element", who);
    return SK_OK;
}

uint64_t sk_policy_loss_workspace(uint64_t tokens, uint64_t sequences) {
    return tokens && tokens < (1ull << 40) && sequences < kMaxExtent ? policy_workspace(tokens, sequences) : 0;
}

static PolicyArgs policy_args(const float* nll, const float* old_nll, const float* advantages, int advantage_of_sequences, const int64_t* targets,
                              const int64_t* offsets, uint64_t sequences, const float* reference_nll, uint64_t tokens, double clip_low, double clip_high,
                              double kl) {
    PolicyArgs a{};
    a.nll = nll; a.old_nll = old_nll; a.advantages = advantages; a.advantage_of_sequences = advantage_of_sequences;
    a.targets = targets; a.offsets = offsets; a.sequences = sequences; a.reference = reference_nll; a.tokens = tokens;
    a.log_low = std::log1p(-clip_low); a.log_high = std::log1p(clip_high);
    a.border_low = (float)a.log_low; a.border_high = (float)a.log_high;
    a.low = (float)(1.0 - clip_low); a.high = (float)(1.0 + clip_high); a.kl = (float)kl;
    return a;
}

int sk_policy_loss(const float* nll, const float* old_nll, const float* advantages, int advantage_of_sequences, const int64_t* targets,
                   const int64_t* offsets, uint64_t sequences, const float* reference_nll, uint64_t tokens, double clip_low, double clip_high, double kl,
                   int average_sequences, float* result, float* norm, void* workspace, uint64_t workspace_bytes, void* stream) {
    const char* who = "sk_policy_loss";
    PolicyArgs a = policy_args(nll, old_nll, advantages, advantage_of_sequences, targets, offsets, sequences, reference_nll, tokens, clip_low, clip_high, kl);
    a.average_sequences = average_sequences; a.result = result; a.norm = norm; a.workspace = (float4*)workspace;
    if (int rc = policy_checked(who, a, clip_low, clip_high)) return rc;
    if (!result || !norm) return set_error(SK_EINVAL, "%s: null argument", who);
    if (!tokens) {
        SK_OP_CUDA(cudaMemsetAsync(result, 0, 12, (cudaStream_t)stream));
        SK_OP_CUDA(cudaMemsetAsync(norm, 0, sequences * 4, (cudaStream_t)stream));
        return SK_OK;
    }
    if (int rc = check_workspace(who, workspace, workspace_bytes, policy_workspace(tokens, sequences))) return rc;
    return launch_policy(a, (cudaStream_t)stream);
}

int sk_policy_loss_backward(const float* dloss, const float* nll, const float* old_nll, const float* advantages, int advantage_of_sequences,
                            const int64_t* targets, const int64_t* offsets, uint64_t sequences, const float* reference_nll, uint64_t tokens,
                            double clip_low, double clip_high, double kl, const float* norm, float* dnll, void* stream) {
    const char* who = "sk_policy_loss_backward";
    PolicyArgs a = policy_args(nll, old_nll, advantages, advantage_of_sequences, targets, offsets, sequences, reference_nll, tokens, clip_low, clip_high, kl);
    a.dloss = dloss; a.norm = const_cast<float*>(norm); a.dnll = dnll;
    if (int rc = policy_checked(who, a, clip_low, clip_high)) return rc;
    if (!tokens) return SK_OK;
    if (!norm || !dnll) return set_error(SK_EINVAL, "%s: null argument", who);
    if (dnll == norm || dnll == dloss || (advantage_of_sequences && dnll == advantages))         // read by other tokens' threads too
        return set_error(SK_EINVAL, "%s: the gradient can be written over what has one value a token only", who);
    return launch_policy_backward(a, (cudaStream_t)stream);
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
