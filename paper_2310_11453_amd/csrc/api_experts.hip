// C ABI of the operators of a mixture of BitLinear layers: argument checks on the host, then launches.
// Declarations and argument semantics: include/bitlinear.h.
#include <algorithm>

#include "../../include/bitlinear.h"
#include "common.h"
#include "experts.h"
#include "kernels.h"

using namespace bl;

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30;
constexpr int kMaxTopK = 64;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
int check_hip(hipError_t e) { return e == hipSuccess ? BL_OK : BL_ERR_HIP; }
bool gran_ok(int g) { return g == BL_GAMMA_PER_TOKEN || g == BL_GAMMA_PER_TENSOR; }
bool weights_ok(int64_t N, int64_t K) {
    return N > 0 && K > 0 && N <= kMaxDim && K <= kMaxDim && K % 32 == 0 && N * K <= ((int64_t)1 << 40);
}
bool tokens_ok(int64_t M, int top_k) {
    return M >= 0 && M <= kMaxDim && top_k >= 1 && top_k <= kMaxTopK && M * top_k <= kMaxDim;
}
// operands read 4, 8 or 16 bytes at a time: an address that allows it
template <class... P>
bool aligned16(const P*... p) {
    return ((... | (uintptr_t)p) & 15) == 0;
}
bool experts_ok(int experts) { return experts >= 1 && experts <= kMaxExperts; }

size_t route_bytes(int64_t T, int experts) {
    const int64_t blocks = route_blocks(T);
    return blocks > 1 ? align256((size_t)(blocks + 1) * experts * 4) : 0;
}

// what both products check and describe alike
int experts_status(int64_t M, int top_k, int64_t N, int64_t K, int experts, int granularity) {
    if (!tokens_ok(M, top_k) || !weights_ok(N, K) || !experts_ok(experts)) return BL_ERR_SHAPE;
    if (!gran_ok(granularity) || K > kMaxGemmK) return BL_ERR_UNSUPPORTED;
    return BL_OK;
}
ExpertsArgs experts_args(const int8_t* codes, const float* gamma, int64_t M, int top_k, int64_t N, int64_t K,
                         const int32_t* order, const int32_t* offsets, int experts, const void* packed,
                         const float* beta, int granularity) {
    ExpertsArgs a{};
    a.codes = codes; a.gamma = gamma; a.T = M * top_k; a.rows = order ? M : a.T; a.K = K; a.N = N;
    a.order = order; a.top_k = top_k; a.offsets = offsets; a.E = experts;
    a.packed = (const uint32_t*)packed; a.beta = beta;
    a.per_tensor = granularity == BL_GAMMA_PER_TENSOR;
    return a;
}

bool function_ok(int fn) { return (fn >= BL_FN_RELU && fn <= BL_FN_SILU) || fn == BL_FN_RELU_MARKED; }
// a workgroup's threads times the rows stay below 2^32, which is what a launch takes
bool nonlinear_rows_ok(int64_t M, int64_t K) { return M < ((int64_t)1 << 24) && M * K <= ((int64_t)1 << 36); }
struct NonlinearWs {
    size_t rowstats, gmax, total;
};
NonlinearWs nonlinear_ws(int64_t M) {
    NonlinearWs w{};
    w.gmax = align256((size_t)M * 16);
    w.total = w.gmax + 256;
    return w;
}

}  // namespace

extern "C" {

size_t bitlinear_workspace_bytes_experts(int op, int64_t M, int top_k, int64_t N, int64_t K, int experts,
                                         int granularity) {
    if (!tokens_ok(M, top_k) || !gran_ok(granularity)) return 0;
    switch (op) {
        case BL_OP_ROUTE:
            return experts_ok(experts) && M * top_k <= kMaxRouteSlots ? route_bytes(M * top_k, experts) : 0;
        case BL_OP_QUANT_NONLINEAR:
            return granularity == BL_GAMMA_PER_TENSOR && nonlinear_rows_ok(M * top_k, 0)
                       ? nonlinear_ws(M * top_k).total : 0;
        case BL_OP_BACKWARD:
            if (experts_status(M, top_k, N, K, experts, granularity) != BL_OK) return 0;
            return experts_backward_bytes(M * top_k, N, K, experts, granularity == BL_GAMMA_PER_TENSOR) + 256;
        default:
            return 0;
    }
}

int bitlinear_route(const int32_t* expert, int64_t M, int top_k, int experts, int32_t* order, int32_t* position,
                    int32_t* offsets, void* workspace, size_t workspace_bytes, void* stream) {
    if (!tokens_ok(M, top_k) || !experts_ok(experts)) return BL_ERR_SHAPE;
    if (M * top_k > kMaxRouteSlots) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!expert || !order || !position || !offsets) return BL_ERR_NULL;
    const size_t need = route_bytes(M * top_k, experts);
    if (need && (!workspace || workspace_bytes < need)) return BL_ERR_WORKSPACE;
    RouteArgs a{expert, (uint32_t)(M * top_k), (uint32_t)experts, order, position, offsets, (uint32_t*)workspace};
    return check_hip(launch_route(a, (hipStream_t)stream));
}

int bitlinear_matmul_experts(const int8_t* codes, const float* gamma, const int32_t* rowsum, int64_t M, int top_k,
                             int64_t K, const int32_t* order, const int32_t* offsets, int experts, const void* packed,
                             int64_t N, const float* beta, int granularity, unsigned flags, float* Y, void* stream) {
    if (const int st = experts_status(M, top_k, N, K, experts, granularity)) return st;
    if (flags & ~BL_FLAG_OUT_ACC_I32) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!codes || !gamma || !rowsum || !offsets || !packed || !beta || !Y) return BL_ERR_NULL;
    if (!aligned16(codes, (const char*)packed)) return BL_ERR_UNSUPPORTED;
    ExpertsArgs a = experts_args(codes, gamma, M, top_k, N, K, order, offsets, experts, packed, beta, granularity);
    a.rowsum = rowsum;
    a.out_acc = (flags & BL_FLAG_OUT_ACC_I32) != 0;
    a.Y = Y;
    return check_hip(launch_matmul_experts(a, (hipStream_t)stream));
}

int bitlinear_backward_ste_experts(const void* dY, int64_t M, int top_k, int64_t N, int64_t K, const int8_t* codes,
                                   const float* gamma, int granularity, const int32_t* order, const int32_t* offsets,
                                   int experts, const void* packed, const float* beta, float* dX, float* dW,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if (const int st = experts_status(M, top_k, N, K, experts, granularity)) return st;
    if (M == 0 || (!dX && !dW)) return BL_OK;
    if (!dY || !gamma || !offsets) return BL_ERR_NULL;
    if (dX && (!packed || !beta)) return BL_ERR_NULL;
    if (dW && !codes) return BL_ERR_NULL;
    if ((experts_dy_direct(N) && !aligned16((const char*)dY)) || (dX && !aligned16((const char*)packed)) ||
        (dW && !aligned16(codes)))
        return BL_ERR_UNSUPPORTED;
    const bool per_tensor = granularity == BL_GAMMA_PER_TENSOR;
    if (!workspace || workspace_bytes < experts_backward_bytes(M * top_k, N, K, experts, per_tensor) + 256)
        return BL_ERR_WORKSPACE;
    ExpertsArgs a = experts_args(codes, gamma, M, top_k, N, K, order, offsets, experts, packed, beta, granularity);
    a.dY = (const uint16_t*)dY; a.dX = dX; a.dW = dW;
    a.workspace = (void*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255);
    a.workspace_bytes = workspace_bytes - ((uintptr_t)a.workspace - (uintptr_t)workspace);
    return check_hip(launch_experts_backward(a, (hipStream_t)stream));
}

int bitlinear_combine(const float* slots, const int32_t* position, const float* weights, int64_t M, int top_k,
                      int64_t N, float* Y, void* stream) {
    if (!tokens_ok(M, top_k) || N <= 0 || N > kMaxDim) return BL_ERR_SHAPE;
    if (M == 0) return BL_OK;
    if (!slots || !position || !Y) return BL_ERR_NULL;
    CombineArgs a{};
    a.slots = slots; a.position = position; a.weights = weights; a.M = M; a.N = N; a.T = M * top_k; a.top_k = top_k;
    a.Y = Y;
    return check_hip(launch_combine(a, (hipStream_t)stream));
}

int bitlinear_combine_backward(const float* dY, const float* slots, const int32_t* position, const float* weights,
                               int64_t M, int top_k, int64_t N, void* dslots, float* dweights, void* stream) {
    if (!tokens_ok(M, top_k) || N <= 0 || N > kMaxDim) return BL_ERR_SHAPE;
    if (M == 0) return BL_OK;
    if (!dY || !position || !dslots || (dweights && !slots)) return BL_ERR_NULL;
    CombineArgs a{};
    a.slots = slots; a.position = position; a.weights = weights; a.M = M; a.N = N; a.T = M * top_k; a.top_k = top_k;
    a.dY = dY; a.dSlots = (uint16_t*)dslots; a.dWeights = dweights;
    return check_hip(launch_combine_backward(a, (hipStream_t)stream));
}

int bitlinear_quant_nonlinear(const float* U, int64_t M, int64_t K, int fn, float ln_eps, const int32_t* rows,
                              int granularity, int8_t* codes, float* gamma, int32_t* rowsum, int8_t* check,
                              float* check_scale, void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || M > kMaxDim || K <= 0 || K > kMaxDim || K % 32) return BL_ERR_SHAPE;
    if (!gran_ok(granularity) || !function_ok(fn) || K > kMaxNonlinearK) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!nonlinear_rows_ok(M, K)) return BL_ERR_UNSUPPORTED;
    if (!U || !codes || !gamma || (check && !check_scale)) return BL_ERR_NULL;
    const NonlinearWs ws = nonlinear_ws(M);
    const bool per_tensor = granularity == BL_GAMMA_PER_TENSOR;
    if (!aligned16(U, codes, check) || (per_tensor && !aligned16((const char*)workspace))) return BL_ERR_UNSUPPORTED;
    if (per_tensor && (!workspace || workspace_bytes < ws.total)) return BL_ERR_WORKSPACE;
    NonlinearArgs a{};
    a.U = U; a.M = M; a.K = K; a.eps = ln_eps; a.rows = rows; a.per_tensor = per_tensor;
    a.codes = codes; a.gamma = gamma; a.rowsum = rowsum; a.check = check; a.check_scale = check_scale;
    if (per_tensor) {
        a.rowstats = (double*)workspace;
        a.gmax_bits = (uint32_t*)((char*)workspace + ws.gmax);
    }
    return check_hip(launch_quant_nonlinear(a, fn, (hipStream_t)stream));
}

int bitlinear_nonlinear_backward(const float* dXhat, const int8_t* check, const float* check_scale, int64_t M,
                                 int64_t K, int fn, float ln_eps, const int32_t* rows, int type, void* dU,
                                 void* stream) {
    if (M < 0 || M > kMaxDim || K <= 0 || K > kMaxDim || K % 32) return BL_ERR_SHAPE;
    if (!function_ok(fn) || (type != BL_F32 && type != BL_BF16) || K > kMaxNonlinearK) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!nonlinear_rows_ok(M, K)) return BL_ERR_UNSUPPORTED;
    if (!dXhat || !check || !check_scale || !dU) return BL_ERR_NULL;
    if (!aligned16(dXhat, check, (const char*)dU)) return BL_ERR_UNSUPPORTED;
    NonlinearArgs a{};
    a.dXhat = dXhat; a.check = const_cast<int8_t*>(check); a.check_scale = const_cast<float*>(check_scale);
    a.M = M; a.K = K; a.eps = ln_eps; a.rows = rows; a.dU = dU; a.bf16 = type == BL_BF16;
    return check_hip(launch_nonlinear_backward(a, fn, (hipStream_t)stream));
}

}  // extern "C"
