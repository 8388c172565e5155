// C ABI of the operators around an 8-bit linear layer: argument checks on the host, then launches.
// Declarations and argument semantics: include/bitlinear.h.
#include <math.h>

#include "../../include/bitlinear.h"
#include "common.h"
#include "i8.h"
#include "kernels.h"

using namespace bl;

static_assert((int)kF32 == BL_F32 && (int)kBF16 == BL_BF16 && (int)kI8 == BL_I8, "element types");

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30;
constexpr int64_t kMaxElements = (int64_t)1 << 40;

inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
int check_hip(hipError_t e) { return e == hipSuccess ? BL_OK : BL_ERR_HIP; }
bool gran_ok(int g) { return g == BL_GAMMA_PER_TOKEN || g == BL_GAMMA_PER_TENSOR; }
bool float_ok(int type) { return type == BL_F32 || type == BL_BF16; }
bool rows_ok(int64_t M, int64_t K) {
    return M >= 0 && M <= kMaxDim && K > 0 && K <= kMaxDim && K % 32 == 0 && M * K <= kMaxElements;
}
bool weights_ok(int64_t N, int64_t K) {
    return N > 0 && K > 0 && N <= kMaxDim && K <= kMaxDim && K % 32 == 0 && N * K <= kMaxElements;
}
bool eps_ok(float eps) { return eps >= 0.f && eps < INFINITY; }
// operands read 4, 8 or 16 bytes at a time: an address that allows it
template <class... P>
bool aligned16(const P*... p) {
    return ((... | (uintptr_t)p) & 15) == 0;
}

// per tensor: 1/rms of each row, and the largest magnitudes
struct RmsWs {
    size_t most, total;
};
RmsWs rms_ws(int64_t M) {
    RmsWs w{};
    w.most = align256((size_t)M * 8);
    w.total = w.most + kRmsMostBytes + 256;
    return w;
}
size_t rms_backward_bytes(int64_t M, int64_t K) { return rms_backward_part_bytes(M, K) + 256; }
int product_status(int64_t M, int64_t N, int64_t K) {
    if (!rows_ok(M, K) || !weights_ok(N, K)) return BL_ERR_SHAPE;
    return K > kMaxGemmK ? BL_ERR_UNSUPPORTED : BL_OK;
}

}  // namespace

namespace bl {

// bitlinear_workspace_bytes of the operators here
size_t workspace_bytes_i8(int op, int64_t M, int64_t N, int64_t K, int granularity) {
    switch (op) {
        case BL_OP_QUANT_RMSNORM:
            return rows_ok(M, K) && granularity == BL_GAMMA_PER_TENSOR ? rms_ws(M).total : 0;
        case BL_OP_RMSNORM_BACKWARD:
            return rows_ok(M, K) ? rms_backward_bytes(M, K) : 0;
        case BL_OP_MATMUL_I8:
            return product_status(M, N, K) == BL_OK ? gemm_i8_part_bytes(M, N, K) : 0;
        case BL_OP_BACKWARD_I8:
            return product_status(M, N, K) == BL_OK ? backward_i8_bytes(M, N, K) + 256 : 0;
        default:
            return 0;
    }
}

}  // namespace bl

extern "C" {

int bitlinear_quant_rmsnorm(const void* X, int x_type, const void* residual, int h_type, int64_t M, int64_t K,
                            const float* gain, float eps, int granularity, void* H, int8_t* codes, float* gamma,
                            int32_t* rowsum, float* xhat_dump, void* workspace, size_t workspace_bytes, void* stream) {
    if (!rows_ok(M, K)) return BL_ERR_SHAPE;
    if (!gran_ok(granularity) || !float_ok(x_type) || !float_ok(h_type) || !eps_ok(eps)) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!X || !codes || !gamma) return BL_ERR_NULL;
    if (H && !residual) return BL_ERR_UNSUPPORTED;
    if (!aligned16((const char*)X, (const char*)residual, (const char*)H, (const char*)gain, (const char*)codes,
                   (const char*)xhat_dump))
        return BL_ERR_UNSUPPORTED;
    if (H && H == X && x_type != h_type) return BL_ERR_UNSUPPORTED;
    const bool per_tensor = granularity == BL_GAMMA_PER_TENSOR;
    const RmsWs ws = rms_ws(M);
    if (per_tensor && (!workspace || workspace_bytes < ws.total)) return BL_ERR_WORKSPACE;
    QuantRmsArgs a{};
    a.X = X; a.R = residual; a.H = H; a.x_bf16 = x_type == BL_BF16; a.h_bf16 = h_type == BL_BF16;
    a.M = M; a.K = K; a.gain = gain; a.eps = (double)eps; a.per_tensor = per_tensor;
    a.codes = codes; a.gamma = gamma; a.rowsum = rowsum; a.xhat = xhat_dump;
    if (per_tensor) {
        char* at = (char*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255);
        a.rstd = (double*)at;
        a.most = (int*)(at + ws.most);
    }
    return check_hip(launch_quant_rmsnorm(a, (hipStream_t)stream));
}

int bitlinear_rmsnorm_backward(const void* dXhat, int g_type, const void* H, int h_type, const void* dresidual,
                               int d_type, int64_t M, int64_t K, const float* gain, float eps, void* dH, float* dgain,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!rows_ok(M, K)) return BL_ERR_SHAPE;
    if (!float_ok(g_type) || !float_ok(h_type) || !float_ok(d_type) || !eps_ok(eps)) return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!dXhat || !H || !dH) return BL_ERR_NULL;
    if (!aligned16((const char*)dXhat, (const char*)H, (const char*)dresidual, (const char*)gain, (const char*)dH))
        return BL_ERR_UNSUPPORTED;
    if ((dH == dXhat && d_type != g_type) || (dH == H && d_type != h_type)) return BL_ERR_UNSUPPORTED;
    if (dgain && (!workspace || workspace_bytes < rms_backward_bytes(M, K))) return BL_ERR_WORKSPACE;
    RmsBackwardArgs a{};
    a.G = dXhat; a.H = H; a.dR = dresidual; a.dH = dH;
    a.g_bf16 = g_type == BL_BF16; a.h_bf16 = h_type == BL_BF16; a.d_bf16 = d_type == BL_BF16;
    a.M = M; a.K = K; a.gain = gain; a.eps = (double)eps; a.dgain = dgain;
    a.partials = dgain ? (void*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255) : nullptr;
    return check_hip(launch_rmsnorm_backward(a, (hipStream_t)stream));
}

size_t bitlinear_packed_bytes_i8(int64_t N, int64_t K) { return weights_ok(N, K) ? i8_blob_bytes(N, K) : 0; }

int bitlinear_pack_weights_i8(const void* W, int w_type, int64_t N, int64_t K, void* packed, float* scale, void* stream) {
    if (!weights_ok(N, K)) return BL_ERR_SHAPE;
    if (!float_ok(w_type) && w_type != BL_I8) return BL_ERR_UNSUPPORTED;
    if (!W || !packed || (!scale && w_type != BL_I8)) return BL_ERR_NULL;
    if (!aligned16((const char*)W, (const char*)packed)) return BL_ERR_UNSUPPORTED;
    return check_hip(launch_pack_i8({W, w_type, N, K, (uint8_t*)packed, scale}, (hipStream_t)stream));
}

int bitlinear_unpack_weights_i8(const void* packed, const float* scale, int64_t N, int64_t K, int type, void* out,
                                void* stream) {
    if (!weights_ok(N, K)) return BL_ERR_SHAPE;
    if (!float_ok(type) && type != BL_I8) return BL_ERR_UNSUPPORTED;
    if (!packed || !out || (!scale && type != BL_I8)) return BL_ERR_NULL;
    if (!aligned16((const char*)packed, (const char*)out)) return BL_ERR_UNSUPPORTED;
    return check_hip(launch_unpack_i8({(const uint8_t*)packed, scale, N, K, type, out}, (hipStream_t)stream));
}

int bitlinear_matmul_i8(const int8_t* codes, const float* gamma, int64_t M, int64_t K, const void* packed, int64_t N,
                        const float* scale, int granularity, unsigned flags, int y_type, void* Y, void* workspace,
                        size_t workspace_bytes, void* stream) {
    if (const int st = product_status(M, N, K)) return st;
    const bool out_acc = (flags & BL_FLAG_OUT_ACC_I32) != 0;
    if (!gran_ok(granularity) || (flags & ~BL_FLAG_OUT_ACC_I32) || !float_ok(y_type) || (out_acc && y_type != BL_F32))
        return BL_ERR_UNSUPPORTED;
    if (M == 0) return BL_OK;
    if (!codes || !packed || !Y || (!out_acc && (!gamma || !scale))) return BL_ERR_NULL;
    if (!aligned16((const char*)codes, (const char*)packed)) return BL_ERR_UNSUPPORTED;
    GemmI8Args a{};
    a.codes = codes; a.gamma = gamma; a.M = M; a.K = K; a.N = N; a.packed = (const uint8_t*)packed; a.scale = scale;
    a.per_tensor = granularity == BL_GAMMA_PER_TENSOR; a.out_acc = out_acc; a.y_bf16 = y_type == BL_BF16; a.Y = Y;
    if (workspace) {
        a.part = (int32_t*)(((uintptr_t)workspace + 15) & ~(uintptr_t)15);
        const size_t lost = (uintptr_t)a.part - (uintptr_t)workspace;
        a.part_bytes = workspace_bytes > lost ? workspace_bytes - lost : 0;
    }
    return check_hip(launch_gemm_i8(a, (hipStream_t)stream));
}

int bitlinear_backward_ste_i8(const void* dY, int dy_type, int64_t M, int64_t N, int64_t K, const int8_t* codes,
                              const float* gamma, int granularity, const void* packed, const float* scale, void* dX,
                              int dx_type, float* dW, void* workspace, size_t workspace_bytes, void* stream) {
    if (const int st = product_status(M, N, K)) return st;
    if (!gran_ok(granularity) || !float_ok(dy_type) || !float_ok(dx_type)) return BL_ERR_UNSUPPORTED;
    if (M == 0 || (!dX && !dW)) return BL_OK;
    if (!dY || (dX && (!packed || !scale)) || (dW && (!codes || !gamma))) return BL_ERR_NULL;
    if (!aligned16((const char*)dY, dX ? (const char*)packed : nullptr, dW ? (const char*)codes : nullptr, (const char*)dX))
        return BL_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < backward_i8_min_bytes(M, N, K) + 256) return BL_ERR_WORKSPACE;
    BackwardI8Args a{};
    a.dY = dY; a.dy_bf16 = dy_type == BL_BF16; a.dx_bf16 = dx_type == BL_BF16; a.M = M; a.N = N; a.K = K;
    a.codes = codes; a.gamma = gamma; a.per_tensor = granularity == BL_GAMMA_PER_TENSOR;
    a.packed = (const uint8_t*)packed; a.scale = scale; a.dX = dX; a.dW = dW;
    a.workspace = (void*)(((uintptr_t)workspace + 255) & ~(uintptr_t)255);
    a.workspace_bytes = workspace_bytes - ((uintptr_t)a.workspace - (uintptr_t)workspace);
    return check_hip(launch_backward_i8(a, (hipStream_t)stream));
}

}  // extern "C"
