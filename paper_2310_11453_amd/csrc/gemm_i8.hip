// int8 x int8 product with scales for each token and channel:
//   acc[m][n] = sum_k q[m][k] * w[n][k]  (int32, at most 2^14 K <= 2^30),   Y[m][n] = float(acc) * (scale_n * (gamma_m / 128))
#include "common.h"
#include "i8.h"

namespace bl {

// A wave takes 16 rows of weights and 16 tokens; both operands come from memory as the MFMA wants them.
__global__ __launch_bounds__(256) void gemm_i8_plain(GemmI8Args a, int64_t items, int64_t tn) {
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave, c = l & 15, g = l >> 4;
    const int64_t TK = i8_tiles_k(a.K);
    for (int64_t it = (int64_t)blockIdx.x * 4 + w; it < items; it += (int64_t)gridDim.x * 4) {
        const int64_t tile = it % tn, m0 = it / tn * 16;
        const int64_t m = m0 + c < a.M ? m0 + c : a.M - 1;
        const v4i* wt = reinterpret_cast<const v4i*>(a.packed + tile * TK * 1024) + l;
        const int8_t* q = a.codes + m * a.K;
        v4i acc = {0, 0, 0, 0};
        for (int64_t t = 0; t < TK; ++t) {
            int64_t k = t * 64 + 16 * g;
            if (k >= a.K) k = 0;  // the weights there are zeros
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wt[t * 64], *reinterpret_cast<const v4i*>(q + k), acc, 0, 0, 0);
        }
        if (m0 + c >= a.M) continue;
        const float gm = a.out_acc ? 0.f : (a.per_tensor ? *a.gamma : a.gamma[m]) * (1.0f / 128.0f);  // (null with out_acc)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = tile * 16 + 4 * g + r;
            if (n >= a.N) continue;
            const int64_t at = m * a.N + n;
            if (a.out_acc) {
                static_cast<int32_t*>(a.Y)[at] = acc[r];
            } else {
                const float y = (float)acc[r] * (a.scale[n] * gm);
                if (a.y_bf16) static_cast<uint16_t*>(a.Y)[at] = (uint16_t)bf16_pair(y, 0.f);
                else static_cast<float*>(a.Y)[at] = y;
            }
        }
    }
}

size_t gemm_i8_part_bytes(int64_t M, int64_t N, int64_t K) {
    (void)M, (void)N, (void)K;
    return 0;
}
hipError_t launch_gemm_i8(const GemmI8Args& a, hipStream_t s) {
    const int64_t tn = tiles_n(a.N), items = tn * ((a.M + 15) / 16), wgs = (items + 3) / 4;
    gemm_i8_plain<<<(unsigned)(wgs < (1 << 20) ? wgs : (1 << 20)), 256, 0, s>>>(a, items, tn);
    return hipGetLastError();
}

}  // namespace bl
