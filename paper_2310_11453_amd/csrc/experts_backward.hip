// Straight-through backward of the products of a mixture of BitLinear layers (arXiv 2310.11453, Section 2.2):
//   dXs[s,k]  = beta_e sum_n dY[s,n] S_e[n,k]             for the slots s of expert e
//   dW_e[n,k] = sum_{s of e} dY[s,n] q[r,k] gamma_r/128    r the row that s reads; zeros where e has no slots
// dY is bf16.
#include "common.h"
#include "experts.h"

namespace bl {

__device__ inline float bf16_value(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// the sign of weight (n, k) of a blob
__device__ inline float sign_at(const uint32_t* blob, int64_t TK, int64_t n, int64_t k) {
    const int kl = (int)(k & (kChunkK - 1));
    const int i = kl >> 6, g = (kl & 63) >> 4, d = (kl & 15) >> 2, j = kl & 3;
    const uint32_t w = blob[tile_dword_offset(n >> 4, k >> 9, TK) + (g * 16 + (n & 15)) * 4 + d];
    return (w >> (8 * j + i)) & 1 ? 1.f : -1.f;
}

// 64 x 64 outputs a workgroup, 4 x 4 a thread, 16 reduction elements at a time through LDS
__global__ __launch_bounds__(256) void experts_dx_kernel(ExpertsArgs a, int64_t blob) {
    __shared__ float A[16][65], B[16][65];
    const int T = (int)a.T, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t k0 = (int64_t)blockIdx.x * 64, TK = tiles_k(a.K);
    for (int e = 0; e < a.E; ++e) {
        const int s0 = slot_bound(a.offsets, e, T), s1 = slot_bound(a.offsets, e + 1, T);
        for (int m0 = s0 + (int)blockIdx.y * 64; m0 < s1; m0 += (int)gridDim.y * 64) {
            float acc[4][4] = {};
            for (int64_t n0 = 0; n0 < a.N; n0 += 16) {
                __syncthreads();
                for (int i = threadIdx.x; i < 16 * 64; i += 256) {
                    const int r = i & 15, c = i >> 4, cc = i & 63, rr = i >> 6;
                    A[r][c] = m0 + c < s1 && n0 + r < a.N ? bf16_value(a.dY[(int64_t)(m0 + c) * a.N + n0 + r]) : 0.f;
                    B[rr][cc] = n0 + rr < a.N && k0 + cc < a.K ? sign_at(a.packed + e * blob, TK, n0 + rr, k0 + cc) : 0.f;
                }
                __syncthreads();
                for (int r = 0; r < 16; ++r)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int x = 0; x < 4; ++x) acc[y][x] += A[r][ty + 16 * y] * B[r][tx + 16 * x];
            }
            const float beta = a.beta[e];
            for (int y = 0; y < 4; ++y)
                for (int x = 0; x < 4; ++x) {
                    const int64_t m = m0 + ty + 16 * y, k = k0 + tx + 16 * x;
                    if (m < s1 && k < a.K) a.dX[m * a.K + k] = beta * acc[y][x];
                }
        }
    }
}

__global__ __launch_bounds__(256) void experts_dw_kernel(ExpertsArgs a) {
    __shared__ float A[16][65], B[16][65];
    const int T = (int)a.T, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t k0 = (int64_t)blockIdx.x * 64, n0 = (int64_t)blockIdx.y * 64;
    for (int e = (int)blockIdx.z; e < a.E; e += (int)gridDim.z) {
        const int s0 = slot_bound(a.offsets, e, T), s1 = slot_bound(a.offsets, e + 1, T);
        float acc[4][4] = {};
        for (int m0 = s0; m0 < s1; m0 += 16) {
            __syncthreads();
            for (int i = threadIdx.x; i < 16 * 64; i += 256) {
                const int c = i & 63, m = m0 + (i >> 6);
                const bool in = m < s1;
                const int64_t r = code_row(a.order, (uint32_t)a.top_k, (uint32_t)a.rows, (uint32_t)(in ? m : s0));
                const float g = in && n0 + c < a.N ? bf16_value(a.dY[(int64_t)m * a.N + n0 + c]) : 0.f;
                A[i >> 6][c] = a.per_tensor ? g : g * (a.gamma[r] / 128.f);
                B[i >> 6][c] = in && k0 + c < a.K ? (float)a.codes[r * a.K + k0 + c] : 0.f;
            }
            __syncthreads();
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int y = 0; y < 4; ++y)
#pragma unroll
                    for (int x = 0; x < 4; ++x) acc[y][x] += A[r][ty + 16 * y] * B[r][tx + 16 * x];
        }
        const float scale = a.per_tensor ? *a.gamma / 128.f : 1.f;
        for (int y = 0; y < 4; ++y)
            for (int x = 0; x < 4; ++x) {
                const int64_t n = n0 + ty + 16 * y, k = k0 + tx + 16 * x;
                if (n < a.N && k < a.K) a.dW[((int64_t)e * a.N + n) * a.K + k] = scale * acc[y][x];
            }
    }
}

size_t experts_backward_bytes(int64_t, int64_t, int64_t, int) { return 256; }

hipError_t launch_experts_backward(const ExpertsArgs& a, hipStream_t s) {
    const unsigned kt = (unsigned)((a.K + 63) / 64);
    if (a.dX) {
        const int64_t mt = (a.T + 63) / 64;
        experts_dx_kernel<<<dim3(kt, (unsigned)(mt < 65535 ? mt : 65535)), 256, 0, s>>>(a, tiles_n(a.N) * tiles_k(a.K) * 256);
    }
    if (a.dW) experts_dw_kernel<<<dim3(kt, (unsigned)((a.N + 63) / 64), (unsigned)a.E), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace bl
