// Straight-through backward of the 8-bit product (rounding is identity, the scales are constants):
//   dX[M,K] = (dY * scale) W            dW[N,K] = dY^T (q * gamma / 128)
// on the bf16 product of backward.hip, C[I][J] = sum_r A[I][r] B[J][r]: int8 codes of either operand are exact in bf16, dY is
// rounded once, with the factor that belongs to the reduction index (scale_n for dX; gamma_m / 128 for dW where gamma is
// per token).  The operands are copied first into that product's layout (blocks of 32 reduction indices, padded with zeros):
//   g   [M][Np]  dY * scale       (A of dX)       wT [K][Np]  weights transposed  (B of dX)
//   gwT [N][Mp]  dY transposed    (A of dW)       qT [K][Mp]  codes transposed    (B of dW)
#include "common.h"
#include "i8.h"
#include "kernels.h"

namespace bl {

static inline int64_t pad32(int64_t v) { return (v + 31) / 32 * 32; }
// (row, r) of a copy with R rows
__device__ inline int64_t copy_offset(int64_t row, int64_t r, int64_t R) { return ((r >> 5) * R + row) * 32 + (r & 31); }
__device__ inline float element(const float* p, int64_t i) { return p[i]; }
__device__ inline float element(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ inline float element(const int8_t* p, int64_t i) { return (float)p[i]; }

// in[R][C] -> rows[R][Cp] = bf16(in * col_scale) and tr[C][Rp] = bf16(in * row_gamma / 128), either null: tiles of 64 x 64
template <typename IN>
__global__ __launch_bounds__(256) void copy_operand(const IN* __restrict__ in, int64_t R, int64_t C,
                                                    const float* __restrict__ col_scale,
                                                    const float* __restrict__ row_gamma, uint16_t* __restrict__ rows,
                                                    uint16_t* __restrict__ tr, int64_t tiles_c, int64_t items) {
    __shared__ uint16_t tile[64][66];
    const int64_t Cp = (C + 31) / 32 * 32, Rp = (R + 31) / 32 * 32;
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int64_t r0 = it / tiles_c * 64, c0 = it % tiles_c * 64;
        __syncthreads();
        for (int e = threadIdx.x; e < 64 * 64; e += 256) {
            const int64_t r = r0 + e / 64, c = c0 + e % 64;
            const float v = r < R && c < C ? element(in, r * C + c) : 0.f;
            if (rows && r < R && c < Cp)
                rows[copy_offset(r, c, R)] = (uint16_t)bf16_pair(col_scale && c < C ? v * col_scale[c] : v, 0.f);
            tile[e / 64][e % 64] = (uint16_t)bf16_pair(row_gamma && r < R ? v * (row_gamma[r] / 128.0f) : v, 0.f);
        }
        __syncthreads();
        if (!tr) continue;
        for (int e = threadIdx.x; e < 64 * 64; e += 256) {
            const int64_t c = c0 + e / 64, r = r0 + e % 64;
            if (c < C && r < Rp) tr[copy_offset(c, r, C)] = tile[e % 64][e / 64];
        }
    }
}
template <typename IN>
static void launch_copy(const IN* in, int64_t R, int64_t C, const float* col_scale, const float* row_gamma,
                        uint16_t* rows, uint16_t* tr, hipStream_t s) {
    const int64_t tc = (C + 63) / 64, items = tc * ((R + 63) / 64);
    copy_operand<IN><<<(unsigned)(items < (1 << 20) ? items : (1 << 20)), 256, 0, s>>>(in, R, C, col_scale, row_gamma, rows,
                                                                                   tr, tc, items);
}
// tiles of the blob -> wT[K][Np]: a workgroup takes 32 rows x 64 columns
__global__ __launch_bounds__(256) void copy_weights(const uint8_t* __restrict__ packed, int64_t N, int64_t K,
                                                    uint16_t* __restrict__ wT, int64_t items) {
    __shared__ uint8_t sm[2][1024];
    const int64_t TN = tiles_n(N), TK = i8_tiles_k(K);
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int64_t nb = it / TK, tk = it % TK;
        __syncthreads();
        for (int e = threadIdx.x; e < 512; e += 256) {
            const int t = e / 256;
            const uint32_t v = 2 * nb + t < TN
                ? reinterpret_cast<const uint32_t*>(packed + ((2 * nb + t) * TK + tk) * 1024)[e % 256] : 0u;
            reinterpret_cast<uint32_t*>(sm[t])[e % 256] = v;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 64 * 32; e += 256) {
            const int kl = e / 32, n = e % 32;
            const int64_t k = tk * 64 + kl;
            if (k >= K) continue;
            const int8_t v = (int8_t)sm[n / 16][(kl / 16) * 256 + (n % 16) * 16 + kl % 16];
            wT[copy_offset(k, nb * 32 + n, K)] = (uint16_t)bf16_pair((float)v, 0.f);
        }
    }
}
__global__ __launch_bounds__(256) void round_to_bf16(const float* __restrict__ in, uint16_t* __restrict__ out, int64_t n4) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (int64_t)gridDim.x * 256)
        store4(out, i, load4(in, i));
}

// Copies, each 256-byte aligned, then room for the fp32 sums of a bf16 dX, then (optional) for the products' slices.
struct BackwardI8Ws {
    size_t wT, gwT, qT, dx, total;
};
static BackwardI8Ws backward_i8_ws(int64_t M, int64_t N, int64_t K) {
    const int64_t Np = pad32(N), Mp = pad32(M);
    auto al = [](size_t v) { return (v + 255) & ~(size_t)255; };
    BackwardI8Ws w{};
    w.wT = al((size_t)M * Np * 2);
    w.gwT = w.wT + al((size_t)K * Np * 2);
    w.qT = w.gwT + al((size_t)N * Mp * 2);
    w.dx = w.qT + al((size_t)K * Mp * 2);
    w.total = w.dx + al((size_t)M * K * 4);
    return w;
}
size_t backward_i8_min_bytes(int64_t M, int64_t N, int64_t K) { return backward_i8_ws(M, N, K).total; }
size_t backward_i8_bytes(int64_t M, int64_t N, int64_t K) {
    const size_t dx = gemm_tn_slices_bytes(M, K, pad32(N)), dw = gemm_tn_slices_bytes(N, K, pad32(M));
    return backward_i8_ws(M, N, K).total + (dx > dw ? dx : dw);
}

hipError_t launch_backward_i8(const BackwardI8Args& a, hipStream_t s) {
    const int64_t M = a.M, N = a.N, K = a.K, Np = pad32(N), Mp = pad32(M);
    const BackwardI8Ws ws = backward_i8_ws(M, N, K);
    char* base = (char*)a.workspace;
    uint16_t *g = (uint16_t*)base, *wT = (uint16_t*)(base + ws.wT), *gwT = (uint16_t*)(base + ws.gwT),
             *qT = (uint16_t*)(base + ws.qT);
    float* part = (float*)(base + ws.total);
    const size_t part_bytes = a.workspace_bytes > ws.total ? a.workspace_bytes - ws.total : 0;
    uint16_t *rows = a.dX ? g : nullptr, *tr = a.dW ? gwT : nullptr;
    const float* row_gamma = a.per_tensor ? nullptr : a.gamma;
    if (a.dy_bf16) launch_copy((const uint16_t*)a.dY, M, N, a.scale, row_gamma, rows, tr, s);
    else launch_copy((const float*)a.dY, M, N, a.scale, row_gamma, rows, tr, s);
    if (a.dX) {
        const int64_t items = (Np / 32) * i8_tiles_k(K);
        copy_weights<<<(unsigned)(items < (1 << 20) ? items : (1 << 20)), 256, 0, s>>>(a.packed, N, K, wT, items);
        float* out = a.dx_bf16 ? (float*)(base + ws.dx) : (float*)a.dX;
        launch_gemm_tn(g, wT, M, K, Np, nullptr, 1.0f, out, part, part_bytes, s);
        if (a.dx_bf16) {
            const int64_t n4 = M * K / 4, wgs = (n4 + 255) / 256;
            round_to_bf16<<<(unsigned)(wgs < (1 << 16) ? wgs : (1 << 16)), 256, 0, s>>>(out, (uint16_t*)a.dX, n4);
        }
    }
    if (a.dW) {
        launch_copy(a.codes, M, K, nullptr, nullptr, nullptr, qT, s);
        launch_gemm_tn(gwT, qT, N, K, Mp, a.per_tensor ? a.gamma : nullptr, a.per_tensor ? 1.0f / 128.0f : 1.0f, a.dW, part,
                       part_bytes, s);
    }
    return hipGetLastError();
}

}  // namespace bl
