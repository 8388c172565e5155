// 1-bit x 8-bit products of a mixture of BitLinear layers (Eq. 7 and 11 of arXiv 2310.11453, a weight matrix per expert):
//   Y[s,n] = (sum_k q[r,k] S_e[n,k]) * (beta_e gamma_r / 128)    for the slots s of expert e, r the row that s reads
// Few rows an expert: bound by the packed weights of the experts that have any.
#include "common.h"
#include "experts.h"
#include "kernels.h"

namespace bl {

namespace rows {
constexpr int kTiles = 4;     // 16-row weight tiles of a workgroup
constexpr int kMaxWaves = 8;  // share the 512-chunks of K
constexpr int kTokens = 16;   // slots of a pass
}  // namespace rows

// blockIdx.x: a group of weight tiles, blockIdx.y: the how-manieth expert that has slots.  Wave w takes the 512-chunks w,
// w + W, ... of K; the weights are the row operand of v_mfma_i32_16x16x64_i8, 16 slots its columns; a lane's 16
// bytes of a packed tile hold 16 consecutive k of each of eight bit planes, (w >> i) & 0x01010101 is plane i as {0,1}
// bytes, and sum_k q s = 2 sum_k q b - sum_k q.  The waves' sums meet in LDS.  More than 16 slots: pass after pass.
__global__ __launch_bounds__(rows::kMaxWaves* kWave) void experts_rows_kernel(ExpertsArgs a, int64_t blob) {
    using namespace rows;
    __shared__ int red[kMaxWaves][kTiles][kTokens][kTileN + 1];
    const int W = (int)blockDim.x / kWave;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x & (kWave - 1);
    const int T = (int)a.T;
    int e = -1, left = (int)blockIdx.y;
    for (int b = 0; b < a.E; b += kWave) {
        const bool some = b + l < a.E && slot_bound(a.offsets, b + l, T) < slot_bound(a.offsets, b + l + 1, T);
        uint64_t m = __ballot(some);
        const int n = __popcll(m);
        if (left >= n) {
            left -= n;
            continue;
        }
        for (; left > 0; --left) m &= m - 1;
        e = b + __ffsll((unsigned long long)m) - 1;
        break;
    }
    if (e < 0) return;  // uniform: fewer experts have slots
    const int s0 = slot_bound(a.offsets, e, T), s1 = slot_bound(a.offsets, e + 1, T);
    const int64_t TN = tiles_n(a.N), TK = tiles_k(a.K);
    const int t0 = (int)blockIdx.x * kTiles, nt = (int)(TN - t0 < kTiles ? TN - t0 : kTiles);
    const uint32_t* wbase = a.packed + e * blob;
    const float beta = a.beta[e];
    const int col = l & 15, g = l >> 4;

    for (int m0 = s0; m0 < s1; m0 += kTokens) {
        const int s = m0 + col < s1 ? m0 + col : s1 - 1;
        const int8_t* x = a.codes + (int64_t)code_row(a.order, (uint32_t)a.top_k, (uint32_t)a.rows, (uint32_t)s) * a.K;
        v4i acc[kTiles] = {};
        for (int64_t c = w; c < TK; c += W) {
            v4i act[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int64_t k = c * kChunkK + 64 * i + 16 * g;
                if (k > a.K - 16) k = a.K - 16;  // the packed bits there are zero
                act[i] = *reinterpret_cast<const v4i*>(x + k);
            }
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const int tn = t < nt ? t0 + t : t0;
                const v4i q = *reinterpret_cast<const v4i*>(wbase + tile_dword_offset(tn, c, TK) + l * 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v4i b;
#pragma unroll
                    for (int d = 0; d < 4; ++d) b[d] = (int)(((uint32_t)q[d] >> i) & 0x01010101u);
                    acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, act[i], acc[t], 0, 0, 0);
                }
            }
        }
        // lane: slot col, weight rows 4 g + r of each tile
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) red[w][t][col][4 * g + r] = acc[t][r];
        __syncthreads();
        for (int i = threadIdx.x; i < nt * kTokens * kTileN; i += blockDim.x) {
            const int n16 = i & 15, m = (i >> 4) % kTokens, t = (i >> 4) / kTokens;
            const int64_t n = (int64_t)(t0 + t) * kTileN + n16;
            if (m0 + m >= s1 || n >= a.N) continue;
            int sum = 0;
            for (int v = 0; v < W; ++v) sum += red[v][t][m][n16];
            const int64_t r = code_row(a.order, (uint32_t)a.top_k, (uint32_t)a.rows, (uint32_t)(m0 + m));
            sum = 2 * sum - a.rowsum[r];
            const int64_t o = (int64_t)(m0 + m) * a.N + n;
            if (a.out_acc) reinterpret_cast<int*>(a.Y)[o] = sum;
            else a.Y[o] = (float)sum * ((beta * a.gamma[a.per_tensor ? 0 : r]) / 128.0f);
        }
        __syncthreads();
    }
}

hipError_t launch_matmul_experts(const ExpertsArgs& a, hipStream_t s) {
    const int force = tuning().experts_tile;
    const int tile = force ? force : a.T / a.E > 160 ? 2 : a.T / a.E > 32 ? 1 : 4;
    if (tile <= 2 && (int64_t)a.rows * a.K < (int64_t)1 << 32) {
        GemmArgs g{};
        g.codes = a.codes; g.gamma = a.gamma; g.rowsum = a.rowsum; g.M = a.T; g.K = a.K; g.N = a.N;
        g.packed = a.packed; g.beta = a.beta; g.per_tensor = a.per_tensor; g.out_acc = a.out_acc; g.Y = a.Y;
        g.ldy = a.N; g.ldq = a.K; g.gstride = 1; g.beta_rows = a.N;
        g.offsets = a.offsets; g.order = a.order; g.experts = a.E; g.top_k = a.top_k; g.rows = (uint32_t)a.rows;
        g.blob = tiles_n(a.N) * tiles_k(a.K) * 256;
        return launch_experts_tiles(g, tile, s);
    }
    const int64_t TN = tiles_n(a.N), TK = tiles_k(a.K);
    const int W = (int)(TK < rows::kMaxWaves ? TK : rows::kMaxWaves);
    const dim3 grid((unsigned)((TN + rows::kTiles - 1) / rows::kTiles), (unsigned)(a.T < a.E ? a.T : a.E));
    experts_rows_kernel<<<grid, W * kWave, 0, s>>>(a, tiles_n(a.N) * TK * 256);
    return hipGetLastError();
}

}  // namespace bl
