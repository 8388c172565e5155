// 1-bit x 8-bit products of a mixture of BitLinear layers (Eq. 7 and 11 of arXiv 2310.11453, a weight matrix per
// expert):
//   Y[s,n] = (sum_k q[r,k] S_e[n,k]) * (beta_e gamma_r / 128)    for the slots s of expert e, r the row that s reads
// Few rows an expert: bound by the packed weights of the experts that have any.
#include <algorithm>

#include "common.h"
#include "experts.h"
#include "kernels.h"

namespace bl {

namespace rows {
constexpr int kMaxWaves = 8;  // share the 512-chunks of K
constexpr int kSlots = 16;    // slots of a workgroup
struct Args {
    const int8_t* codes;
    const uint32_t* packed;
    const int32_t *offsets, *order;
    uint32_t T, E, top_k, rows, TN, TK, K, N;
    int64_t blob;
    const float *gamma, *beta;
    const int32_t* rowsum;
    bool per_tensor, out_acc;
    float* Y;
};
}  // namespace rows

// blockIdx.x: a group of TILES 16-row weight tiles, blockIdx.y (and z): the how-manieth 16 slots of an expert.  Wave w
// takes the 512-chunks w, w + W, ... of K; the weights are the row operand of v_mfma_i32_16x16x64_i8, the slots its
// columns; a lane's 16 bytes of a packed tile hold 16 consecutive k of each of eight bit planes, (w >> i) & 0x01010101
// is plane i as {0,1} bytes, and sum_k q s = 2 sum_k q b - sum_k q.  The waves' sums meet in LDS.
// A launch is a chain of trips to memory: the experts' bounds, then the weights and (in two trips) the codes, whose
// rows are known only with the order.  Loads return in the order of their requests, so the order is asked for first,
// then a quarter of the first chunk's weights, then the codes, which are what the matrix instructions wait for, then
// the rest of the weights, which arrive while the first tiles are multiplied.  (All weights ahead of the order, and so
// of everything: 96 slots, 16 experts, 4096 -> 4096 13.4 us a call, 11.7 so; 64, 32, 6144 -> 2048 13.9, 11.7.)
template <int TILES>
__global__ __launch_bounds__(rows::kMaxWaves* kWave) void experts_rows_kernel(rows::Args a) {
    using namespace rows;
    __shared__ int red[kMaxWaves][TILES][kSlots][kTileN + 1];
    __shared__ float sm_scale[kSlots];
    __shared__ int sm_sum[kSlots];
    const int W = (int)blockDim.x / kWave;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x & (kWave - 1);
    const int col = l & 15, g = l >> 4;

    // the expert of this workgroup's slots: a lane counts the sixteens of an expert
    int e = -1, s0 = 0, s1 = 0, left = (int)(blockIdx.z * gridDim.y + blockIdx.y);
    for (int b = 0; b < (int)a.E; b += kWave) {
        const int at = b + l < (int)a.E ? b + l : (int)a.E - 1;
        const int from = slot_bound(a.offsets, at, (int)a.T), to = slot_bound(a.offsets, at + 1, (int)a.T);
        const int n = b + l < (int)a.E && to > from ? (to - from + kSlots - 1) / kSlots : 0;
        int v = n;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int o = __shfl_up(v, d, kWave);
            if (l >= d) v += o;
        }
        const uint64_t behind = __ballot(v > left);
        if (behind) {
            const int lane = __ffsll((unsigned long long)behind) - 1;
            e = b + lane;
            s0 = __builtin_amdgcn_readlane(from, lane) + (left - __builtin_amdgcn_readlane(v - n, lane)) * kSlots;
            s1 = __builtin_amdgcn_readlane(to, lane);
            break;
        }
        left -= __builtin_amdgcn_readlane(v, kWave - 1);
    }
    if (e < 0) return;  // uniform: the grid is a bound

    constexpr int kFirst = TILES > 4 ? TILES / 4 : 1;
    const uint32_t t0 = blockIdx.x * TILES, last = a.TN - 1;
    const uint32_t* const wbase = a.packed + e * a.blob;
    auto load = [&](v4i (&q)[TILES], uint32_t c, int from, int to) {
#pragma unroll
        for (int t = from; t < to; ++t) {
            const uint32_t tn = t0 + t < last ? t0 + t : last;
            const uint32_t* const at = wbase + ((uint64_t)tn * a.TK + c) * 256 + l * 4;
            q[t] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(at));
        }
    };
    v4i q[TILES];
    const int s = s0 + col < s1 ? s0 + col : s1 - 1;
    const int place = a.order ? a.order[s] : 0;
    __builtin_amdgcn_sched_barrier(0);
    load(q, w, 0, kFirst);
    __builtin_amdgcn_sched_barrier(0);
    const uint32_t row = row_of(a.order ? (uint32_t)place / a.top_k : (uint32_t)s, a.rows);
    const int8_t* const x = a.codes + (uint64_t)row * a.K + 16 * g;
    const int klast = (int)a.K - 16 - 16 * g;  // past the row its last 16 bytes again: the packed bits there are zero
    float gamma = 0.f;
    int sum = 0;
    if (w == 0 && l < kSlots) {
        gamma = a.gamma[a.per_tensor ? 0 : row];
        sum = a.rowsum[row];
    }
    const float beta = a.beta[e];

    v4i acc[TILES] = {};
    auto chunk = [&](v4i (&act)[8], uint32_t c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int k = (int)c * kChunkK + 64 * i;
            act[i] = *reinterpret_cast<const v4i*>(x + (k < klast ? k : klast));
        }
    };
    auto multiply = [&](const v4i(&act)[8]) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v4i b;
#pragma unroll
                for (int d = 0; d < 4; ++d) b[d] = (int)(((uint32_t)q[t][d] >> i) & 0x01010101u);
                acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, act[i], acc[t], 0, 0, 0);
            }
    };
    v4i act[8];
    chunk(act, w);
    __builtin_amdgcn_sched_barrier(0);
    load(q, w, kFirst, TILES);
    __builtin_amdgcn_sched_barrier(0);
    multiply(act);
    for (uint32_t c = w + W; c < a.TK; c += W) {
        chunk(act, c);
        __builtin_amdgcn_sched_barrier(0);
        load(q, c, 0, TILES);
        __builtin_amdgcn_sched_barrier(0);
        multiply(act);
    }
    // lane: slot col, weight rows 4 g + r of each tile
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) red[w][t][col][4 * g + r] = acc[t][r];
    if (w == 0 && l < kSlots) {
        sm_scale[l] = (beta * gamma) / 128.0f;
        sm_sum[l] = sum;
    }
    __syncthreads();
    const int n_slots = s1 - s0 < kSlots ? s1 - s0 : kSlots;
    for (int i = threadIdx.x; i < n_slots * TILES * kTileN; i += blockDim.x) {
        const int nl = i % (TILES * kTileN), m = i / (TILES * kTileN);
        const uint32_t n = t0 * kTileN + nl;
        if (n >= a.N) continue;
        int v = 0;
        for (int p = 0; p < W; ++p) v += red[p][nl >> 4][m][nl & 15];
        v = 2 * v - sm_sum[m];
        float* const o = a.Y + (uint64_t)(s0 + m) * a.N + n;
        if (a.out_acc) *reinterpret_cast<int*>(o) = v;
        else *o = (float)v * sm_scale[m];
    }
}

static void launch_rows(const ExpertsArgs& a, hipStream_t s) {
    const int64_t TN = tiles_n(a.N), TK = tiles_k(a.K);
    const int64_t A = a.T < a.E ? a.T : a.E, blocks = a.T / rows::kSlots + A;
    // Tiles of a workgroup: more of them share the fixed chain and the codes, fewer leave no CU idle; eight leave two
    // workgroups of a long reduction on a CU.  us with 2 / 4 / 8, T slots of E experts: T = 8, E = 8, 4096 -> 1024 4.3
    // / 4.7 / 5.7, 4096 -> 2048 5.1 / 4.9 / 5.8; T = 128, E = 16, 4096 -> 1024 6.3 / 5.8 / 7.0, 2048 -> 8192 17.4 /
    // 14.4 / 15.3; T = 64, E = 32, 6144 -> 2048 17.5 / 14.8 / 11.7; T = 128, E = 32, 4096 -> 5120 34.4 / 27.6 / 21.9.
    int tiles = tuning().decode_tiles;
    const int64_t all = blocks * TN;
    if (!tiles) tiles = all < 512 ? 1 : all < 1024 || TK < 4 ? 2 : TK >= 8 && all >= 2048 ? 8 : 4;
    rows::Args r{};
    r.codes = a.codes; r.packed = a.packed; r.offsets = a.offsets; r.order = a.order;
    r.T = (uint32_t)a.T; r.E = (uint32_t)a.E; r.top_k = (uint32_t)a.top_k; r.rows = (uint32_t)a.rows;
    r.TN = (uint32_t)TN; r.TK = (uint32_t)TK; r.K = (uint32_t)a.K; r.N = (uint32_t)a.N;
    r.blob = TN * TK * 256;
    r.gamma = a.gamma; r.beta = a.beta; r.rowsum = a.rowsum;
    r.per_tensor = a.per_tensor; r.out_acc = a.out_acc; r.Y = a.Y;
    const unsigned threads = (unsigned)(TK < rows::kMaxWaves ? TK : rows::kMaxWaves) * kWave;
    auto launch = [&](auto kernel, int n) {
        const int64_t most = 32768;  // of a dimension of a grid, which the bound may pass
        const dim3 grid((unsigned)((TN + n - 1) / n), (unsigned)(blocks < most ? blocks : most),
                        (unsigned)((blocks + most - 1) / most));
        kernel<<<grid, threads, 0, s>>>(r);
    };
    if (tiles <= 1) launch(experts_rows_kernel<1>, 1);
    else if (tiles <= 2) launch(experts_rows_kernel<2>, 2);
    else if (tiles <= 4) launch(experts_rows_kernel<4>, 4);
    else launch(experts_rows_kernel<8>, 8);
}

// The kernel: the cheapest by these costs in us, fitted to graph replays under each of them over 260 shapes (1 to 16384
// slots, 2 to 32 experts of uneven popularity, K and N of 256 to 8192).  How the slots fall on the experts is not known
// here: an expert's last row of tiles is taken to be half full, and a round to be 0.4 of a round longer than they say.
//   128 x 256 tiles   0.3 + rounds (7.3 + 0.37 n)    n stages of 64 k, c chunks of 512
//   256 x 256        -3.5 + rounds (17.5 + 0.62 n)
//   128 x 128         0.2 + rounds (6.8 + 2.84 c / 2)
//   64 x 128          0.6 + rounds (5.75 + 3.14 c / 4)
//   16 slots at a time  2.7 + 1.4 c / 8 + (0.05 c + 0.2) per 16 x 16 outputs and CU
// 0.5 % slower than the best of the five on average over 210 more, 23 % at most (1552 slots, 6 experts, 3296 -> 1155:
// 24.2, 19.6 as 128 x 128).  The extremes, 16 slots at a time / 128 x 256: 64 slots, 8 experts, 4096 -> 4096 10.0 / 29;
// 8900 slots, 12 experts, 3840 -> 4808 787 / 181.
static int experts_plan(const ExpertsArgs& a) {
    const double cus = num_cus(), T = (double)a.T, A = (double)(a.T < a.E ? a.T : a.E);
    const double c = (double)tiles_k(a.K), n = (double)((a.K + 63) / 64);
    auto up = [](double v) { return (double)(int64_t)(v + 0.999999); };
    auto rows_of_tiles = [&](double bm) { return std::max(0.9 * A, T / bm + 0.5 * A); };
    auto rounds = [&](double bm, int64_t bn) {
        return std::max(1.0, rows_of_tiles(bm) * (double)((a.N + bn - 1) / bn) / cus + 0.4);
    };
    const double small = rows_of_tiles(16) * (double)tiles_n(a.N) / cus;
    const double us[5] = {0.3 + rounds(128, 256) * (7.3 + 0.37 * n), -3.5 + rounds(256, 256) * (17.5 + 0.62 * n),
                          0.2 + rounds(128, 128) * (6.8 + 2.84 * up(c / 2)),
                          0.6 + rounds(64, 128) * (5.75 + 3.14 * up(c / 4)),
                          2.7 + 1.4 * up(c / 8) + (0.05 * c + 0.2) * small};
    return 1 + (int)(std::min_element(us, us + 5) - us);
}

hipError_t launch_matmul_experts(const ExpertsArgs& a, hipStream_t s) {
    // the tiled kernels keep offsets into all of the codes in 32 bits
    int tile = tuning().experts_tile ? tuning().experts_tile : experts_plan(a);
    if ((int64_t)a.rows * a.K >= (int64_t)1 << 32) tile = 5;
    if (tile <= 4) {
        GemmArgs g{};
        g.codes = a.codes; g.gamma = a.gamma; g.rowsum = a.rowsum; g.M = a.T; g.K = a.K; g.N = a.N;
        g.packed = a.packed; g.beta = a.beta; g.per_tensor = a.per_tensor; g.out_acc = a.out_acc; g.Y = a.Y;
        g.ldy = a.N; g.ldq = a.K; g.gstride = 1; g.beta_rows = a.N;
        g.offsets = a.offsets; g.order = a.order; g.experts = a.E; g.top_k = a.top_k; g.rows = (uint32_t)a.rows;
        g.blob = tiles_n(a.N) * tiles_k(a.K) * 256;
        return launch_experts_tiles(g, tile, s);
    }
    launch_rows(a, s);
    return hipGetLastError();
}

}  // namespace bl
