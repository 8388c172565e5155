// Root-mean-square norm with the residual's addition and the 8-bit quantiser, and its backward pass.
//   h = x + r (rounded to the residual's type),  1/rms = 1 / sqrt(mean h^2 + eps),  x^ = fl32(h / rms) * gain
//   gamma = max |x^|,  codes = clamp(rne(x^ * (128 / gamma)), -128, 127)            (the quantiser of Eq. 4-5)
// and with n = h / rms, t = g * gain for the gradient g of x^:
//   dh = (t - n * mean(t n)) / rms (+ the residual's own gradient),  dgain = sum over rows of g * n
// The mean square and 1/rms are fp64, so that the fp32 value handed to the rounding is the correctly rounded one; what
// decides a code behind it are single fp32 operations, as in the LayerNorm's quantiser.
#include <type_traits>

#include "common.h"
#include "i8.h"
#include "rowops.h"

namespace bl {

enum RmsMode { kRmsFull = 0, kRmsStats = 1, kRmsApply = 2 };

// Per tensor the first pass leaves the largest magnitude of each workgroup's rows, and every workgroup of the second
// folds them: no launch between the two.  The second pass goes through the rows from the end, which are still in the
// caches.
constexpr int kRmsGroups = kRmsMostBytes / 4;

__device__ inline float4 rounded(float4 v, const uint16_t*) {
    const uint32_t a = bf16_pair(v.x, v.y), b = bf16_pair(v.z, v.w);
    return make_float4(__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16),
                       __uint_as_float(b & 0xffff0000u));
}
__device__ inline float4 rounded(float4 v, const float*) { return v; }
__device__ inline float4 add4(const float4& a, const float4& b) {
    return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
}
__device__ inline float4 mul4(const float4& a, const float4& b) {
    return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w);
}
__device__ inline float4 times(const float4& v, double f) {
    return make_float4((float)((double)v.x * f), (float)((double)v.y * f), (float)((double)v.z * f), (float)((double)v.w * f));
}
__device__ inline void add_squares(double& q, const float4& v) {
    q = fma((double)v.x, (double)v.x, q);
    q = fma((double)v.y, (double)v.y, q);
    q = fma((double)v.z, (double)v.z, q);
    q = fma((double)v.w, (double)v.w, q);
}
// (of an infinity and of NaN: NaN, the step's 0 * inf, so that x^ and gamma are NaN)
__device__ inline double rms_inverse(double mean_square, double eps) {
    const double v = mean_square + eps;
    return v == 0.0 ? 0.0 : rsqrt64_step(v, __builtin_amdgcn_rsq(v));  // (a row of zeros with eps = 0)
}
// gamma: at least 1e-5; a NaN stays
__device__ inline float gamma_of(int most) {
    const float m = __int_as_float(most);
    return m < 1e-5f ? 1e-5f : m;
}
template <int NW>
__device__ inline int block_most(int m, int* sm) {
    m = wave_reduce(m, OpMostBits{});
    __syncthreads();
    if ((threadIdx.x & (kWave - 1)) == 0) sm[threadIdx.x / kWave] = m;
    __syncthreads();
    return fold_slots<NW>(sm, OpMostBits{});
}
// the largest of what the first pass left, in every lane; NW waves
template <int NW>
__device__ inline int tensor_most(const QuantRmsArgs& a, int* sm) {
    int m = 0;
    for (int i = threadIdx.x; i < a.groups; i += NW * kWave) m = OpMostBits{}(m, a.most[i]);
    return block_most<NW>(m, sm);
}

// WPR waves share a row, which lies in their registers (NV float4 a lane) from its one reading on; workgroups have four
// waves at least, so short rows are handled several to a workgroup, without a barrier.  Bound by HBM for large batches,
// by the length of a row's chain for small ones (one reduction without a gain: the largest |x^| is then that of the
// largest |h|).  8192 x 4096, fp32, residual, per token 78 us (5.6 TB/s); per tensor both passes 101 us; one row of
// 2048 2.8 us.
template <typename XT, typename RT, bool RES, int WPR, int NV>
__global__ __launch_bounds__((WPR < 4 ? 4 : WPR) * kWave, 4) void quant_rms_rows(QuantRmsArgs a, int mode) {
    constexpr int NW = WPR < 4 ? 4 : WPR, RPW = NW / WPR, LANES = WPR * kWave;
    __shared__ double smd[NW];
    __shared__ int smm[2][NW];
    __shared__ int smi[NW];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), rw = wave / WPR, wr = wave % WPR;
    const int t = wr * kWave + (threadIdx.x & (kWave - 1)), K4 = (int)(a.K / 4);
    // a row's loads before the last one's sum and barriers (with a residual there is no room for them)
    constexpr bool AHEAD = !RES;
    float gamma = 0.f;
    int best = 0;
    float4 v[NV];
    // unconditional (the last piece again past the row), so that all are in flight before the first is needed
    auto load_x = [&](int64_t row) {
        const XT* x = static_cast<const XT*>(a.X) + (mode == kRmsApply ? a.M - 1 - row : row) * a.K;
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = load4(x, t + j * LANES < K4 ? t + j * LANES : K4 - 1);
    };
    const int64_t first = (int64_t)blockIdx.x * RPW + rw, stride = (int64_t)gridDim.x * RPW;
    if (AHEAD) load_x(first < a.M ? first : a.M - 1);
    if (mode == kRmsApply) {
        gamma = gamma_of(tensor_most<NW>(a, smm[0]));
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.gamma = gamma;
    }
    static_assert(WPR == 1 || RPW == 1, "no barriers where a workgroup has rows past the last one");
    for (int64_t at = first; at < a.M; at += stride) {
        const int64_t row = mode == kRmsApply ? a.M - 1 - at : at;
        const RT* r = RES ? static_cast<const RT*>(a.R) + row * a.K : nullptr;
        float4 u[RES ? NV : 1];
        if (!AHEAD) load_x(at);
        if constexpr (RES)
#pragma unroll
            for (int j = 0; j < NV; ++j) u[j] = load4(r, t + j * LANES < K4 ? t + j * LANES : K4 - 1);
        double q = 0.0;
        int m = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (RES) v[j] = rounded(add4(v[j], u[j]), r);
            if (K4 < (j + 1) * LANES && t + j * LANES >= K4) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mode != kRmsApply) {
                add_squares(q, v[j]);
                m = most_bits(m, v[j]);
            }
        }
        if constexpr (RES)
            if (a.H) {
                RT* h = static_cast<RT*>(a.H) + row * a.K;
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (t + j * LANES < K4) store4(h, t + j * LANES, v[j]);
            }
        double rstd;
        if (mode == kRmsApply) {
            rstd = a.rstd[row];
        } else {
            q = wave_reduce(q, OpSum{});
            m = wave_reduce(m, OpMostBits{});
            if constexpr (WPR > 1) {
                if ((threadIdx.x & (kWave - 1)) == 0) {
                    smd[wave] = q;
                    smm[0][wave] = m;
                }
                __syncthreads();
                q = fold_slots<WPR>(smd + rw * WPR, OpSum{});
                m = fold_slots<WPR>(smm[0] + rw * WPR, OpMostBits{});
            }
            rstd = rms_inverse(q * a.inv_k, a.eps);
            m = most_bits(0, (float)((double)__int_as_float(m) * rstd));
        }
        // (hidden from the optimiser, which would keep the converted copies of all elements alive)
        if constexpr (NV > 2)
#pragma unroll
            for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
        if (mode != kRmsStats || a.gain) {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = times(v[j], rstd);
            if (a.gain) {
#pragma unroll
                for (int j = 0; j < NV; ++j) v[j] = mul4(v[j], load4(a.gain, t + j * LANES < K4 ? t + j * LANES : K4 - 1));
                if (mode != kRmsApply) {
                    m = 0;
#pragma unroll
                    for (int j = 0; j < NV; ++j) m = most_bits(m, v[j]);
                    m = row_reduce<WPR>(m, OpMostBits{}, smm[1], rw, wr);
                }
            }
        }
        if (mode == kRmsStats) {
            best = OpMostBits{}(best, m);
            if (t == 0) a.rstd[row] = rstd;
            if (AHEAD && at + stride < a.M) load_x(at + stride);
            if (WPR > 1) __syncthreads();  // the slots are read
            continue;
        }
        if (mode == kRmsFull) gamma = gamma_of(m);
        const float scale = 128.0f / gamma;
        int rs = 0;
        uint32_t* c4 = reinterpret_cast<uint32_t*>(a.codes + row * a.K);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * LANES;
            const uint32_t w = code_word(v[j].x * scale, v[j].y * scale, v[j].z * scale, v[j].w * scale);
            rs = __builtin_amdgcn_sdot4((int)w, 0x01010101, rs, false);  // (zeros past the row)
            if (i < K4) {
                c4[i] = w;
                if (a.xhat) store4(a.xhat + row * a.K, i, v[j]);
            }
        }
        if (AHEAD && at + stride < a.M) load_x(at + stride);
        if (a.rowsum) {
            rs = row_reduce<WPR>(rs, OpSum{}, smi, rw, wr);
            if (t == 0) a.rowsum[row] = rs;
        }
        if (t == 0 && mode == kRmsFull) a.gamma[row] = gamma;
        if (WPR > 1) __syncthreads();
    }
    if (mode == kRmsStats) {
        __syncthreads();
        best = block_most<NW>(best, smm[0]);
        if (threadIdx.x == 0) a.most[blockIdx.x] = best;
    }
}

// Rows past registers (K > 32768): a workgroup walks a row from memory once per step.
template <typename XT, typename RT, bool RES>
__global__ __launch_bounds__(512) void quant_rms_long(QuantRmsArgs a, int mode) {
    constexpr int NW = 8, T = NW * kWave;
    __shared__ double smd[NW];
    __shared__ int smm[NW];
    __shared__ int smi[NW];
    const int t = threadIdx.x;
    const int64_t K4 = a.K / 4;
    float gamma = 0.f;
    int best = 0;
    if (mode == kRmsApply) {
        gamma = gamma_of(tensor_most<NW>(a, smm));
        if (blockIdx.x == 0 && t == 0) *a.gamma = gamma;
    }
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const XT* x = static_cast<const XT*>(a.X) + row * a.K;
        const RT* r = RES ? static_cast<const RT*>(a.R) + row * a.K : nullptr;
        RT* h = RES && a.H ? static_cast<RT*>(a.H) + row * a.K : nullptr;
        auto sum_at = [&](int64_t i) {
            const float4 v = load4(x, i);
            if constexpr (RES) return rounded(add4(v, load4(r, i)), r);
            return v;
        };
        double rstd;
        if (mode == kRmsApply) {
            rstd = a.rstd[row];
        } else {
            double q = 0.0;
            for (int64_t i = t; i < K4; i += T) add_squares(q, sum_at(i));
            rstd = rms_inverse(block_sum<NW>(q, smd) * a.inv_k, a.eps);
        }
        auto hat = [&](const float4& v, int64_t i) {
            const float4 o = times(v, rstd);
            return a.gain ? mul4(o, load4(a.gain, i)) : o;
        };
        // (h may be x or r: an element is read and written by the same thread, and not read there again)
        if (mode != kRmsApply) {
            int m = 0;
            for (int64_t i = t; i < K4; i += T) m = most_bits(m, hat(sum_at(i), i));
            m = block_most<NW>(m, smm);
            if (mode == kRmsStats) {
                best = OpMostBits{}(best, m);
                if (t == 0) a.rstd[row] = rstd;
                if (h)
                    for (int64_t i = t; i < K4; i += T) store4(h, i, sum_at(i));
                __syncthreads();  // the slots of the reductions are read
                continue;
            }
            gamma = gamma_of(m);
        }
        const float scale = 128.0f / gamma;
        uint32_t* c4 = reinterpret_cast<uint32_t*>(a.codes + row * a.K);
        int rs = 0;
        for (int64_t i = t; i < K4; i += T) {
            const float4 v = sum_at(i), o = hat(v, i);
            if (h) store4(h, i, v);
            if (a.xhat) store4(a.xhat + row * a.K, i, o);
            const uint32_t w = code_word(o.x * scale, o.y * scale, o.z * scale, o.w * scale);
            rs = __builtin_amdgcn_sdot4((int)w, 0x01010101, rs, false);
            c4[i] = w;
        }
        if (a.rowsum) {
            rs = block_sum<NW>(rs, smi);
            if (t == 0) a.rowsum[row] = rs;
        }
        if (t == 0 && mode == kRmsFull) a.gamma[row] = gamma;
        __syncthreads();
    }
    if (mode == kRmsStats && t == 0) a.most[blockIdx.x] = best;
}

// Waves a row and float4 a lane (1, 2, 3, 4, 6, 8: with powers of two alone 5784 x 5472 bf16 took 45 us instead of 38, 1600 x
// 20480 66 instead of 55); more waves where the batch alone would leave SIMDs idle.
struct RmsShape {
    int wpr, nv;
};
static RmsShape rms_shape(int64_t M, int64_t K) {
    const int64_t K4 = K / 4;
    int wpr = 1;
    while (wpr < 16 && K4 > (int64_t)wpr * kWave * 8) wpr *= 4;
    while (wpr < 16 && M * wpr < 1024 && K4 >= (int64_t)wpr * kWave * 4) wpr *= 4;
    // eight waves, so that a CU holds two rows: 3705 x 9056 bf16 61 us, with sixteen 78 (with eight float4 a lane;
    // now 46)
    if (wpr == 16 && M > 512 && K4 <= 8 * kWave * 8) wpr = 8;
    const int64_t per_lane = (K4 + wpr * kWave - 1) / (wpr * kWave);
    int nv = 1;
    while (nv < per_lane) nv *= 2;
    if (nv >= 4 && per_lane <= nv / 4 * 3) nv = nv / 4 * 3;
    return {wpr, nv};
}
static unsigned rms_groups(int64_t M, int rpw) {
    const int64_t g = (M + rpw - 1) / rpw;
    return (unsigned)(g < kRmsGroups ? g : kRmsGroups);
}

template <typename XT, typename RT, bool RES>
static int launch_rms_typed(const QuantRmsArgs& a, int mode, hipStream_t s) {
    if (a.K > 32768) {
        const unsigned grid = rms_groups(a.M, 1);
        quant_rms_long<XT, RT, RES><<<grid, 512, 0, s>>>(a, mode);
        return (int)grid;
    }
    const RmsShape sh = rms_shape(a.M, a.K);
    const int nw = sh.wpr < 4 ? 4 : sh.wpr, rpw = nw / sh.wpr;
    const int64_t wgs = (a.M + rpw - 1) / rpw;
    // (the second pass: four workgroups a CU, whose next rows are on their way: 8192 x 4096 bf16 both passes 64 us, without 67;
    // with two workgroups a CU 74)
    const int64_t most = mode == kRmsFull ? 1 << 20 : mode == kRmsApply ? 1024 : kRmsGroups;
    const unsigned grid = (unsigned)(wgs < most ? wgs : most);
#define BL_RMS_CASE(W, V) \
    if (sh.wpr == W && sh.nv == V) quant_rms_rows<XT, RT, RES, W, V><<<grid, nw * kWave, 0, s>>>(a, mode); else
    BL_RMS_CASE(1, 1) BL_RMS_CASE(1, 2) BL_RMS_CASE(1, 3) BL_RMS_CASE(1, 4) BL_RMS_CASE(1, 6) BL_RMS_CASE(1, 8)
    BL_RMS_CASE(4, 1) BL_RMS_CASE(4, 2) BL_RMS_CASE(4, 3) BL_RMS_CASE(4, 4) BL_RMS_CASE(4, 6) BL_RMS_CASE(4, 8)
    BL_RMS_CASE(8, 6) BL_RMS_CASE(8, 8)
    BL_RMS_CASE(16, 1) BL_RMS_CASE(16, 2) BL_RMS_CASE(16, 3) BL_RMS_CASE(16, 4) BL_RMS_CASE(16, 6) BL_RMS_CASE(16, 8)
    return -1;
#undef BL_RMS_CASE
    return (int)grid;
}
static int launch_rms(const QuantRmsArgs& a, int mode, hipStream_t s) {
    if (!a.R)
        return a.x_bf16 ? launch_rms_typed<uint16_t, uint16_t, false>(a, mode, s)
                        : launch_rms_typed<float, float, false>(a, mode, s);
    if (a.x_bf16)
        return a.h_bf16 ? launch_rms_typed<uint16_t, uint16_t, true>(a, mode, s)
                        : launch_rms_typed<uint16_t, float, true>(a, mode, s);
    return a.h_bf16 ? launch_rms_typed<float, uint16_t, true>(a, mode, s) : launch_rms_typed<float, float, true>(a, mode, s);
}

hipError_t launch_quant_rmsnorm(const QuantRmsArgs& a_in, hipStream_t s) {
    QuantRmsArgs a = a_in;
    a.inv_k = 1.0 / (double)a.K;
    if (!a.per_tensor) return launch_rms(a, kRmsFull, s) < 0 ? hipErrorInvalidValue : hipGetLastError();
    a.groups = launch_rms(a, kRmsStats, s);
    if (a.R && a.H) {  // x + r is there now
        a.X = a.H;
        a.x_bf16 = a.h_bf16;
        a.R = nullptr;
        a.H = nullptr;
    }
    return a.groups < 0 || launch_rms(a, kRmsApply, s) < 0 ? hipErrorInvalidValue : hipGetLastError();
}

// ---- backward -----------------------------------------------------------------------------------------
// The workgroups are as many as fill the chip and go through the rows; a lane has the same columns of all its rows, so that
// their share of dgain is summed in its registers, and each workgroup leaves one sum a column for fold_dgain.  A row is
// read once; bound by HBM.  8192 x 4096, fp32 gradients, bf16 h, a residual's gradient: 86 us (5.5 TB/s), with dgain
// 93; all bf16, with dgain, 8192 x 4096 62 us (4.3), 2048 x 16384 82 us (3.3).
// A lane's sums are fp64, but with six or eight float4 a lane (K > 16384) fp32, for which there is room, over 64 rows at most:
// there are as many workgroups as that takes.  What leaves a wave for LDS and a workgroup for memory is rounded to fp32, half the
// bytes: two roundings of parts of the sum beside the result's own; fold_dgain adds in fp64.  With six or eight the gradient is
// read again, out of the cache, where it is used, instead of kept: 1600 x 20480 bf16 70 us (76 with eight float4 a lane, 159 with
// both in registers, which spill, 193 with the sums in memory), all with h as the residual's gradient; with one of its own 96.
// Rows past registers (K > 32768): fp64 sums in memory.
constexpr int64_t kRmsBackwardWide = 16384, kRmsBackwardK = 32768;
static int rms_backward_groups(int64_t M, int64_t K) {
    if (K <= kRmsBackwardWide) return (int)(M < 512 ? M : 512);
    const int64_t g = M < 256 ? M : 256, rows = (M + 63) / 64;
    return (int)(K <= kRmsBackwardK && rows > g ? rows : g);
}
size_t rms_backward_part_bytes(int64_t M, int64_t K) {
    return (size_t)rms_backward_groups(M, K) * (size_t)K * (K > kRmsBackwardK ? 8 : 4);
}
template <typename GT, typename HT, typename DT, int WPR, int NV>
__global__ __launch_bounds__((WPR < 8 ? 8 : WPR) * kWave, 4) void rms_backward_rows(RmsBackwardArgs a) {
    constexpr int NW = WPR < 8 ? 8 : WPR, RPW = NW / WPR, LANES = WPR * kWave;
    constexpr bool WIDE = NV > 4;  // 32-bit sums; the residual's gradient is read where it is added
    __shared__ double smd[2][2][NW];
    __shared__ float smg[RPW > 1 ? RPW - 1 : 1][NV][LANES][4];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), rw = wave / WPR, wr = wave % WPR;
    int t = wr * kWave + (threadIdx.x & (kWave - 1));
    const int K4 = (int)(a.K / 4);
    using Sum = std::conditional_t<WIDE, float, double>;
    Sum dg[NV][4];
#pragma unroll
    for (int j = 0; j < NV; ++j) dg[j][0] = dg[j][1] = dg[j][2] = dg[j][3] = 0;
    int parity = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * RPW; row0 < a.M; row0 += (int64_t)gridDim.x * RPW) {
        // (addresses and gains are not kept from row to row, which would spill: 4096 x 8192 95 -> 79 us)
        if constexpr (NV >= 4) asm volatile("" : "+v"(t));
        int64_t row = row0 + rw;
        const bool live = row < a.M;
        if (!live) {
            if (WPR == 1) break;  // no barriers behind
            row = a.M - 1;
        }
        const GT* g = static_cast<const GT*>(a.G) + row * a.K;
        const HT* h = static_cast<const HT*>(a.H) + row * a.K;
        const DT* dr = a.dR ? static_cast<const DT*>(a.dR) + row * a.K : nullptr;
        float4 v[NV], u[NV], w[WIDE ? 1 : NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) v[j] = load4(h, t + j * LANES < K4 ? t + j * LANES : K4 - 1);
#pragma unroll
        for (int j = 0; j < NV; ++j) u[j] = load4(g, t + j * LANES < K4 ? t + j * LANES : K4 - 1);
        if constexpr (!WIDE) {
            if (dr)
#pragma unroll
                for (int j = 0; j < NV; ++j) w[j] = load4(dr, t + j * LANES < K4 ? t + j * LANES : K4 - 1);
            else
#pragma unroll
                for (int j = 0; j < NV; ++j) w[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        double q = 0.0, c = 0.0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (K4 < (j + 1) * LANES && t + j * LANES >= K4) v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
            const float4 s = a.gain ? mul4(u[j], load4(a.gain, t + j * LANES < K4 ? t + j * LANES : K4 - 1)) : u[j];
            add_squares(q, v[j]);
            c = fma((double)v[j].x, (double)s.x, c);
            c = fma((double)v[j].y, (double)s.y, c);
            c = fma((double)v[j].z, (double)s.z, c);
            c = fma((double)v[j].w, (double)s.w, c);
        }
        q = wave_reduce(q, OpSum{});
        c = wave_reduce(c, OpSum{});
        if constexpr (WPR > 1) {
            if ((threadIdx.x & (kWave - 1)) == 0) {
                smd[parity][0][wave] = q;
                smd[parity][1][wave] = c;
            }
            __syncthreads();
            q = fold_slots<WPR>(smd[parity][0] + rw * WPR, OpSum{});
            c = fold_slots<WPR>(smd[parity][1] + rw * WPR, OpSum{});
            parity ^= 1;  // read before the barrier of the next row, written behind it
        }
        const double rstd = rms_inverse(q * a.inv_k, a.eps);
        // 1/rms of a row below 2^-60 or above 2^60, or what is made of it, may be past fp32's range or have lost digits there: it
        // is taken as inv64 * half then, half a power of two of half its exponent, and h as h * half (uniform in a row).  The
        // branch costs 0 to 3 % (5784 x 5472 58.3 -> 60.1 us); powers of two in every row's arithmetic, or a loop of its own for
        // such rows, 1 to 8 %.
        double inv64 = rstd;
        float half = 1.0f;
        if (__builtin_amdgcn_readfirstlane(rstd != 0.0 && !(rstd > 0x1p-60 && rstd < 0x1p60))) {
            int e;
            frexp(rstd, &e);
            half = (float)ldexp(1.0, e / 2);
            inv64 = rstd * ldexp(1.0, -(e / 2));
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = make_float4(v[j].x * half, v[j].y * half, v[j].z * half, v[j].w * half);
        }
        const float inv = (float)inv64, along = (float)(c * a.inv_k * rstd * inv64);  // mean(t n) / rms (/ half)
        // (hidden from the optimiser, which would keep the converted copies of all elements alive)
#pragma unroll
        for (int j = 0; j < NV; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
        if constexpr (WIDE) asm volatile("" : "+v"(t));
        DT* dh = static_cast<DT*>(a.dH) + row * a.K;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = t + j * LANES;
            if (i < K4 && live) {
                if constexpr (WIDE) u[j] = load4(g, i);
                const float4 s = a.gain ? mul4(u[j], load4(a.gain, i)) : u[j];
                float4 r = w[WIDE ? 0 : j];
                if constexpr (WIDE) r = dr ? load4(dr, i) : make_float4(0.f, 0.f, 0.f, 0.f);
                float4 d;  // (with half = 1 the sum)
                d.x = fmaf((s.x - v[j].x * along) * inv, half, r.x);
                d.y = fmaf((s.y - v[j].y * along) * inv, half, r.y);
                d.z = fmaf((s.z - v[j].z * along) * inv, half, r.z);
                d.w = fmaf((s.w - v[j].w * along) * inv, half, r.w);
                store4(dh, i, d);
                if (a.dgain) {  // (n first: g h may be past the largest float, or have lost its digits)
                    const Sum f = WIDE ? (Sum)inv : (Sum)inv64;
                    dg[j][0] = fma((Sum)u[j].x, (Sum)v[j].x * f, dg[j][0]);
                    dg[j][1] = fma((Sum)u[j].y, (Sum)v[j].y * f, dg[j][1]);
                    dg[j][2] = fma((Sum)u[j].z, (Sum)v[j].z * f, dg[j][2]);
                    dg[j][3] = fma((Sum)u[j].w, (Sum)v[j].w * f, dg[j][3]);
                }
            }
        }
    }
    if (!a.dgain) return;
    // the rows of the workgroup's waves together
    if constexpr (RPW > 1) {
        if (rw > 0)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) smg[rw - 1][j][t][e] = (float)dg[j][e];
        __syncthreads();
        if (rw > 0) return;
#pragma unroll
        for (int p = 0; p < RPW - 1; ++p)
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) dg[j][e] += (Sum)smg[p][j][t][e];
    }
    float* part = static_cast<float*>(a.partials) + (int64_t)blockIdx.x * a.K;
#pragma unroll
    for (int j = 0; j < NV; ++j)
        if (t + j * LANES < K4)
            store4(part, t + j * LANES, make_float4((float)dg[j][0], (float)dg[j][1], (float)dg[j][2], (float)dg[j][3]));
}

// Rows past registers: each is walked twice, and the columns' sums (fp64) lie in memory, where only one thread writes them.
template <typename GT, typename HT, typename DT>
__global__ __launch_bounds__(512) void rms_backward_long(RmsBackwardArgs a) {
    constexpr int NW = 8, T = NW * kWave;
    __shared__ double smd[2][NW];
    const int t = threadIdx.x;
    const int64_t K4 = a.K / 4;
    double* const part = a.dgain ? static_cast<double*>(a.partials) + (int64_t)blockIdx.x * a.K : nullptr;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const GT* g = static_cast<const GT*>(a.G) + row * a.K;
        const HT* h = static_cast<const HT*>(a.H) + row * a.K;
        const DT* dr = a.dR ? static_cast<const DT*>(a.dR) + row * a.K : nullptr;
        DT* dh = static_cast<DT*>(a.dH) + row * a.K;
        auto scaled = [&](const float4& v, int64_t i) { return a.gain ? mul4(v, load4(a.gain, i)) : v; };
        double q = 0.0, c = 0.0;
        for (int64_t i = t; i < K4; i += T) {
            const float4 v = load4(h, i), u = scaled(load4(g, i), i);
            add_squares(q, v);
            c = fma((double)v.x, (double)u.x, c);
            c = fma((double)v.y, (double)u.y, c);
            c = fma((double)v.z, (double)u.z, c);
            c = fma((double)v.w, (double)u.w, c);
        }
        const double rstd = rms_inverse(block_sum<NW>(q, smd[0]) * a.inv_k, a.eps);
        const double along = block_sum<NW>(c, smd[1]) * a.inv_k * rstd * rstd;  // mean(t n) / rms
        for (int64_t i = t; i < K4; i += T) {
            const float4 v = load4(h, i), u0 = load4(g, i), u = scaled(u0, i);
            double d[4] = {((double)u.x - (double)v.x * along) * rstd, ((double)u.y - (double)v.y * along) * rstd,
                           ((double)u.z - (double)v.z * along) * rstd, ((double)u.w - (double)v.w * along) * rstd};
            if (dr) {
                const float4 w = load4(dr, i);
                d[0] += w.x; d[1] += w.y; d[2] += w.z; d[3] += w.w;
            }
            store4(dh, i, make_float4((float)d[0], (float)d[1], (float)d[2], (float)d[3]));
            if (part) {
                double* p = part + 4 * i;
                const bool first = row == blockIdx.x;
                p[0] = fma((double)u0.x, (double)v.x * rstd, first ? 0.0 : p[0]);
                p[1] = fma((double)u0.y, (double)v.y * rstd, first ? 0.0 : p[1]);
                p[2] = fma((double)u0.z, (double)v.z * rstd, first ? 0.0 : p[2]);
                p[3] = fma((double)u0.w, (double)v.w * rstd, first ? 0.0 : p[3]);
            }
        }
        __syncthreads();
    }
}
// 32 columns a workgroup, the groups' sums dealt to 32 lanes of each
template <typename PT>
__global__ __launch_bounds__(1024) void fold_dgain(const PT* __restrict__ part, int groups, int64_t K,
                                                   float* __restrict__ dgain) {
    __shared__ double sm[32][33];
    const int c = threadIdx.x & 31, p = threadIdx.x >> 5;
    for (int64_t k0 = (int64_t)blockIdx.x * 32; k0 < K; k0 += (int64_t)gridDim.x * 32) {
        double s = 0.0;
#pragma unroll 4
        for (int b = p; b < groups; b += 32) s += (double)part[b * K + k0 + c];
        sm[p][c] = s;
        __syncthreads();
        if (p == 0) {
#pragma unroll
            for (int i = 1; i < 32; ++i) s += sm[i][c];
            dgain[k0 + c] = (float)s;
        }
        __syncthreads();
    }
}

template <typename GT, typename HT, typename DT>
static int launch_rms_backward_typed(const RmsBackwardArgs& a, hipStream_t s) {
    if (a.K > kRmsBackwardK) {
        const int grid = rms_backward_groups(a.M, a.K);
        rms_backward_long<GT, HT, DT><<<(unsigned)grid, 512, 0, s>>>(a);
        return grid;
    }
    // two float4 a lane as long as eight waves hold a row so, then three or four, then sixteen waves
    const int64_t K4 = a.K / 4;
    int wpr = 1;
    while (wpr < 8 && K4 > (int64_t)wpr * kWave * 2) wpr *= 2;
    if (K4 > 8 * kWave * 4) wpr = 16;
    int nv = K4 <= kWave ? 1 : K4 <= (int64_t)wpr * kWave * 2 ? 2 : K4 <= (int64_t)wpr * kWave * 4 ? 4 : 8;
    if (nv >= 4 && K4 <= (int64_t)wpr * kWave * (nv / 4 * 3)) nv = nv / 4 * 3;
    const int rpw = wpr < 8 ? 8 / wpr : 1, threads = wpr < 8 ? 512 : wpr * kWave;
    const int64_t wgs = (a.M + rpw - 1) / rpw;
    const int most = rms_backward_groups(a.M, a.K), grid = (int)(wgs < most ? wgs : most);
#define BL_RMS_CASE(W, V) \
    if (wpr == W && nv == V) rms_backward_rows<GT, HT, DT, W, V><<<(unsigned)grid, threads, 0, s>>>(a); else
    BL_RMS_CASE(1, 1) BL_RMS_CASE(1, 2) BL_RMS_CASE(2, 2) BL_RMS_CASE(4, 2) BL_RMS_CASE(8, 2) BL_RMS_CASE(8, 3)
    BL_RMS_CASE(8, 4) BL_RMS_CASE(16, 3) BL_RMS_CASE(16, 4) BL_RMS_CASE(16, 6) BL_RMS_CASE(16, 8) return -1;
#undef BL_RMS_CASE
    return grid;
}
template <typename GT, typename HT>
static int launch_rms_backward(const RmsBackwardArgs& a, hipStream_t s) {
    return a.d_bf16 ? launch_rms_backward_typed<GT, HT, uint16_t>(a, s) : launch_rms_backward_typed<GT, HT, float>(a, s);
}
hipError_t launch_rmsnorm_backward(const RmsBackwardArgs& a_in, hipStream_t s) {
    RmsBackwardArgs a = a_in;
    a.inv_k = 1.0 / (double)a.K;
    const int groups = a.g_bf16 ? a.h_bf16 ? launch_rms_backward<uint16_t, uint16_t>(a, s)
                                           : launch_rms_backward<uint16_t, float>(a, s)
                     : a.h_bf16 ? launch_rms_backward<float, uint16_t>(a, s)
                                : launch_rms_backward<float, float>(a, s);
    if (groups < 0) return hipErrorInvalidValue;
    if (a.dgain) {
        const int64_t wgs = a.K / 32;
        const unsigned grid = (unsigned)(wgs < 65536 ? wgs : 65536);
        if (a.K > kRmsBackwardK) fold_dgain<<<grid, 1024, 0, s>>>(static_cast<const double*>(a.partials), groups, a.K, a.dgain);
        else fold_dgain<<<grid, 1024, 0, s>>>(static_cast<const float*>(a.partials), groups, a.K, a.dgain);
    }
    return hipGetLastError();
}

}  // namespace bl
