// Root-mean-square norm with the residual's addition and the 8-bit quantiser, and its backward pass.
//   h = x + r (rounded to the residual's type),  1/rms = 1 / sqrt(mean h^2 + eps),  x^ = fl32(h / rms) * gain
//   gamma = max |x^|,  codes = clamp(rne(x^ * (128 / gamma)), -128, 127)            (the quantiser of Eq. 4-5)
// and with n = h / rms, t = g * gain for the gradient g of x^:
//   dh = (t - n * mean(t n)) / rms (+ the residual's own gradient),  dgain = sum over rows of g * n
// The mean square and 1/rms are fp64, so that the fp32 value handed to the rounding is the correctly rounded one; what
// decides a code behind it are single fp32 operations, as in the LayerNorm's quantiser.
#include "common.h"
#include "i8.h"
#include "rowops.h"

namespace bl {

enum RmsMode { kRmsFull = 0, kRmsStats = 1, kRmsApply = 2 };

// A workgroup walks a row from memory once per step.
template <typename XT, typename RT, bool RES>
__global__ __launch_bounds__(512) void quant_rms_long(QuantRmsArgs a, int mode) {
    constexpr int NW = 8, T = NW * kWave;
    __shared__ double smd[NW];
    __shared__ float smf[NW];
    __shared__ int smi[NW];
    const int t = threadIdx.x;
    const int64_t K4 = a.K / 4;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const XT* x = static_cast<const XT*>(a.X) + row * a.K;
        const RT* r = RES ? static_cast<const RT*>(a.R) + row * a.K : nullptr;
        RT* h = RES && a.H ? static_cast<RT*>(a.H) + row * a.K : nullptr;
        auto sum_at = [&](int64_t i) {
            float4 v = load4(x, i);
            if constexpr (RES) {
                const float4 u = load4(r, i);
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                if constexpr (sizeof(RT) == 2) {
                    const uint2 w = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
                    v = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u),
                                    __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
                }
            }
            return v;
        };
        double rstd;
        if (mode == kRmsApply) {
            rstd = a.rstd[row];
        } else {
            double q = 0.0;
            for (int64_t i = t; i < K4; i += T) {
                const float4 v = sum_at(i);
                q = fma((double)v.x, (double)v.x, q);
                q = fma((double)v.y, (double)v.y, q);
                q = fma((double)v.z, (double)v.z, q);
                q = fma((double)v.w, (double)v.w, q);
            }
            q = block_sum<NW>(q, smd) * a.inv_k + a.eps;
            rstd = q > 0.0 ? rsqrt64(q) : 0.0;
        }
        // (h may be x or r: an element is read and written by the same thread, and not read there again)
        auto hat_at = [&](float4 v, int64_t i) {
            v.x = (float)((double)v.x * rstd);
            v.y = (float)((double)v.y * rstd);
            v.z = (float)((double)v.z * rstd);
            v.w = (float)((double)v.w * rstd);
            if (a.gain) {
                const float4 g = load4(a.gain, i);
                v.x *= g.x; v.y *= g.y; v.z *= g.z; v.w *= g.w;
            }
            return v;
        };
        float gamma;
        if (mode == kRmsApply) {
            gamma = *a.gamma;
        } else {
            float m = 0.f;
            for (int64_t i = t; i < K4; i += T) {
                const float4 v = sum_at(i), o = hat_at(v, i);
                m = fmaxf(m, fmaxf(fmaxf(fabsf(o.x), fabsf(o.y)), fmaxf(fabsf(o.z), fabsf(o.w))));
            }
            m = block_max<NW>(m, smf);
            if (mode == kRmsStats) {
                if (t == 0) {
                    a.rstd[row] = rstd;
                    a.most[row] = m;
                }
                if (h)
                    for (int64_t i = t; i < K4; i += T) store4(h, i, sum_at(i));
                __syncthreads();  // the slots of the reductions are read
                continue;
            }
            gamma = fmaxf(m, 1e-5f);
        }
        const float scale = 128.0f / gamma;
        uint32_t* c4 = reinterpret_cast<uint32_t*>(a.codes + row * a.K);
        int rs = 0;
        for (int64_t i = t; i < K4; i += T) {
            const float4 v = sum_at(i), o = hat_at(v, i);
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
}

// gamma of the tensor from the rows' largest values
__global__ __launch_bounds__(1024) void fold_most(const float* __restrict__ most, int64_t M, float* __restrict__ gamma) {
    constexpr int NW = 16;
    __shared__ float sm[NW];
    float m = 0.f;
    for (int64_t i = threadIdx.x; i < M; i += 1024) m = fmaxf(m, most[i]);
    m = block_max<NW>(m, sm);
    if (threadIdx.x == 0) *gamma = fmaxf(m, 1e-5f);
}

template <typename XT, typename RT, bool RES>
static void launch_rms_typed(const QuantRmsArgs& a, int mode, hipStream_t s) {
    const unsigned grid = (unsigned)(a.M < (1 << 20) ? a.M : (1 << 20));
    quant_rms_long<XT, RT, RES><<<grid, 512, 0, s>>>(a, mode);
}
static void launch_rms(const QuantRmsArgs& a, int mode, hipStream_t s) {
    if (!a.R) {
        if (a.x_bf16) launch_rms_typed<uint16_t, uint16_t, false>(a, mode, s);
        else launch_rms_typed<float, float, false>(a, mode, s);
    } else if (a.x_bf16) {
        if (a.h_bf16) launch_rms_typed<uint16_t, uint16_t, true>(a, mode, s);
        else launch_rms_typed<uint16_t, float, true>(a, mode, s);
    } else {
        if (a.h_bf16) launch_rms_typed<float, uint16_t, true>(a, mode, s);
        else launch_rms_typed<float, float, true>(a, mode, s);
    }
}

hipError_t launch_quant_rmsnorm(const QuantRmsArgs& a_in, hipStream_t s) {
    QuantRmsArgs a = a_in;
    a.inv_k = 1.0 / (double)a.K;
    if (!a.per_tensor) {
        launch_rms(a, kRmsFull, s);
        return hipGetLastError();
    }
    launch_rms(a, kRmsStats, s);
    fold_most<<<1, 1024, 0, s>>>(a.most, a.M, a.gamma);
    if (a.R && a.H) {  // x + r is there now
        a.X = a.H;
        a.x_bf16 = a.h_bf16;
        a.R = nullptr;
        a.H = nullptr;
    }
    launch_rms(a, kRmsApply, s);
    return hipGetLastError();
}

// ---- backward -----------------------------------------------------------------------------------------
// Workgroup b takes rows b, b + groups, ...; a thread has the same columns of all of them, so their share of dgain is
// summed where only it writes.
int rms_backward_groups(int64_t M, int64_t K) {
    (void)K;
    return (int)(M < 256 ? M : 256);
}
template <typename GT, typename HT, typename DT>
__global__ __launch_bounds__(512) void rms_backward_long(RmsBackwardArgs a) {
    constexpr int NW = 8, T = NW * kWave;
    __shared__ double smd[2][NW];
    const int t = threadIdx.x;
    const int64_t K4 = a.K / 4;
    double* const part = a.dgain ? a.partials + (int64_t)blockIdx.x * a.K : nullptr;
    for (int64_t row = blockIdx.x; row < a.M; row += gridDim.x) {
        const GT* g = static_cast<const GT*>(a.G) + row * a.K;
        const HT* h = static_cast<const HT*>(a.H) + row * a.K;
        const DT* dr = a.dR ? static_cast<const DT*>(a.dR) + row * a.K : nullptr;
        DT* dh = static_cast<DT*>(a.dH) + row * a.K;
        auto scaled = [&](float4 v, int64_t i) {
            if (a.gain) {
                const float4 w = load4(a.gain, i);
                v.x *= w.x; v.y *= w.y; v.z *= w.z; v.w *= w.w;
            }
            return v;
        };
        double q = 0.0, c = 0.0;
        for (int64_t i = t; i < K4; i += T) {
            const float4 v = load4(h, i), u = scaled(load4(g, i), i);
            q = fma((double)v.x, (double)v.x, q);
            q = fma((double)v.y, (double)v.y, q);
            q = fma((double)v.z, (double)v.z, q);
            q = fma((double)v.w, (double)v.w, q);
            c = fma((double)v.x, (double)u.x, c);
            c = fma((double)v.y, (double)u.y, c);
            c = fma((double)v.z, (double)u.z, c);
            c = fma((double)v.w, (double)u.w, c);
        }
        q = block_sum<NW>(q, smd[0]) * a.inv_k + a.eps;
        c = block_sum<NW>(c, smd[1]) * a.inv_k;
        const double rstd = q > 0.0 ? rsqrt64(q) : 0.0;
        const double along = c * rstd * rstd;  // mean(t n) / rms
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
__global__ __launch_bounds__(256) void fold_dgain(const double* __restrict__ part, int groups, int64_t K,
                                                  float* __restrict__ dgain) {
    for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < K; k += (int64_t)gridDim.x * 256) {
        double s = 0.0;
        for (int b = 0; b < groups; ++b) s += part[b * K + k];
        dgain[k] = (float)s;
    }
}

template <typename GT, typename HT>
static void launch_rms_backward_typed(const RmsBackwardArgs& a, unsigned grid, hipStream_t s) {
    if (a.d_bf16) rms_backward_long<GT, HT, uint16_t><<<grid, 512, 0, s>>>(a);
    else rms_backward_long<GT, HT, float><<<grid, 512, 0, s>>>(a);
}
hipError_t launch_rmsnorm_backward(const RmsBackwardArgs& a_in, hipStream_t s) {
    RmsBackwardArgs a = a_in;
    a.inv_k = 1.0 / (double)a.K;
    const unsigned grid = (unsigned)rms_backward_groups(a.M, a.K);
    if (a.g_bf16) {
        if (a.h_bf16) launch_rms_backward_typed<uint16_t, uint16_t>(a, grid, s);
        else launch_rms_backward_typed<uint16_t, float>(a, grid, s);
    } else {
        if (a.h_bf16) launch_rms_backward_typed<float, uint16_t>(a, grid, s);
        else launch_rms_backward_typed<float, float>(a, grid, s);
    }
    if (a.dgain) {
        const int64_t wgs = (a.K + 255) / 256;
        fold_dgain<<<(unsigned)(wgs < 65536 ? wgs : 65536), 256, 0, s>>>(a.partials, (int)grid, a.K, a.dgain);
    }
    return hipGetLastError();
}

}  // namespace bl
