// Between the two projections of a feed-forward network of BitLinear layers: a non-linear function f, the LayerNorm of
// Eq. 12 and the 8-bit quantiser of Eq. 4-5 in one pass over the first projection's output u, with an optional 8-bit
// checkpoint of u; and the backward pass, from that checkpoint.
//   forward    h = f(u), x^ = (h - mean h) / sqrt(var h + eps), gamma = max|x^|, code = clamp(rne(x^ * (128 / gamma)))
//              checkpoint, per block b of 128 elements of a row: c = rne(u * (127 / amax_b)), kept beside amax_b / 127
//              (amax_b, where not zero, at least kLeastMax; -128 for what the marked rectifier tells from zero)
//   backward   v = c * (amax_b / 127), h = f(v), n = (h - mean h) / sqrt(var h + eps)
//              du = f'(v) * (g - mean g - n mean(g n)) / sqrt(var h + eps),  g = the gradient of x^
// The backward is the derivative of the forward at v, exactly: its statistics are those of f(v), which come out of the
// row that is in registers anyway, and nothing but the checkpoint has to be kept (1.03 bytes an element where u has
// four).  f and f' are evaluated in fp32, the sums of a row in fp64 (as in the quantiser and in the LayerNorm
// backward). Bound by HBM: 4 bytes read and 1 (with the checkpoint 2) written an element, twice the reading with a
// gamma per tensor; backward 5 read, 2 or 4 written.
#include "common.h"
#include "experts.h"
#include "kernels.h"
#include "rowops.h"

namespace bl {

enum Fn { kRelu = 0, kRelu2 = 1, kGelu = 2, kSilu = 3, kReluMarked = 8 };
enum RowMode { kOnce = 0, kRowStats = 1, kRowApply = 2 };

// f(u) of the forward, whose codes are decided next to a border: the library's functions, an ulp or so off.
template <int FN>
__device__ inline float fn_value(float u) {
    if constexpr (FN == kRelu || FN == kReluMarked) return u > 0.f ? u : 0.f;
    else if constexpr (FN == kRelu2) return u > 0.f ? u * u : 0.f;
    else if constexpr (FN == kGelu) return 0.5f * u * (1.f + erff(u * 0.70710678118654752f));
    else return u / (1.f + expf(-u));
}
// f(v) and f'(v) of the backward, where they are factors of a gradient.  GELU: Phi(u) = (1 + erf(z)) / 2, z = u / sqrt
// 2, with erf as in Abramowitz and Stegun 7.1.26 (erf z = 1 - (a1 t + ... + a5 t^5) e^(-z^2), t = 1 / (1 + p z), z >=
// 0: off by at most 1.5e-7), which shares its exponential with f'.  The hardware's exponential and reciprocal are off
// by an ulp.  (16384 x 8192 with the library's erff and expf 455 us, 219 so.  The forward would gain 14 %, and a code
// in a million fall on the other side of a border.)
struct FnPair {
    float value, slope;
};
template <int FN>
__device__ inline FnPair fn_pair(float u) {
    if constexpr (FN == kRelu) {
        return {u > 0.f ? u : 0.f, u > 0.f ? 1.f : 0.f};
    } else if constexpr (FN == kRelu2) {
        const float r = u > 0.f ? u : 0.f;
        return {r * r, 2.f * r};
    } else if constexpr (FN == kGelu) {
        const float z = fabsf(u) * 0.70710678118654752f;
        const float e = __builtin_amdgcn_exp2f(u * u * -0.72134752044448170f);  // e^(-u^2 / 2)
        const float t = __builtin_amdgcn_rcpf(fmaf(z, 0.3275911f, 1.f));
        float p = fmaf(1.061405429f, t, -1.453152027f);
        p = fmaf(fmaf(fmaf(p, t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
        const float tail = 0.5f * (p * t * e);  // Phi(-|u|)
        const float phi = u < 0.f ? tail : 1.f - tail;
        return {u * phi, fmaf(u * 0.39894228040143268f, e, phi)};
    } else {
        const float s = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u * -1.4426950408889634f));
        return {u * s, fmaf(u * s, 1.f - s, s)};
    }
}
// A rectifier's slope jumps at zero, and what is positive and rounds to zero would lose its whole gradient: of 8192 values
// N(0,1) 9.3 % of the norm, N(-2,1) 20 %, one in a hundred 30 times as large 26 % (squared rectifier, GELU and SiLU 0.4 to
// 5.3 %, the rounding of f and f' themselves).  The marked one stores -128 there, which no rounding gives: value 0, slope 1,
// and 0.02, 0.27 and 0.07 % are left.  (The other functions are smooth at zero.)
template <int FN>
__device__ inline FnPair code_pair(int8_t code, float scale) {
    if constexpr (FN == kReluMarked) {
        const bool marked = code == -128;
        return {code > 0 ? (float)code * scale : 0.f, code > 0 || marked ? 1.f : 0.f};
    } else {
        return fn_pair<FN>((float)code * scale);
    }
}
// the largest value of 32 lanes, one half of a wave
__device__ inline float half_wave_max(float v) {
    v = max_raw(v, dpp_mov<0xB1>(v));
    v = max_raw(v, dpp_mov<0x4E>(v));
    v = max_raw(v, dpp_mov<0x141>(v));
    v = max_raw(v, dpp_mov<0x140>(v));
    float lo, hi;
    lane_swap<false>(v, lo, hi);
    return max_raw(lo, hi);
}

// Of a block of tiny values 127 / m passes the largest float (m < 3.7e-37), and its zeros would be 0 * inf: its step m / 127
// is taken to be 2^-127.
constexpr float kLeastMax = 127.f * 0x1p-127f;

// WPR waves share a row, a lane holds NV float4 of it.  kRowStats and kRowApply: the two passes of a gamma per tensor;
// the first leaves the row's statistics in rowstats and its largest magnitude where its codes will be, which nobody
// writes before the second.
template <int FN, int WPR, int NV, int MODE>
__global__ __launch_bounds__((WPR < 4 ? 4 : WPR) * kWave) void nonlinear_rows(NonlinearArgs a) {
    constexpr int NW = WPR < 4 ? 4 : WPR, RPW = NW / WPR, RT = WPR * kWave;
    __shared__ double sm_k[2 * NW];
    __shared__ float sm_f[2 * NW];
    __shared__ int smi[NW];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int rw = wave / WPR, wr = wave % WPR;
    const int t = wr * kWave + (threadIdx.x & (kWave - 1));
    const int64_t M = a.rows ? (*a.rows < a.M ? *a.rows : a.M) : a.M;
    int64_t row = (int64_t)blockIdx.x * RPW + rw;
    if ((int64_t)blockIdx.x * RPW >= M) return;  // uniform for the workgroup
    const bool live = row < M;
    if (!live) row = M - 1;
    const int K4 = (int)(a.K / 4);
    const float4* __restrict__ x4 = reinterpret_cast<const float4*>(a.U + row * a.K);

    float4 v[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int idx = t + j * RT;
        v[j] = x4[(uint32_t)(idx < K4 ? idx : K4 - 1)];
    }
    const float first = fn_value<FN>(a.U[row * a.K]);

    if (MODE != kRowApply && a.check) {  // uniform
        uint32_t* __restrict__ c4 = reinterpret_cast<uint32_t*>(a.check + row * a.K);
        const int blocks = (int)((a.K + kCheckBlock - 1) / kCheckBlock);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int idx = t + j * RT;
            const bool in = idx < K4;
            const float4 x = v[j];
            const float mine = max_raw(max_raw(fabsf(x.x), fabsf(x.y)), max_raw(fabsf(x.z), fabsf(x.w)));
            float big = half_wave_max(in ? mine : 0.f);
            big = big > 0.f ? max_raw(big, kLeastMax) : 0.f;
            const float up = big > 0.f ? 127.f / big : 0.f;
            if (in && live) {
                if constexpr (FN == kReluMarked) {
                    auto marked = [&](float u) { return u > 0.f && u * up <= 0.5f ? -128.f : u * up; };
                    c4[idx] = code_word(marked(x.x), marked(x.y), marked(x.z), marked(x.w));
                } else {
                    c4[idx] = code_word(x.x * up, x.y * up, x.z * up, x.w * up, -127.f);
                }
                if ((t & 31) == 0) a.check_scale[row * blocks + (idx >> 5)] = big / 127.f;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        v[j].x = fn_value<FN>(v[j].x);
        v[j].y = fn_value<FN>(v[j].y);
        v[j].z = fn_value<FN>(v[j].z);
        v[j].w = fn_value<FN>(v[j].w);
        // Long rows: one float4 after the other, or all of them are under way at once in 111 registers (GELU) and no
        // second workgroup hides this one's loads: per token 2000 x 28672 111 -> 87 us, 8000 x 16384 193 -> 166.  Up to
        // four float4 fit as they are, and a few short rows are 0.2 us of 5.5 faster so.
        if constexpr (NV >= 8)
            if (j + 1 < NV)
                asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w), "+v"(v[j + 1].x),
                                  "+v"(v[j + 1].y), "+v"(v[j + 1].z), "+v"(v[j + 1].w));
    }

    const float cf = stats_centre(first);
    const double c = (double)cf;
    RowNorm n;
    float amax = 0.f;
    if constexpr (MODE == kRowApply) {
        n.shift = a.rowstats[2 * row];
        n.rstd = a.rowstats[2 * row + 1];
    } else {
        RowStats rs;
        rs.mx = cf;
        rs.nmn = -cf;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (K4 < (j + 1) * RT) {  // uniform: this piece of the row is ragged
                const bool in = t + j * RT < K4;
                v[j].x = in ? v[j].x : cf;
                v[j].y = in ? v[j].y : cf;
                v[j].z = in ? v[j].z : cf;
                v[j].w = in ? v[j].w : cf;
            }
            double d[4];
            stats_add(rs, v[j], c, d);
        }
        PairStats st = stats_wave(rs);
        if constexpr (WPR > 1) {
            stats_leave(st, sm_k, sm_f, wave);
            __syncthreads();
            st = stats_fold(sm_k + 2 * rw * WPR, sm_f + 2 * rw * WPR, WPR);
        }
        float lo, hi;
        n = stats_finish(st, c, a.inv_k, (double)a.eps, lo, hi);
        amax = fmaxf(fabsf(lo), fabsf(hi));  // h -> x^ is monotone
        if constexpr (MODE == kRowStats) {
            if (t == 0 && live) {
                a.rowstats[2 * row] = n.shift;
                a.rowstats[2 * row + 1] = n.rstd;
                reinterpret_cast<uint32_t*>(a.codes)[row] = __float_as_uint(amax);
            }
            return;
        }
    }
    const float gamma = fmaxf(MODE == kRowApply ? __uint_as_float(*a.gmax_bits) : amax, 1e-5f);
    const float scale = 128.0f / gamma;
    int sum = 0;
    uint32_t* __restrict__ q4 = reinterpret_cast<uint32_t*>(a.codes + row * a.K);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int idx = t + j * RT;
        // (hidden from the optimiser, which would keep what the sums made of them alive)
        if constexpr (MODE == kOnce && NV >= 8) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
        auto scaled = [&](float h) { return normalised(n, (double)h - c) * scale; };
        const uint32_t wd = code_word(scaled(v[j].x), scaled(v[j].y), scaled(v[j].z), scaled(v[j].w));
        if (idx < K4) {
            sum = __builtin_amdgcn_sdot4((int)wd, 0x01010101, sum, false);
            if (live) q4[(uint32_t)idx] = wd;
        }
    }
    if (a.rowsum) {  // uniform
        sum = row_reduce<WPR>(sum, OpSum{}, smi, rw, wr);
        if (t == 0 && live) a.rowsum[row] = sum;
    }
    if (t == 0 && live && (MODE == kOnce || row == 0)) a.gamma[row] = gamma;
}

// the largest of the rows' magnitudes (non-negative floats order like their bit patterns)
__global__ __launch_bounds__(1024) void nonlinear_fold(NonlinearArgs a) {
    constexpr int NW = 16;
    __shared__ float sm[NW];
    const int64_t M = a.rows ? (*a.rows < a.M ? *a.rows : a.M) : a.M;
    float most = 0.f;
    const float* const rows = reinterpret_cast<const float*>(a.codes);
    for (int64_t i = threadIdx.x; i < M; i += 8 * 1024) {  // eight loads in flight; behind the last row that one again
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = rows[i + u * 1024 < M ? i + u * 1024 : M - 1];
#pragma unroll
        for (int u = 0; u < 8; ++u) most = max_raw(most, v[u]);
    }
    most = wave_reduce(most, OpMax{});
    if (threadIdx.x % kWave == 0) sm[threadIdx.x / kWave] = most;
    __syncthreads();
    if (threadIdx.x >= kWave) return;
    most = fold_slots<NW>(sm, OpMax{});
    if (threadIdx.x != 0) return;
    *a.gmax_bits = __float_as_uint(most);
    if (M <= 0) *a.gamma = 1e-5f;  // no row to write the lower bound of gamma
}

// ---- backward -----------------------------------------------------------------------------------------
// One reading of the row: g, and of the checkpoint f(v) and f'(v), stay in registers; the four sums that the derivative
// of the LayerNorm needs (of h, h^2, g and g h) are taken together.  With eight float4 a lane and 16 waves a row, which
// have 128 registers, the pairs are evaluated a second time instead of kept (2000 x 28672: 473 us kept and spilled, 148
// so).
template <int FN, int WPR, int NV>
__global__ __launch_bounds__((WPR < 4 ? 4 : WPR) * kWave) void nonlinear_backward_rows(NonlinearArgs a) {
    constexpr int NW = WPR < 4 ? 4 : WPR, RPW = NW / WPR, RT = WPR * kWave;
    __shared__ double smd[4][NW];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int rw = wave / WPR, wr = wave % WPR;
    const int t = wr * kWave + (threadIdx.x & (kWave - 1));
    const int64_t M = a.rows ? (*a.rows < a.M ? *a.rows : a.M) : a.M;
    int64_t row = (int64_t)blockIdx.x * RPW + rw;
    if ((int64_t)blockIdx.x * RPW >= M) return;  // uniform for the workgroup
    const bool live = row < M;
    if (!live) row = M - 1;
    const int K4 = (int)(a.K / 4);
    const int blocks = (int)((a.K + kCheckBlock - 1) / kCheckBlock);
    const float4* __restrict__ g4 = reinterpret_cast<const float4*>(a.dXhat + row * a.K);
    const uint32_t* __restrict__ c4 = reinterpret_cast<const uint32_t*>(a.check + row * a.K);
    const float* __restrict__ scales = a.check_scale + row * blocks;

    constexpr bool KEEP = NV < 8 || WPR < 16;
    float4 g[NV], h[KEEP ? NV : 1], f[KEEP ? NV : 1];
    uint32_t q[NV];
    float sc[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int idx = t + j * RT, at = idx < K4 ? idx : K4 - 1;
        g[j] = g4[(uint32_t)at];
        q[j] = c4[(uint32_t)at];
        sc[j] = scales[(uint32_t)at >> 5];
    }
    // sums about an element of the row, so that a large common offset costs nothing
    const double c = (double)code_pair<FN>((int8_t)c4[0], scales[0]).value;
    auto pairs = [](uint32_t codes, float scale, float4& value, float4& slope) {
        const FnPair x = code_pair<FN>((int8_t)codes, scale);
        const FnPair y = code_pair<FN>((int8_t)(codes >> 8), scale);
        const FnPair z = code_pair<FN>((int8_t)(codes >> 16), scale);
        const FnPair w = code_pair<FN>((int8_t)(codes >> 24), scale);
        value = make_float4(x.value, y.value, z.value, w.value);
        slope = make_float4(x.slope, y.slope, z.slope, w.slope);
    };
    double s[4] = {0.0, 0.0, 0.0, 0.0};  // of h - c, (h - c)^2, g, g (h - c)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int k = KEEP ? j : 0;
        pairs(q[j], sc[j], h[k], f[k]);
        if (K4 < (j + 1) * RT && t + j * RT >= K4) {  // behind the row: nothing to the sums
            h[k] = make_float4((float)c, (float)c, (float)c, (float)c);
            g[j] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        auto add = [&](float value, float d) {
            const double x = (double)value - c;
            s[0] += x;
            s[1] = fma(x, x, s[1]);
            s[2] += (double)d;
            s[3] = fma((double)d, x, s[3]);
        };
        add(h[k].x, g[j].x);
        add(h[k].y, g[j].y);
        add(h[k].z, g[j].z);
        add(h[k].w, g[j].w);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = wave_reduce(s[i], OpSum{});
    if constexpr (WPR > 1) {
        if ((threadIdx.x & (kWave - 1)) == 0)
            for (int i = 0; i < 4; ++i) smd[i][wave] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fold_slots<WPR>(smd[i] + rw * WPR, OpSum{});
    }
    const double dm = s[0] * a.inv_k, var = fmax(fma(-dm, dm, s[1] * a.inv_k), 0.0);
    const double rstd = rsqrt64(var + (double)a.eps);
    const float r = (float)rstd;
    const float m1 = (float)(s[2] * a.inv_k), m2 = (float)((s[3] - dm * s[2]) * rstd * a.inv_k);
    const double nshift = -(dm * rstd);
    // hide them from the optimiser, which would keep what the sums made of them alive
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if constexpr (KEEP) asm volatile("" : "+v"(h[j].x), "+v"(h[j].y), "+v"(h[j].z), "+v"(h[j].w));
        else asm volatile("" : "+v"(q[j]), "+v"(sc[j]));
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int idx = t + j * RT, k = KEEP ? j : 0;
        if constexpr (!KEEP) pairs(q[j], sc[j], h[k], f[k]);
        auto du = [&](float value, float slope, float d) {
            const float n = (float)fma((double)value - c, rstd, nshift);
            return r * ((d - m1) - n * m2) * slope;
        };
        const float x = du(h[k].x, f[k].x, g[j].x), y = du(h[k].y, f[k].y, g[j].y);
        const float z = du(h[k].z, f[k].z, g[j].z), w = du(h[k].w, f[k].w, g[j].w);
        if (idx < K4 && live) {
            if (a.bf16)
                reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.dU) + row * a.K)[(uint32_t)idx] =
                    make_uint2(bf16_word(x, y), bf16_word(z, w));
            else
                reinterpret_cast<float4*>(reinterpret_cast<float*>(a.dU) + row * a.K)[(uint32_t)idx] =
                    make_float4(x, y, z, w);
        }
    }
}

// Waves a row and float4 a lane.  A batch of few rows is the length of one row's chain: more waves share it, down to
// two float4 a lane; a large one is bound by HBM.
struct RowShape {
    int wpr, nv;
};
static RowShape row_shape(int64_t M, int64_t K) {
    const int64_t K4 = K / 4;
    int wpr = 1, nv = 2;
    auto wider = [&]() { wpr = wpr == 1 ? 4 : wpr * 2; };
    while (wpr < 16 && K4 > (int64_t)wpr * kWave * 8) wider();
    // (us, forward / backward: 32 x 8192 with 4, 8, 16 waves 4.9 / 6.8, 4.3 / 5.0, 4.6 / 5.6; 32 x 2048 with 1, 4, 8
    // 4.4 / 6.6, 3.0 / 3.1, 3.4 / 3.5; 16384 x 8192 with 4, 8, 16 126 / 219, 144 / 216, 194 / 297)
    while (wpr < 8 && M * wpr <= 1024 && K4 > (int64_t)wpr * kWave * 2) wider();
    if (const int v = tuning().quant_wpr)
        if ((v == 1 || v == 4 || v == 8) && K4 <= (int64_t)v * kWave * 8) wpr = v;
    while ((int64_t)wpr * kWave * nv < K4) nv *= 2;
    return {wpr, nv};
}

template <int FN, int WPR, int NV>
static void launch_forward(const NonlinearArgs& a, hipStream_t s) {
    constexpr int NW = WPR < 4 ? 4 : WPR, RPW = NW / WPR;
    const unsigned grid = (unsigned)((a.M + RPW - 1) / RPW);
    if (!a.per_tensor) {
        nonlinear_rows<FN, WPR, NV, kOnce><<<grid, NW * kWave, 0, s>>>(a);
        return;
    }
    nonlinear_rows<FN, WPR, NV, kRowStats><<<grid, NW * kWave, 0, s>>>(a);
    nonlinear_fold<<<1, 1024, 0, s>>>(a);
    constexpr int VALUE = FN == kReluMarked ? kRelu : FN;  // no checkpoint in this pass
    nonlinear_rows<VALUE, WPR, NV, kRowApply><<<grid, NW * kWave, 0, s>>>(a);
}
template <int FN, int WPR, int NV>
static void launch_backward_rows(const NonlinearArgs& a, hipStream_t s) {
    constexpr int NW = WPR < 4 ? 4 : WPR, RPW = NW / WPR;
    nonlinear_backward_rows<FN, WPR, NV><<<(unsigned)((a.M + RPW - 1) / RPW), NW * kWave, 0, s>>>(a);
}

template <int FN>
static hipError_t launch_fn(const NonlinearArgs& a_in, bool backward, hipStream_t s) {
    NonlinearArgs a = a_in;
    a.inv_k = 1.0 / (double)a.K;
    const RowShape q = row_shape(a.M, a.K);
#define BL_ROWS(W, V)                                        \
    if (q.wpr == W && q.nv == V) {                           \
        if (backward) launch_backward_rows<FN, W, V>(a, s);  \
        else launch_forward<FN, W, V>(a, s);                 \
    } else
    BL_ROWS(1, 2) BL_ROWS(1, 4) BL_ROWS(1, 8) BL_ROWS(4, 2) BL_ROWS(4, 4) BL_ROWS(4, 8) BL_ROWS(8, 2) BL_ROWS(8, 4)
    BL_ROWS(8, 8) BL_ROWS(16, 8)  // (16 waves: more than 8 hold)
    return hipErrorInvalidValue;
#undef BL_ROWS
    return hipGetLastError();
}
static hipError_t launch_any(const NonlinearArgs& a, int fn, bool backward, hipStream_t s) {
    switch (fn) {
        case kRelu: return launch_fn<kRelu>(a, backward, s);
        case kRelu2: return launch_fn<kRelu2>(a, backward, s);
        case kGelu: return launch_fn<kGelu>(a, backward, s);
        case kReluMarked: return launch_fn<kReluMarked>(a, backward, s);
        default: return launch_fn<kSilu>(a, backward, s);
    }
}
hipError_t launch_quant_nonlinear(const NonlinearArgs& a, int fn, hipStream_t s) {
    return launch_any(a, fn, false, s);
}
hipError_t launch_nonlinear_backward(const NonlinearArgs& a, int fn, hipStream_t s) {
    return launch_any(a, fn, true, s);
}

}  // namespace bl
