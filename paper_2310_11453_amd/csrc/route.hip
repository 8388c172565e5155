// Tokens to experts and back, for a mixture of BitLinear layers.
//   route     a stable counting sort of the router's choices: slot s of expert e holds the choice order[s] = t top_k + j,
//             position is the inverse, offsets[e] the first slot of expert e
//   combine   Y[t] = sum_j w[t,j] Ys[position[t,j]], j in ascending order
//   combine's gradient: dYs[position[t,j]] = w[t,j] dY[t] (every slot belongs to one choice, so nothing is added and no
//             order matters), dw[t,j] = <dY[t], Ys[position[t,j]]>
// The sort is bound by latency, the other two by HBM: each row is read and written once.
#include "common.h"
#include "experts.h"

namespace bl {

namespace route {
constexpr int kThreads = 1024, kRows = 64;        // rows of 64 choices
constexpr int kChunk = kRows * kWave;             // choices of a workgroup
constexpr int kRowsWave = kRows / (kThreads / kWave);
}  // namespace route

// The place of a choice inside its expert is the number of earlier choices of that expert: of earlier workgroups
// (counts), of earlier rows of 64 of this workgroup (cnt, summed down the rows) and of lower lanes of its row (a ballot for
// each bit of the expert's number).  Nothing depends on which wave is first.
// COUNT: only this workgroup's choices of each expert are counted, for the launch that follows.
template <bool COUNT>
__global__ __launch_bounds__(route::kThreads) void route_kernel(RouteArgs a, int bits) {
    using namespace route;
    __shared__ uint16_t cnt[kRows][kMaxExperts];
    __shared__ uint32_t base[kMaxExperts + 1], wave_sums[kMaxExperts / kWave];
    const uint32_t c0 = blockIdx.x * kChunk, n = a.T - c0 < kChunk ? a.T - c0 : kChunk;
    const int l = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    const int nrows = (int)((n + kWave - 1) / kWave);
    for (int i = threadIdx.x; i < nrows * kMaxExperts; i += blockDim.x) (&cnt[0][0])[i] = 0;
    __syncthreads();
    uint32_t id[kRowsWave], rank[kRowsWave];
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const int r = it * (kThreads / kWave) + w;
        const uint32_t i = (uint32_t)(r * kWave + l);
        id[it] = i < n ? (uint32_t)a.expert[c0 + i] : 0xffffffffu;
        const bool in = id[it] < a.E;
        uint64_t same = __ballot(in);
        for (int b = 0; b < bits; ++b) {
            const bool set = (id[it] >> b) & 1;
            const uint64_t bal = __ballot(set);
            same &= set ? bal : ~bal;
        }
        rank[it] = (uint32_t)__popcll(same & (((uint64_t)1 << l) - 1));
        if (in && rank[it] == 0) cnt[r][id[it]] = (uint16_t)__popcll(same);
    }
    __syncthreads();
    // thread e: expert e's choices in the rows above each row, in this workgroup, before it and in all
    const uint32_t e = threadIdx.x;
    uint32_t mine = 0, before = 0, all = 0;
    if (e < a.E) {
        for (int r = 0; r < nrows; ++r) {
            const uint32_t c = cnt[r][e];
            cnt[r][e] = (uint16_t)mine;
            mine += c;
        }
        if constexpr (COUNT) {
            a.counts[blockIdx.x * a.E + e] = mine;
        } else if (gridDim.x > 1) {
            for (uint32_t b = 0; b < gridDim.x; ++b) {
                const uint32_t c = a.counts[b * a.E + e];
                before += b < blockIdx.x ? c : 0;
                all += c;
            }
        } else {
            all = mine;
        }
    }
    if constexpr (COUNT) return;
    if (e < kMaxExperts) {  // whole waves: a scan over the experts
        uint32_t v = all;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)v, d, kWave);
            if (l >= d) v += o;
        }
        if (l == kWave - 1) wave_sums[w] = v;
        base[e + 1] = v;
    }
    __syncthreads();
    uint32_t lower = 0;
    if (e < kMaxExperts)
        for (int i = 0; i < w; ++i) lower += wave_sums[i];
    const uint32_t end = e < kMaxExperts ? base[e + 1] + lower : 0;
    __syncthreads();
    if (e < a.E) {
        if (blockIdx.x == 0) {
            a.offsets[e + 1] = (int32_t)end;
            if (e == 0) a.offsets[0] = 0;
        }
        base[e] = end - all + before;
        if (e == a.E - 1) base[kMaxExperts] = end;
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const int r = it * (kThreads / kWave) + w;
        const uint32_t i = (uint32_t)(r * kWave + l);
        if (i >= n) continue;
        int32_t at = -1;
        if (id[it] < a.E) {
            at = (int32_t)(base[id[it]] + cnt[r][id[it]] + rank[it]);
            a.order[at] = (int32_t)(c0 + i);
        }
        a.position[c0 + i] = at;
        if (c0 + i >= base[kMaxExperts]) a.order[c0 + i] = -1;
    }
}

int64_t route_blocks(int64_t T) { return (T + route::kChunk - 1) / route::kChunk; }

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    const unsigned blocks = (unsigned)route_blocks(a.T);
    int bits = 0;
    while ((1u << bits) < a.E) ++bits;
    if (blocks > 1) route_kernel<true><<<blocks, route::kThreads, 0, s>>>(a, bits);
    route_kernel<false><<<blocks, route::kThreads, 0, s>>>(a, bits);
    return hipGetLastError();
}

// ---- slots back to tokens ---------------------------------------------------------------------------
__device__ inline uint32_t bf16_rne(float v) {
    uint32_t u = __float_as_uint(v);
    u += 0x7fffu + ((u >> 16) & 1u);
    return u >> 16;
}

// A workgroup: a token and 256 pieces of its row, of four elements (VEC: N % 4 == 0) or one; items beyond the grid in turn.
template <bool VEC>
__device__ inline void combine_piece(const CombineArgs& a, int64_t t, int64_t n) {
    constexpr int E = VEC ? 4 : 1;
    float y[E] = {};
    for (int j = 0; j < a.top_k; ++j) {
        const uint32_t at = (uint32_t)a.position[t * a.top_k + j];
        if (at >= (uint64_t)a.T) continue;  // no expert took this choice
        const float wt = a.weights ? a.weights[t * a.top_k + j] : 1.f;
        const float* src = a.slots + (int64_t)at * a.N + n;
        if constexpr (VEC) {
            const float4 v = *reinterpret_cast<const float4*>(src);
            y[0] += wt * v.x, y[1] += wt * v.y, y[2] += wt * v.z, y[3] += wt * v.w;
        } else {
            y[0] += wt * *src;
        }
    }
    if constexpr (VEC) *reinterpret_cast<float4*>(a.Y + t * a.N + n) = make_float4(y[0], y[1], y[2], y[3]);
    else a.Y[t * a.N + n] = y[0];
}
template <bool VEC>
__global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    constexpr int E = VEC ? 4 : 1;
    for (int64_t t = blockIdx.x; t < a.M; t += gridDim.x)
        for (int64_t n = ((int64_t)blockIdx.y * 256 + threadIdx.x) * E; n < a.N; n += (int64_t)gridDim.y * 256 * E)
            combine_piece<VEC>(a, t, n);
}

// A workgroup: a token; its choices one after another, the token's row out of the cache from the second on.
template <bool VEC>
__device__ inline void combine_backward_token(const CombineArgs& a, int64_t t, float (&sums)[4]) {
    constexpr int E = VEC ? 4 : 1;
    for (int j = 0; j < a.top_k; ++j) {
        const uint32_t at = (uint32_t)a.position[t * a.top_k + j];
        if (at >= (uint64_t)a.T) {  // uniform
            if (a.dWeights && threadIdx.x == 0) a.dWeights[t * a.top_k + j] = 0.f;
            continue;
        }
        const float wt = a.weights ? a.weights[t * a.top_k + j] : 1.f;
        float dot = 0.f;
        for (int64_t n = (int64_t)threadIdx.x * E; n < a.N; n += 256 * E) {
            const float* g = a.dY + t * a.N + n;
            const int64_t o = (int64_t)at * a.N + n;
            if constexpr (VEC) {
                const float4 v = *reinterpret_cast<const float4*>(g);
                *reinterpret_cast<uint2*>(a.dSlots + o) =
                    make_uint2(bf16_rne(wt * v.x) | bf16_rne(wt * v.y) << 16, bf16_rne(wt * v.z) | bf16_rne(wt * v.w) << 16);
                if (a.dWeights) {
                    const float4 y = *reinterpret_cast<const float4*>(a.slots + o);
                    dot += (v.x * y.x + v.y * y.y) + (v.z * y.z + v.w * y.w);
                }
            } else {
                a.dSlots[o] = (uint16_t)bf16_rne(wt * *g);
                if (a.dWeights) dot += *g * a.slots[o];
            }
        }
        if (!a.dWeights) continue;
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) dot += __shfl_xor(dot, m, kWave);
        __syncthreads();
        if ((threadIdx.x & (kWave - 1)) == 0) sums[threadIdx.x / kWave] = dot;
        __syncthreads();
        if (threadIdx.x == 0) a.dWeights[t * a.top_k + j] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    }
}

template <bool VEC>
__global__ __launch_bounds__(256) void combine_backward_kernel(CombineArgs a) {
    __shared__ float sums[4];
    for (int64_t t = blockIdx.x; t < a.M; t += gridDim.x) combine_backward_token<VEC>(a, t, sums);
}

static unsigned token_grid(int64_t M) { return (unsigned)(M < (1 << 20) ? M : 1 << 20); }

hipError_t launch_combine(const CombineArgs& a, hipStream_t s) {
    const bool vec = a.N % 4 == 0 && ((uintptr_t)a.slots & 15) == 0 && ((uintptr_t)a.Y & 15) == 0;
    const int64_t per = 256 * (vec ? 4 : 1);
    const int64_t pieces = (a.N + per - 1) / per;
    const dim3 grid(token_grid(a.M), (unsigned)(pieces < 1024 ? pieces : 1024));
    if (vec) combine_kernel<true><<<grid, 256, 0, s>>>(a);
    else combine_kernel<false><<<grid, 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_combine_backward(const CombineArgs& a, hipStream_t s) {
    const bool vec = a.N % 4 == 0 && (((uintptr_t)a.slots | (uintptr_t)a.dY) & 15) == 0 && ((uintptr_t)a.dSlots & 7) == 0;
    if (vec) combine_backward_kernel<true><<<token_grid(a.M), 256, 0, s>>>(a);
    else combine_backward_kernel<false><<<token_grid(a.M), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace bl
