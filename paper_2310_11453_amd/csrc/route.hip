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
constexpr int kRowsWave = 4;  // rows of 64 choices of a wave
constexpr int kSmall = 256, kLarge = 1024;  // threads of a workgroup: up to 1024 choices, and more
constexpr int kScan = 256, kScanned = 64;   // threads of the scan, and the workgroups above which there is one
constexpr int chunk(int threads) { return threads * kRowsWave; }
}  // namespace route

// Lanes of a row whose choice is the same expert's (0 where it is none's).
__device__ inline uint64_t same_expert(uint32_t id, uint32_t E, int bits) {
    uint64_t same = __ballot(id < E);
    if (id >= E) return 0;
    for (int b = 0; b < bits; ++b) {
        const bool set = (id >> b) & 1;
        const uint64_t bal = __ballot(set);
        same &= set ? bal : ~bal;
    }
    return same;
}

// How many of a workgroup's choices are each expert's.
__global__ __launch_bounds__(route::kLarge) void route_count_kernel(RouteArgs a, int bits) {
    using namespace route;
    __shared__ uint32_t sums[kMaxExperts];
    const uint32_t c0 = blockIdx.x * chunk(kLarge), n = a.T - c0 < chunk(kLarge) ? a.T - c0 : chunk(kLarge);
    uint32_t id[kRowsWave];
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const uint32_t i = it * kLarge + threadIdx.x;
        id[it] = i < n ? (uint32_t)a.expert[c0 + i] : 0xffffffffu;
    }
    if (threadIdx.x < a.E) sums[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const uint64_t same = same_expert(id[it], a.E, bits);
        // the lowest lane of those adds for all (integers: no order matters)
        if (same && (same & (((uint64_t)1 << (threadIdx.x & (kWave - 1))) - 1)) == 0)
            atomicAdd(&sums[id[it]], (uint32_t)__popcll(same));
    }
    __syncthreads();
    if (threadIdx.x < a.E) a.counts[blockIdx.x * a.E + threadIdx.x] = sums[threadIdx.x];
}

// Of many workgroups' counts, where each workgroup's choices of an expert begin inside the expert, in place of the
// count, and how many the expert has, behind them.  blockIdx.x: the expert.  (Each workgroup adding up what it needs is
// quadratic in their number: 16777216 choices of 64 experts 779 us a call so, 134 with this, 4194304 83 and 48, 1048576
// 29 and 27, and it would be a launch for nothing at 262144, 23.)
__global__ __launch_bounds__(route::kScan) void route_scan_kernel(RouteArgs a, int blocks) {
    using namespace route;
    constexpr int kMost = (int)(kMaxRouteSlots / chunk(kLarge) / kScan);  // counts of a thread
    __shared__ int ends[kScan / kWave];
    const int per = (blocks + kScan - 1) / kScan, b0 = (int)threadIdx.x * per;
    uint32_t* const at = a.counts + blockIdx.x;
    uint32_t v[kMost];
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        v[i] = i < per && b0 + i < blocks ? at[(int64_t)(b0 + i) * a.E] : 0;
        sum += v[i];
    }
    const int end = wave_sums((int)sum), w = (int)threadIdx.x / kWave;
    if (threadIdx.x % kWave == kWave - 1) ends[w] = end;
    __syncthreads();
    uint32_t before = (uint32_t)end - sum;
    for (int i = 0; i < w; ++i) before += (uint32_t)ends[i];
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        if (i < per && b0 + i < blocks) at[(int64_t)(b0 + i) * a.E] = before;
        before += v[i];
    }
    if (threadIdx.x == kScan - 1) at[(int64_t)blocks * a.E] = before;
}

// The place of a choice inside its expert is the number of earlier choices of that expert: of earlier workgroups
// (counts), of earlier rows of 64 of this workgroup (cnt, summed down the rows) and of lower lanes of its row (a ballot
// for each bit of the expert's number).  Nothing depends on which wave is first.  Thread (p, e) sums a part of the rows
// and of the other workgroups' counts for expert e.  (One thread an expert, walking 64 rows and 16 counts one after
// another: 12.9 us for 65528 choices of 64 experts, behind a count of 6.1.)
template <int THREADS>
__global__ __launch_bounds__(THREADS) void route_kernel(RouteArgs a, int bits) {
    using namespace route;
    constexpr int kWaves = THREADS / kWave, kRows = kWaves * kRowsWave, kParts = THREADS / kMaxExperts;
    constexpr int kPart = kRows / kParts;  // rows of a part: 16
    __shared__ uint16_t cnt[kRows][kMaxExperts];
    __shared__ uint32_t part[kParts][kMaxExperts], parts_before[kParts][kMaxExperts], parts_all[kParts][kMaxExperts];
    __shared__ uint32_t base[kParts][kMaxExperts], wave_sums[kMaxExperts / kWave], end_of_all;
    const uint32_t c0 = blockIdx.x * chunk(THREADS), n = a.T - c0 < chunk(THREADS) ? a.T - c0 : chunk(THREADS);
    const int l = threadIdx.x & (kWave - 1), w = threadIdx.x / kWave;
    uint32_t id[kRowsWave], rank[kRowsWave];
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const uint32_t i = it * THREADS + threadIdx.x;
        id[it] = i < n ? (uint32_t)a.expert[c0 + i] : 0xffffffffu;
    }
    const uint32_t e = threadIdx.x % kMaxExperts, p = threadIdx.x / kMaxExperts;
    uint32_t before = 0, all = 0;
    if (gridDim.x > kScanned) {
        if (e < a.E && p == 0) before = a.counts[blockIdx.x * a.E + e], all = a.counts[gridDim.x * a.E + e];
    } else if (gridDim.x > 1 && e < a.E) {
#pragma unroll 4
        for (uint32_t b = p; b < gridDim.x; b += kParts) {
            const uint32_t c = a.counts[b * a.E + e];
            before += b < blockIdx.x ? c : 0;
            all += c;
        }
    }
    const int nrows = (int)((n + kWave - 1) / kWave);
    for (int i = threadIdx.x; i < nrows * kMaxExperts / 2; i += THREADS) reinterpret_cast<uint32_t*>(cnt)[i] = 0;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const uint64_t same = same_expert(id[it], a.E, bits);
        rank[it] = (uint32_t)__popcll(same & (((uint64_t)1 << l) - 1));
        if (same && rank[it] == 0) cnt[it * kWaves + w][id[it]] = (uint16_t)__popcll(same);
    }
    __syncthreads();
    uint32_t mine = 0;
    if (e < a.E) {
        const int last = (int)(p + 1) * kPart < nrows ? (int)(p + 1) * kPart : nrows;
#pragma unroll 4
        for (int r = (int)p * kPart; r < last; ++r) {
            const uint32_t c = cnt[r][e];
            cnt[r][e] = (uint16_t)mine;
            mine += c;
        }
    }
    part[p][e] = mine;
    parts_before[p][e] = before;
    parts_all[p][e] = all;
    __syncthreads();
    // thread e < 256: expert e's choices before this workgroup and in all; a scan over the experts
    uint32_t total = 0, v = 0;
    before = 0;
    if (threadIdx.x < kMaxExperts) {
        uint32_t here = 0;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            here += part[i][e];
            before += parts_before[i][e];
            total += parts_all[i][e];
        }
        if (gridDim.x == 1) total = here;
        v = total;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const uint32_t o = (uint32_t)__shfl_up((int)v, d, kWave);
            if (l >= d) v += o;
        }
        if (l == kWave - 1) wave_sums[w] = v;
    }
    __syncthreads();
    if (threadIdx.x < kMaxExperts) {
        for (int i = 0; i < w; ++i) v += wave_sums[i];  // now where expert e's choices end
        uint32_t at = v - total + before;
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            base[i][e] = at;
            at += part[i][e];
        }
        if (e < a.E && blockIdx.x == 0) {
            a.offsets[e + 1] = (int32_t)v;
            if (e == 0) a.offsets[0] = 0;
        }
        if (e == a.E - 1) end_of_all = v;
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kRowsWave; ++it) {
        const uint32_t i = it * THREADS + threadIdx.x;
        if (i >= n) continue;
        int32_t at = -1;
        if (id[it] < a.E) {
            const int r = it * kWaves + w;
            at = (int32_t)(base[r / kPart][id[it]] + cnt[r][id[it]] + rank[it]);
            a.order[at] = (int32_t)(c0 + i);
        }
        a.position[c0 + i] = at;
        if (c0 + i >= end_of_all) a.order[c0 + i] = -1;
    }
}

int64_t route_blocks(int64_t T) { return (T + route::chunk(route::kLarge) - 1) / route::chunk(route::kLarge); }

hipError_t launch_route(const RouteArgs& a, hipStream_t s) {
    using namespace route;
    const unsigned blocks = (unsigned)route_blocks(a.T);
    int bits = 0;
    while ((1u << bits) < a.E) ++bits;
    if (blocks > 1) route_count_kernel<<<blocks, kLarge, 0, s>>>(a, bits);
    if (blocks > kScanned) route_scan_kernel<<<a.E, kScan, 0, s>>>(a, (int)blocks);
    if (a.T <= chunk(kSmall)) route_kernel<kSmall><<<1, kSmall, 0, s>>>(a, bits);
    else route_kernel<kLarge><<<blocks, kLarge, 0, s>>>(a, bits);
    return hipGetLastError();
}

// ---- slots back to tokens ---------------------------------------------------------------------------
// A workgroup: a token and 256 pieces of its row, of four elements (VEC: N % 4 == 0) or one; items beyond the grid in
// turn.
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
                    make_uint2(bf16_word(wt * v.x, wt * v.y), bf16_word(wt * v.z, wt * v.w));
                if (a.dWeights) {
                    const float4 y = *reinterpret_cast<const float4*>(a.slots + o);
                    dot += (v.x * y.x + v.y * y.y) + (v.z * y.z + v.w * y.w);
                }
            } else {
                a.dSlots[o] = (uint16_t)bf16_word(wt * *g, 0.f);
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
    const bool vec = a.N % 4 == 0 && (((uintptr_t)a.slots | (uintptr_t)a.dY) & 15) == 0 &&
                     ((uintptr_t)a.dSlots & 7) == 0;
    if (vec) combine_backward_kernel<true><<<token_grid(a.M), 256, 0, s>>>(a);
    else combine_backward_kernel<false><<<token_grid(a.M), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace bl
