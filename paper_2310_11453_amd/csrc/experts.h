// Host-side launchers of the operators of a mixture of BitLinear layers; called from api_experts.hip only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace bl {

constexpr int kMaxExperts = 256;
constexpr int64_t kMaxRouteSlots = (int64_t)1 << 24;

// route.hip
struct RouteArgs {
    const int32_t* expert;  // [T]
    uint32_t T, E;
    int32_t *order, *position, *offsets;
    uint32_t* counts;  // [route_blocks][E] and behind them [E], several blocks only
};
int64_t route_blocks(int64_t T);
hipError_t launch_route(const RouteArgs& a, hipStream_t s);

struct CombineArgs {
    const float* slots;  // [T][N]; backward: may be null (no dweights)
    const int32_t* position;
    const float* weights;  // [M][top_k] or null: ones
    int64_t M, N, T;
    int top_k;
    const float* dY;   // backward
    float* Y;          // forward: [M][N]
    uint16_t* dSlots;  // backward: bf16 [T][N]
    float* dWeights;   // backward: [M][top_k] or null
};
hipError_t launch_combine(const CombineArgs& a, hipStream_t s);
hipError_t launch_combine_backward(const CombineArgs& a, hipStream_t s);

// nonlinear.hip
constexpr int64_t kMaxNonlinearK = 32768;
constexpr int kCheckBlock = 128;  // elements of a row that share a scale of the checkpoint
struct NonlinearArgs {
    const float* U;
    int64_t M, K;
    float eps;
    double inv_k;         // 1 / K (set by the launcher)
    const int32_t* rows;  // device: rows that exist, or null: all M
    int8_t* codes;
    float* gamma;
    int32_t* rowsum;     // or null
    int8_t* check;       // or null: no checkpoint
    float* check_scale;  // [M][ceil(K / 128)]
    bool per_tensor;
    double* rowstats;     // per tensor: [M][2]
    uint32_t* gmax_bits;  // per tensor: [1]
    const float* dXhat;   // backward
    void* dU;             // backward: fp32 or bf16
    bool bf16;
};
hipError_t launch_quant_nonlinear(const NonlinearArgs& a, int fn, hipStream_t s);
hipError_t launch_nonlinear_backward(const NonlinearArgs& a, int fn, hipStream_t s);

// experts.hip, experts_backward.hip
// Slot s of expert e, offsets[e] <= s < offsets[e + 1], is row order[s] / top_k of the codes (order null: row s).
struct ExpertsArgs {
    const int8_t* codes;
    const float* gamma;
    const int32_t* rowsum;
    int64_t rows;  // of the codes
    int64_t T, K, N;
    const int32_t* order;
    int top_k;
    const int32_t* offsets;  // [E + 1]
    int E;
    const uint32_t* packed;  // E blobs
    const float* beta;       // [E]
    bool per_tensor, out_acc;
    float* Y;
    const uint16_t* dY;  // backward: bf16 [T][N]
    float *dX, *dW;
    void* workspace;
    size_t workspace_bytes;
};
hipError_t launch_matmul_experts(const ExpertsArgs& a, hipStream_t s);

// backward.hip: the two products of the backward from the copies that experts_backward.hip makes of their operands.
// Reduction indices in blocks of 32 as there (block_offset): g [T rows][Np] (direct: dY itself, by rows), Sw
// [E][Np / 32][K]; gwT [N rows] and qT [K rows] over the slots of expert after expert, each expert's filled up with
// zeros to whole blocks and to `least` of them.
struct ExpertsOperands {
    const uint16_t *g, *gwT, *qT;
    const uint32_t* Sw;
    const uint16_t* dY;
    bool direct, direct_dw;  // dX, dW read dY itself
    const int32_t* offsets;
    int E, least;
    int64_t T, N, K;
    const float *beta, *gamma;  // gamma: of the tensor, or null
    float *dX, *dW, *part;      // part: sums of slices of the reductions
};
struct ExpertsBackwardPlan {
    int dx_slices, dw_tile, dw_splits;  // dx_slices: at most, of a tile in dX's last round
};
size_t experts_dx_part_bytes(int64_t T, int64_t K, int E, const ExpertsBackwardPlan& p);
ExpertsBackwardPlan experts_backward_plan(int64_t T, int64_t N, int64_t K, int E);
void launch_experts_dx(const ExpertsOperands& a, const ExpertsBackwardPlan& p, hipStream_t s);
void launch_experts_dw(const ExpertsOperands& a, const ExpertsBackwardPlan& p, hipStream_t s);
// dX, and dW with one gamma a tensor, read dY where it lies; else copies in whole stages of 32 are made.
inline bool experts_dy_direct(int64_t N) { return N % 32 == 0 && N < (1 << 23); }
size_t experts_backward_bytes(int64_t T, int64_t N, int64_t K, int E, bool per_tensor);
hipError_t launch_experts_backward(const ExpertsArgs& a, hipStream_t s);

#ifdef __HIPCC__
__device__ inline uint32_t bf16_word(float lo, float hi) {  // to nearest, ties to even
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    const v2bf v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
// Segments come from memory: what is read of them is held to 0 .. T, so that no value of theirs leads out of a tensor.
__device__ inline int slot_bound(const int32_t* offsets, int e, int T) {
    const int v = offsets[e];
    return v < 0 ? 0 : v < T ? v : T;
}
__device__ inline uint32_t row_of(uint32_t r, uint32_t rows) { return r < rows ? r : rows - 1; }
// the row of the codes that slot s reads
__device__ inline uint32_t code_row(const int32_t* order, uint32_t top_k, uint32_t rows, uint32_t s) {
    return row_of(order ? (uint32_t)order[s] / top_k : s, rows);
}

// Rows of tiles of BM slots: expert e has those from first[e] on, its slots are from[e] .. to[e] - 1.
struct ExpertTiles {
    int first[kMaxExperts + 1], from[kMaxExperts], to[kMaxExperts];
};
// What offsets as bitlinear_route leaves them come to at most, of E experts with `least` rows of tiles or more each.
__host__ __device__ inline int64_t most_tiles(int64_t T, int64_t E, int BM, int least) {
    return T / BM + (least ? E * least : T < E ? T : E);
}
// v of this lane and of those below it, all lanes active
__device__ inline int wave_sums(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // within rows of 16 lanes: from 1,
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);  // 2,
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);  // 4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);  // and 8 lanes below;
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, true);  // the last lane of rows 0 and 2 to rows 1 and 3;
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, true);  // lane 31 to rows 2 and 3
    return v;
}
// Counts them (no expert has fewer than `least`), all threads of a workgroup of 256 or more; their number, which no
// value of `offsets` takes past most_tiles.  Every workgroup of a product does this before its first load.
__device__ inline int expert_tiles(const int32_t* offsets, int E, int T, int BM, ExpertTiles& sm, int least = 0) {
    const int e = (int)threadIdx.x, most = (int)most_tiles(T, E, BM, least);
    const bool mine = e < kMaxExperts && (e & -kWave) < E;  // whole waves
    if (mine) {
        const int from = e < E ? slot_bound(offsets, e, T) : 0, to = e < E ? slot_bound(offsets, e + 1, T) : 0;
        int v = to > from ? (to - from + BM - 1) / BM : 0;
        if (v < least && e < E) v = least;
        sm.from[e] = from;
        sm.to[e] = to > from ? to : from;
        v = wave_sums(v);
        sm.first[e + 1] = E > kWave ? v : v < most ? v : most;
    }
    if (e == 0) sm.first[0] = 0;
    __syncthreads();
    if (E > kWave) {
        int v = 0;
        if (mine) {
            v = sm.first[e + 1];
            for (int i = kWave; i <= e; i += kWave) v += sm.first[i];
        }
        __syncthreads();
        if (mine) sm.first[e + 1] = v < most ? v : most;
        __syncthreads();
    }
    return sm.first[E];
}
// The expert of a row of tiles, and where that row's slots begin and the expert's end.
__device__ inline int expert_of_tile(const ExpertTiles& sm, int E, int tile, int BM, int& from, int& to) {
    int lo = 0, hi = E - 1;  // the last expert whose first row of tiles is not behind `tile`
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (sm.first[mid] <= tile) lo = mid;
        else hi = mid - 1;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    from = __builtin_amdgcn_readfirstlane(sm.from[lo] + (tile - sm.first[lo]) * BM);
    to = __builtin_amdgcn_readfirstlane(sm.to[lo]);
    return lo;
}
#endif

}  // namespace bl
