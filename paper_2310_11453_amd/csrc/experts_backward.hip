// Straight-through backward of the products of a mixture of BitLinear layers (arXiv 2310.11453, Section 2.2):
//   dXs[s,k]  = beta_e sum_n dY[s,n] S_e[n,k]             for the slots s of expert e
//   dW_e[n,k] = sum_{s of e} dY[s,n] q[r,k] gamma_r/128    r the row that s reads; zeros where e has no slots
// dY is bf16, +-1 and the codes are exact in bf16.  As in the plain layer (backward.hip, whose kernels take the
// products), every operand is first written once in the layout they read:
//   g    [T][Np]       rows of dY                                 (A operand of dX, reduction over N; not where N is a
//                      multiple of 32: the product reads dY itself, at the same speed; 8192 slots 2048 -> 8192
//                      680 us with the copy, 662 without)
//   Sw   [E][Np/32][K] the signs of 32 weight rows of a column    (B operand of dX)
//   gwT  [N][slots]    dY transposed, with a gamma per token scaled and rounded again   (A operand of dW; not with a gamma
//                      per tensor and N a multiple of 32: the product reads dY itself, transposed out of LDS; both
//                      products of those 8192 slots 618 us with the copy, 562 without)
//   qT   [K][slots]    codes transposed, gathered through the order                     (B operand of dW)
// The slots of the last two are those of expert after expert, each expert's filled up with zeros to whole blocks of 32:
// a stage of the products is such a block and belongs to one expert.
#include "common.h"
#include "experts.h"
#include "kernels.h"

namespace bl {

namespace exb {
// An item of the copies: 64 slots x 128 columns, transposed through LDS (the pitch is odd in dwords, so that the rows
// that a lane's eight reads of a column come from are on different banks).
constexpr int kRows = 64, kCols = 128;
typedef uint16_t CastTile[kRows][kCols + 2];

struct Args {
    const uint16_t* dY;
    const int8_t* codes;
    const uint32_t* packed;
    const float* row_gamma;  // null: per tensor
    const int32_t *offsets, *order;
    uint32_t top_k, rows;
    int E, T, least;
    uint16_t *g, *gwT, *qT;  // what is not wanted is null
    uint32_t* Sw;
    int64_t N, K, Np, blob;
    uint32_t bits_items, code_items, items;    // items: of all three parts
    uint32_t bits_x, bits_y, code_x, dy_x;     // items in a row of each part; pairs of rows of sign words of an expert
};
}  // namespace exb

// (block_offset of backward.hip)
__device__ inline int64_t copy_offset(int64_t row, int64_t r, int64_t R) {
    return ((r >> 5) * R + row) * 32 + (r & 31);
}

// dY (bf16) -> g and gwT, or codes -> qT.  VEC: a thread's eight elements are one load.  Everything that an item reads
// is requested before the first of it is used.
template <bool CODES, bool VEC>
__device__ inline void copy_tile(const exb::Args& a, const ExpertTiles& count, int blocks, int r0, int64_t c0,
                                 exb::CastTile& tile) {
    using namespace exb;
    const int64_t C = CODES ? a.K : a.N;
    const int cl = ((int)threadIdx.x & 15) * 8, rt = (int)threadIdx.x >> 4;
    const int64_t c = c0 + cl;
    // of rows rt + 16 it; -1: filled up.  Rows 0 .. 31 of the item are a block, of one expert, 32 .. 63 another
    int slot[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int from = 0, to = 0;
        if ((r0 >> 5) + h < blocks) expert_of_tile(count, a.E, (r0 >> 5) + h, 32, from, to);
#pragma unroll
        for (int i = 0; i < 2; ++i) slot[2 * h + i] = from + rt + 16 * i < to ? from + rt + 16 * i : -1;
    }
    uint32_t v[4][4] = {};  // eight bf16 a row
    float gamma[4];
    uint32_t row[4];
#pragma unroll
    for (int it = 0; it < 4; ++it)
        if (slot[it] >= 0 && (CODES || a.row_gamma)) row[it] = code_row(a.order, a.top_k, a.rows, (uint32_t)slot[it]);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        if (slot[it] < 0 || c >= C) continue;
        if constexpr (CODES) {  // K % 32 == 0
            const int8_t* const src = a.codes + (int64_t)row[it] * C + c;
            const uint2 t = *reinterpret_cast<const uint2*>(src);
            v[it][0] = t.x, v[it][1] = t.y;
        } else {
            const uint16_t* const src = a.dY + (int64_t)slot[it] * C + c;
            if constexpr (VEC) {
                const uint4 t = *reinterpret_cast<const uint4*>(src);
                v[it][0] = t.x, v[it][1] = t.y, v[it][2] = t.z, v[it][3] = t.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[it][e] = (c + 2 * e < C ? src[2 * e] : 0) |
                               (c + 2 * e + 1 < C ? (uint32_t)src[2 * e + 1] << 16 : 0);
            }
            if (a.row_gamma) gamma[it] = a.row_gamma[row[it]];
        }
    }
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int rl = rt + 16 * it;
        if constexpr (CODES) {
            const uint32_t lo = v[it][0], hi = v[it][1];
            auto pair = [](uint32_t w, int sh) {
                return bf16_word((float)(int8_t)(w >> sh), (float)(int8_t)(w >> (sh + 8)));
            };
            v[it][0] = pair(lo, 0), v[it][1] = pair(lo, 16), v[it][2] = pair(hi, 0), v[it][3] = pair(hi, 16);
        } else {
            if (a.g && slot[it] >= 0 && c < a.Np)
                *reinterpret_cast<uint4*>(a.g + copy_offset(slot[it], c, a.T)) =
                    make_uint4(v[it][0], v[it][1], v[it][2], v[it][3]);
            if (a.row_gamma && slot[it] >= 0 && c < C) {
                const float sc = gamma[it] / 128.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[it][e] = bf16_word(__uint_as_float(v[it][e] << 16) * sc,
                                         __uint_as_float(v[it][e] & 0xffff0000u) * sc);
            }
        }
        uint32_t* const t32 = reinterpret_cast<uint32_t*>(&tile[rl][cl]);
#pragma unroll
        for (int e = 0; e < 4; ++e) t32[e] = v[it][e];
    }
    uint16_t* const tr = CODES ? a.qT : a.gwT;
    if (!tr) return;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int idx = it * 256 + (int)threadIdx.x;
        const int cc = idx >> 3, rl = (idx & 7) * 8;
        const int64_t col = c0 + cc;
        if (col >= C || r0 + rl >= blocks * 32) continue;
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = (uint32_t)tile[rl + 2 * e][cc] | (uint32_t)tile[rl + 2 * e + 1][cc] << 16;
        *reinterpret_cast<uint4*>(tr + copy_offset(col, r0 + rl, C)) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// 32 x 32 bits, row l of them in lane l (of each half of a wave), transposed: five exchanges with the lane whose number
// differs in one bit.  What a rotation by s bits brings around lands where the lane keeps its own.
struct BitTranspose {
    uint32_t keep[5], turn[5];
    __device__ inline explicit BitTranspose(int l) {
        constexpr uint32_t kLow[5] = {0x55555555u, 0x33333333u, 0x0f0f0f0fu, 0x00ff00ffu, 0x0000ffffu};
#pragma unroll
        for (int b = 0; b < 5; ++b) {
            const bool high = (l >> b) & 1;
            keep[b] = high ? ~kLow[b] : kLow[b];
            turn[b] = high ? 1u << b : 32u - (1u << b);  // to the right
        }
    }
    template <int B>
    __device__ inline uint32_t step(uint32_t x) const {
        const uint32_t t = (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, (1 << B) << 10 | 0x1f);  // of lane l ^ 2^B
        return (x & keep[B]) | (__builtin_amdgcn_alignbit(t, t, turn[B]) & ~keep[B]);
    }
    __device__ inline uint32_t operator()(uint32_t x) const {
        return step<0>(step<1>(step<2>(step<3>(step<4>(x)))));
    }
};

// signs of two times 32 weight rows x 512 columns of an expert (the bit layout of a word: bits_transpose_tile of
// backward.hip).  A dword of a packed tile is a row's bits of 32 columns, and lane l takes the row that is bit l of a
// word: a wave transposes four times 2 x 32 rows x 32 columns.  (A column's 32 bits picked one by one: the backward of 128
// slots of 8 experts 2048 -> 8192 156 us, 146 so; of 8192 slots 552 and 543.)
__device__ inline void words_tile(const exb::Args& a, int e, int64_t pair, int64_t tk, uint32_t (&sm)[2][8 * 68]) {
    const int64_t TN = tiles_n(a.N), TK = tiles_k(a.K), words = a.Np / 32;
    const int w = (int)threadIdx.x / kWave, l = (int)threadIdx.x & (kWave - 1), b = l & 31;
    const int half = w >> 1, g = 2 * (w & 1) + (l >> 5);
    const int row = ((b >> 4) & 1) | (b & 3) << 1 | ((b >> 2) & 1) << 3 | ((b >> 3) & 1) << 4;
    const int64_t tn = 2 * (2 * pair + half) + (row >> 4);
    uint32_t q[4] = {0, 0, 0, 0};
    if (tn < TN) {
        const uint4 v = *reinterpret_cast<const uint4*>(a.packed + e * a.blob + tile_dword_offset(tn, tk, TK) +
                                                        (g * 16 + (row & 15)) * 4);
        q[0] = v.x, q[1] = v.y, q[2] = v.z, q[3] = v.w;
    }
    const BitTranspose transpose(b);
#pragma unroll
    for (int d = 0; d < 4; ++d)  // bit 8 j + i of a dword: column 64 i + 16 g + 4 d + j
        sm[half][(b & 7) * 68 + 16 * g + 4 * d + (b >> 3)] = ~transpose(q[d]);
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int kl = (it & 1) * 256 + (int)threadIdx.x;
        const int64_t sw = 2 * pair + (it >> 1), k = tk * kChunkK + kl;
        if (sw < words && k < a.K) a.Sw[(e * words + sw) * a.K + k] = sm[it >> 1][(kl >> 6) * 68 + (kl & 63)];
    }
}

template <bool VEC>
__global__ __launch_bounds__(256) void prepare_expert_operands(exb::Args a) {
    __shared__ ExpertTiles count;
    __shared__ __attribute__((aligned(16))) union {
        exb::CastTile tile;
        uint32_t words[2][8 * 68];
    } sm;
    const int blocks = expert_tiles(a.offsets, a.E, a.T, 32, count, a.least);
    for (uint32_t it = blockIdx.x; it < a.items; it += gridDim.x) {
        if (it != blockIdx.x) __syncthreads();  // the item before has been read
        uint32_t i = it;
        if (i < a.bits_items) {
            const uint32_t y = i / a.bits_x, e = y / a.bits_y;  // 512 columns fastest
            if (count.from[e] < count.to[e])  // else nobody reads them
                words_tile(a, (int)e, y % a.bits_y, i % a.bits_x, sm.words);
            continue;
        }
        i -= a.bits_items;
        const bool codes = i < a.code_items;
        if (!codes) i -= a.code_items;
        const uint32_t x = codes ? a.code_x : a.dy_x;
        const int r0 = (int)(i / x) * exb::kRows;
        if (r0 >= blocks * 32) continue;  // uniform: the grid is a bound
        if (codes) copy_tile<true, true>(a, count, blocks, r0, (int64_t)(i % x) * exb::kCols, sm.tile);
        else copy_tile<false, VEC>(a, count, blocks, r0, (int64_t)(i % x) * exb::kCols, sm.tile);
    }
}

namespace {
int64_t pad32(int64_t v) { return (v + 31) / 32 * 32; }
struct ExpertsWs {
    size_t words, gwT, qT, part, total;
};
ExpertsWs experts_ws(int64_t T, int64_t N, int64_t K, int E, bool per_tensor, const ExpertsBackwardPlan& p) {
    auto al = [](size_t v) { return (v + 255) & ~(size_t)255; };
    const int64_t Np = pad32(N), slots = most_tiles(T, E, 32, p.dw_splits) * 32;
    ExpertsWs w{};
    w.words = experts_dy_direct(N) ? 0 : al((size_t)T * Np * 2);
    w.gwT = w.words + al((size_t)E * (Np / 32) * K * 4);
    w.qT = w.gwT + (experts_dy_direct(N) && per_tensor ? 0 : al((size_t)N * slots * 2));
    w.part = w.qT + al((size_t)K * slots * 2);
    // one product after the other
    const size_t dx = experts_dx_part_bytes(T, K, E, p);
    const size_t dw = p.dw_splits > 1 ? (size_t)p.dw_splits * E * N * K * 4 : 0;
    w.total = w.part + (dx > dw ? dx : dw);
    return w;
}
}  // namespace

size_t experts_backward_bytes(int64_t T, int64_t N, int64_t K, int E, bool per_tensor) {
    return experts_ws(T, N, K, E, per_tensor, experts_backward_plan(T, N, K, E)).total;
}

hipError_t launch_experts_backward(const ExpertsArgs& a, hipStream_t s) {
    const ExpertsBackwardPlan p = experts_backward_plan(a.T, a.N, a.K, a.E);
    const ExpertsWs ws = experts_ws(a.T, a.N, a.K, a.E, a.per_tensor, p);
    char* const base = (char*)a.workspace;
    exb::Args b{};
    b.dY = a.dY; b.codes = a.codes; b.packed = a.packed;
    b.row_gamma = a.per_tensor ? nullptr : a.gamma;
    b.offsets = a.offsets; b.order = a.order; b.top_k = (uint32_t)a.top_k; b.rows = (uint32_t)a.rows;
    b.E = a.E; b.T = (int)a.T; b.least = p.dw_splits;
    const bool direct = experts_dy_direct(a.N), direct_dw = direct && a.per_tensor;
    if (a.dX) {
        b.g = direct ? nullptr : (uint16_t*)base;
        b.Sw = (uint32_t*)(base + ws.words);
    }
    if (a.dW) {
        b.gwT = direct_dw ? nullptr : (uint16_t*)(base + ws.gwT);
        b.qT = (uint16_t*)(base + ws.qT);
    }
    b.N = a.N; b.K = a.K; b.Np = pad32(a.N);
    b.blob = tiles_n(a.N) * tiles_k(a.K) * 256;
    auto tiles = [](int64_t v) { return (v + exb::kCols - 1) / exb::kCols; };
    const int64_t rows = (most_tiles(a.T, a.E, 32, b.least) + 1) / 2;
    b.bits_x = (uint32_t)tiles_k(a.K);
    b.bits_y = (uint32_t)((b.Np / 32 + 1) / 2);
    b.code_x = (uint32_t)tiles(a.K);
    b.dy_x = (uint32_t)tiles(b.g ? b.Np : b.N);
    const int64_t bits = a.dX ? (int64_t)a.E * b.bits_y * b.bits_x : 0, codes = a.dW ? rows * b.code_x : 0;
    const int64_t items = bits + codes + (b.g || b.gwT ? rows * b.dy_x : 0);
    if (items >= (int64_t)1 << 32) return hipErrorInvalidValue;
    b.bits_items = (uint32_t)bits;
    b.code_items = (uint32_t)codes;
    b.items = (uint32_t)items;
    const unsigned grid = (unsigned)(items < (1 << 23) ? items : (1 << 23));
    if (a.N % 8 == 0 && ((uintptr_t)a.dY & 15) == 0) prepare_expert_operands<true><<<grid, 256, 0, s>>>(b);
    else prepare_expert_operands<false><<<grid, 256, 0, s>>>(b);

    const ExpertsOperands o{direct ? a.dY : b.g, b.gwT, b.qT, b.Sw, a.dY, direct, direct_dw, a.offsets, a.E, b.least, a.T,
                            a.N, a.K, a.beta, a.per_tensor ? a.gamma : nullptr, a.dX, a.dW, (float*)(base + ws.part)};
    if (a.dX) launch_experts_dx(o, p, s);
    if (a.dW) launch_experts_dw(o, p, s);
    return hipGetLastError();
}

}  // namespace bl
