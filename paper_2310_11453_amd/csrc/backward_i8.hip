// Straight-through backward of the 8-bit product (rounding is identity, the scales are constants):
//   dX[M,K] = (dY * scale) W            dW[N,K] = dY^T (q * gamma / 128)
// on the tiles of gemm_i8.hip with bf16 operands.  int8 codes are exact in bf16, and what is rounded is rounded once: of
// a bf16 dY the weights' values code * scale (dX), of an fp32 dY the product dY * scale; for dW dY, with gamma_m / 128
// where gamma is per token (exact for a bf16 dY and one gamma a tensor).  The operands are copied first, in blocks of 32
// reduction indices padded with zeros:
//   wT [Np/32][K/16] tiles of weights transposed (B of dX)      qT [Mp/32][K/16] tiles of codes transposed (B of dW)
//   g  [Np/32][M][32] dY                          (A of dX)      gwT [Mp/32][N][32] dY transposed             (A of dW)
// g is not made where the product can read a bf16 dY as it lies (N a multiple of 32).
#include "common.h"
#include "i8.h"

namespace bl {

static inline int64_t pad32(int64_t v) { return (v + 31) / 32 * 32; }
// (row, r) of a copy with R rows
__device__ inline int64_t copy_offset(int64_t row, int64_t r, int64_t R) { return ((r >> 5) * R + row) * 32 + (r & 31); }
__device__ inline float element(const float* p, int64_t i) { return p[i]; }
__device__ inline float element(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }

struct CopyI8Args {
    const void* dY;
    const int8_t* codes;
    const uint8_t* packed;
    const float* w_scale;    // of the weights' values, or null: the codes
    const float* col_scale;  // of g, or null
    const float* row_gamma;  // of gwT, or null
    uint16_t *wT, *qT, *g, *gwT;  // what is not wanted is null
    int64_t M, N, K, Np, Mp;
    uint32_t w_items, q_items, items, k_x, dy_x;  // items of the weights, of the codes, of all; in a row of them, of dY
};

// Bytes of 32 rows x 256 columns -> tiles of the transposed copy: 16 columns a KiB, eight rows of a column 16 bytes.  A
// wave takes 64 columns and stores a tile at a time, whole lines; four lanes read the same dwords and take a byte each
// (with stores of 16 bytes 64 apart all copies took 161 us instead of 141, 8192 x 16384 x 4096).  LDS rows are 272
// bytes.
typedef uint8_t ByteTile[32][272];
__device__ inline void transpose_bytes(const ByteTile& tile, uint16_t* __restrict__ out, int64_t r0, int64_t k0, int64_t K,
                                       const float (&scale)[8]) {
    const int l = (int)threadIdx.x & 63, rg = l >> 4, c = l & 15, first = (int)threadIdx.x / 64 * 64;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int64_t k = k0 + first + 16 * j;
        if (k >= K) return;  // uniform; K % 32 == 0
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(&tile[8 * rg + 2 * i + e][first + 16 * j + (c & ~3)]);
                v[e] = (float)(int8_t)(w >> (8 * (c & 3))) * scale[2 * i + e];
            }
            o[i] = bf16_pair(v[0], v[1]);
        }
        *reinterpret_cast<uint4*>(out + ((r0 >> 5) * (K >> 4) + (k >> 4)) * 512 + l * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// dY -> g and gwT: 64 x 64, a thread's 4 x 4 elements loaded before the first is used.  VEC: four elements are one load.
typedef uint16_t HalfTile[64][66];
template <typename IN, bool VEC>
__device__ inline void copy_dy(const CopyI8Args& a, int64_t r0, int64_t c0, HalfTile& tile) {
    const IN* const in = static_cast<const IN*>(a.dY);
    const int cl = ((int)threadIdx.x & 15) * 4;
    const int64_t c = c0 + cl, R = a.M, C = a.N;
    float v[4][4], gamma[4];
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int64_t r = r0 + it * 16 + ((int)threadIdx.x >> 4), at = r < R ? r : R - 1;
        if constexpr (VEC) {
            const float4 t = load4(in + at * C, (c < C ? c : C - 4) / 4);
            v[it][0] = t.x, v[it][1] = t.y, v[it][2] = t.z, v[it][3] = t.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[it][e] = element(in, at * C + (c + e < C ? c + e : C - 1));
        }
        gamma[it] = a.row_gamma ? a.row_gamma[at] * (1.0f / 128.0f) : 1.0f;  // uniform
    }
    float sc[4] = {1.0f, 1.0f, 1.0f, 1.0f};
    if (a.col_scale)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[e] = a.col_scale[c + e < C ? c + e : C - 1];
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int rl = it * 16 + ((int)threadIdx.x >> 4);
        const int64_t r = r0 + rl;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[it][e] = r < R && c + e < C ? v[it][e] : 0.f;
        if (a.g && r < R && c < a.Np)
            *reinterpret_cast<uint2*>(a.g + copy_offset(r, c, R)) =
                make_uint2(bf16_pair(v[it][0] * sc[0], v[it][1] * sc[1]), bf16_pair(v[it][2] * sc[2], v[it][3] * sc[3]));
        uint32_t* t32 = reinterpret_cast<uint32_t*>(&tile[rl][cl]);
        t32[0] = bf16_pair(v[it][0] * gamma[it], v[it][1] * gamma[it]);
        t32[1] = bf16_pair(v[it][2] * gamma[it], v[it][3] * gamma[it]);
    }
    if (!a.gwT) return;
    __syncthreads();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const int idx = it * 256 + (int)threadIdx.x, col = idx >> 4, rl = (idx & 15) * 4;
        if (c0 + col < C && r0 + rl < a.Mp)
            *reinterpret_cast<uint2*>(a.gwT + copy_offset(c0 + col, r0 + rl, C)) =
                make_uint2((uint32_t)tile[rl][col] | ((uint32_t)tile[rl + 1][col] << 16),
                           (uint32_t)tile[rl + 2][col] | ((uint32_t)tile[rl + 3][col] << 16));
    }
}

// All of it in one launch, the small parts first (behind dY they would be the tail).  Bound by HBM: 8192 x 16384 x 4096,
// bf16 dY, 840 MB in 141 us; 333 x 2048 x 2048 in 8.8 us, a chain of two trips to memory.
template <typename IN, bool VEC>
__global__ __launch_bounds__(256) void copy_i8_operands(CopyI8Args a) {
    __shared__ __attribute__((aligned(16))) union {
        ByteTile bytes;
        HalfTile halves;
    } sm;
    const int tid = (int)threadIdx.x;
    for (uint32_t it = blockIdx.x; it < a.items; it += gridDim.x) {
        if (it != blockIdx.x) __syncthreads();  // the item before has been read
        uint32_t i = it;
        if (i < a.w_items) {  // 32 channels x 256 k: tiles of 16 x 64
            const int64_t nb = i / a.k_x, k0 = (int64_t)(i % a.k_x) * 256, TK = i8_tiles_k(a.K), TN = tiles_n(a.N);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t tn = 2 * nb + h, tk = k0 / 64 + tid / 64;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (tn < TN && tk < TK) v = *reinterpret_cast<const uint4*>(a.packed + (tn * TK + tk) * 1024 + (tid & 63) * 16);
                *reinterpret_cast<uint4*>(&sm.bytes[16 * h + (tid & 15)][tid / 64 * 64 + (tid >> 4 & 3) * 16]) = v;
            }
            float sc[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int64_t n = nb * 32 + 8 * (tid >> 4 & 3) + e;
                sc[e] = a.w_scale ? a.w_scale[n < a.N ? n : a.N - 1] : 1.0f;  // (zeros past N)
            }
            __syncthreads();
            transpose_bytes(sm.bytes, a.wT, nb * 32, k0, a.K, sc);
            continue;
        }
        i -= a.w_items;
        if (i < a.q_items) {  // 32 tokens x 256 k
            const int64_t mb = i / a.k_x, k0 = (int64_t)(i % a.k_x) * 256;
            const int64_t m = mb * 32 + tid / 8;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kl = (tid & 7) * 16 + h * 128;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (m < a.M && k0 + kl < a.K) v = *reinterpret_cast<const uint4*>(a.codes + m * a.K + k0 + kl);
                *reinterpret_cast<uint4*>(&sm.bytes[tid / 8][kl]) = v;
            }
            __syncthreads();
            const float one[8] = {1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f, 1.0f};
            transpose_bytes(sm.bytes, a.qT, mb * 32, k0, a.K, one);
            continue;
        }
        i -= a.q_items;
        copy_dy<IN, VEC>(a, (int64_t)(i / a.dy_x) * 64, (int64_t)(i % a.dy_x) * 64, sm.halves);
    }
}

// Whether the product reads dY where it lies: whole stages, and offsets of a tile's rows in 32 bits.
static bool dy_direct(bool bf16, int64_t N) { return bf16 && N % 32 == 0 && N < (1 << 22); }

// The copies, each 256-byte aligned, then (optional) room for the products' slices.  What is asked for does not go by
// the types.
struct BackwardI8Ws {
    size_t wT, gwT, qT, total;
};
static BackwardI8Ws backward_i8_ws(int64_t M, int64_t N, int64_t K) {
    const int64_t Np = pad32(N), Mp = pad32(M);
    auto al = [](size_t v) { return (v + 255) & ~(size_t)255; };
    BackwardI8Ws w{};
    w.wT = al((size_t)M * Np * 2);
    w.gwT = w.wT + al((size_t)K * Np * 2);
    w.qT = w.gwT + al((size_t)N * Mp * 2);
    w.total = w.qT + al((size_t)K * Mp * 2);
    return w;
}
size_t backward_i8_min_bytes(int64_t M, int64_t N, int64_t K) { return backward_i8_ws(M, N, K).total; }
size_t backward_i8_bytes(int64_t M, int64_t N, int64_t K) {
    const size_t dx = gemm_bf16_part_bytes(M, K, pad32(N) / 32), dw = gemm_bf16_part_bytes(N, K, pad32(M) / 32);
    return backward_i8_ws(M, N, K).total + (dx > dw ? dx : dw);
}

hipError_t launch_backward_i8(const BackwardI8Args& a, hipStream_t s) {
    const int64_t M = a.M, N = a.N, K = a.K, Np = pad32(N), Mp = pad32(M);
    const BackwardI8Ws ws = backward_i8_ws(M, N, K);
    char* base = (char*)a.workspace;
    uint16_t *g = (uint16_t*)base, *wT = (uint16_t*)(base + ws.wT), *gwT = (uint16_t*)(base + ws.gwT),
             *qT = (uint16_t*)(base + ws.qT);
    const bool direct = dy_direct(a.dy_bf16, N);
    CopyI8Args c{};
    c.dY = a.dY; c.codes = a.codes; c.packed = a.packed; c.M = M; c.N = N; c.K = K; c.Np = Np; c.Mp = Mp;
    c.w_scale = a.dy_bf16 ? a.scale : nullptr;
    c.col_scale = a.dy_bf16 ? nullptr : a.scale;
    c.row_gamma = a.per_tensor ? nullptr : a.gamma;
    c.wT = a.dX ? wT : nullptr;
    c.g = a.dX && !direct ? g : nullptr;
    c.qT = a.dW ? qT : nullptr;
    c.gwT = a.dW ? gwT : nullptr;
    auto tiles = [](int64_t v, int64_t t) { return (v + t - 1) / t; };
    c.k_x = (uint32_t)tiles(K, 256);
    c.dy_x = (uint32_t)tiles(c.g ? Np : N, 64);
    const int64_t w_items = c.wT ? Np / 32 * c.k_x : 0, q_items = c.qT ? Mp / 32 * c.k_x : 0;
    const int64_t items = w_items + q_items + (c.g || c.gwT ? tiles(c.gwT ? Mp : M, 64) * c.dy_x : 0);
    if (items >= (int64_t)1 << 32) return hipErrorInvalidValue;
    c.w_items = (uint32_t)w_items; c.q_items = (uint32_t)q_items; c.items = (uint32_t)items;
    const unsigned grid = (unsigned)(items < (1 << 22) ? items : (1 << 22));
    const bool vec = N % 4 == 0;
    if (a.dy_bf16) {
        if (vec) copy_i8_operands<uint16_t, true><<<grid, 256, 0, s>>>(c);
        else copy_i8_operands<uint16_t, false><<<grid, 256, 0, s>>>(c);
    } else {
        if (vec) copy_i8_operands<float, true><<<grid, 256, 0, s>>>(c);
        else copy_i8_operands<float, false><<<grid, 256, 0, s>>>(c);
    }
    GemmBF16Args x{};
    x.part = base + ws.total;
    x.part_bytes = a.workspace_bytes > ws.total ? a.workspace_bytes - ws.total : 0;
    GemmBF16Args w = x;
    x.A = direct ? a.dY : g; x.B = wT;
    x.a_pitch = direct ? N * 2 : 64; x.a_step = direct ? 64 : M * 64;
    x.M = M; x.N = K; x.stages = (int)(Np / 32); x.times = 1.0f; x.y_bf16 = a.dx_bf16; x.Y = a.dX;
    w.A = gwT; w.B = qT; w.a_pitch = 64; w.a_step = N * 64;
    w.M = N; w.N = K; w.stages = (int)(Mp / 32);
    w.factor = a.per_tensor ? a.gamma : nullptr; w.times = a.per_tensor ? 1.0f / 128.0f : 1.0f;
    w.y_bf16 = false; w.Y = a.dW;
    if (a.dX && a.dW) return launch_gemm_bf16_two(x, w, s);
    return launch_gemm_bf16(a.dX ? x : w, s);
}

}  // namespace bl
