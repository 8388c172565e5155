// Host-side launchers of the operators around an 8-bit linear layer, and the layout of its weights; called from
// api_i8.hip only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace bl {

// ---------------------------------------------------------------------------
// Packed 8-bit weights.  The [N,K] codes are cut into tiles of 16 rows x 64 columns, padded with zeros: 1 KiB, which a
// wave reads with one fully coalesced 16-byte-per-lane load and then holds as the operand of an i8 MFMA:
//   lane = g*16 + c,  byte b   <->   n = 16*tile_n + c,  k = 64*tile_k + 16*g + b
// Tiles are ordered [tile_n][tile_k], so a row of tiles is one stream.
// ---------------------------------------------------------------------------
constexpr int kI8TileK = 64;
__host__ __device__ inline int64_t i8_tiles_k(int64_t K) { return (K + kI8TileK - 1) / kI8TileK; }
inline size_t i8_blob_bytes(int64_t N, int64_t K) { return (size_t)(tiles_n(N) * i8_tiles_k(K)) * 1024; }

enum ElementType { kF32 = 0, kBF16 = 1, kI8 = 2 };  // as bl_type

// pack_i8.hip
struct PackI8Args {
    const void* W;  // [N][K] of `type`
    int type;
    int64_t N, K;
    uint8_t* packed;
    float* scale;  // [N]; kI8: not touched
};
hipError_t launch_pack_i8(const PackI8Args& a, hipStream_t s);
struct UnpackI8Args {
    const uint8_t* packed;
    const float* scale;  // kI8: not read
    int64_t N, K;
    int type;
    void* out;  // [N][K]
};
hipError_t launch_unpack_i8(const UnpackI8Args& a, hipStream_t s);

// rmsnorm.hip
struct QuantRmsArgs {
    const void* X;  // [M][K] fp32 or bf16
    const void* R;  // residual or null, of the type of H
    void* H;        // X + R, or null; may be X or R
    bool x_bf16, h_bf16;
    int64_t M, K;
    const float* gain;  // [K] or null
    double eps, inv_k;  // inv_k = 1 / K (set by the launcher)
    bool per_tensor;
    int8_t* codes;
    float* gamma;
    int32_t* rowsum;  // or null
    float* xhat;      // or null
    double* rstd;     // per tensor: [M]
    int* most;        // per tensor: the largest magnitude of each workgroup's rows (most_bits), kRmsMostBytes
    int groups;       // how many of those (set by the launcher)
};
constexpr size_t kRmsMostBytes = 2048 * 4;
hipError_t launch_quant_rmsnorm(const QuantRmsArgs& a, hipStream_t s);

struct RmsBackwardArgs {
    const void *G, *H;  // gradient of x^ and the normalised tensor, [M][K]
    const void* dR;     // gradient that H receives besides, or null
    void* dH;           // may be G or dR where the type is the same
    bool g_bf16, h_bf16, d_bf16;
    int64_t M, K;
    const float* gain;  // or null
    double eps, inv_k;
    float* dgain;      // [K] or null
    void* partials;    // with dgain: rms_backward_part_bytes
};
size_t rms_backward_part_bytes(int64_t M, int64_t K);
hipError_t launch_rmsnorm_backward(const RmsBackwardArgs& a, hipStream_t s);

// gemm_i8.hip
struct GemmI8Args {
    const int8_t* codes;
    const float* gamma;
    int64_t M, K, N;
    const uint8_t* packed;
    const float* scale;
    bool per_tensor, out_acc, y_bf16;
    void* Y;
    int32_t* part;  // slices of K (optional)
    size_t part_bytes;
};
size_t gemm_i8_part_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_gemm_i8(const GemmI8Args& a, hipStream_t s);

// The same tiles for the bf16 products of the backward, Y[m][n] = factor * sum_r A[m][r] B[n][r]: stages of 32 r.  A: 64
// bytes of a row are a stage, a_pitch bytes from row to row (256 of them below 2^32), a_step from a stage to the next,
// all 16-byte aligned; B: 16 rows of a stage are a tile of 1 KiB, lane g*16 + c of it the elements 8 g .. 8 g + 7 of row
// c; tiles one after another [stage][N / 16], N a multiple of 16.
struct GemmBF16Args {
    const void *A, *B;
    int64_t a_pitch, a_step, M, N;
    int stages;
    const float* factor;  // device, or null: 1
    float times;          // of the factor
    bool y_bf16;
    void* Y;
    void* part;
    size_t part_bytes;
};
size_t gemm_bf16_part_bytes(int64_t M, int64_t N, int64_t stages);
hipError_t launch_gemm_bf16(const GemmBF16Args& a, hipStream_t s);
// two products that do not need each other; the second is not cut into slices where they share a launch
hipError_t launch_gemm_bf16_two(const GemmBF16Args& a, const GemmBF16Args& a2, hipStream_t s);

// backward_i8.hip
struct BackwardI8Args {
    const void* dY;
    bool dy_bf16, dx_bf16;
    int64_t M, N, K;
    const int8_t* codes;
    const float* gamma;
    bool per_tensor;
    const uint8_t* packed;
    const float* scale;
    void* dX;
    float* dW;
    void* workspace;
    size_t workspace_bytes;  // at least backward_i8_min_bytes
};
size_t backward_i8_min_bytes(int64_t M, int64_t N, int64_t K);
size_t backward_i8_bytes(int64_t M, int64_t N, int64_t K);
hipError_t launch_backward_i8(const BackwardI8Args& a, hipStream_t s);

#ifdef __HIPCC__
// ---- elements of fp32 and bf16 tensors, several at a time ---------------------------------------------
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t bf16_pair(float lo, float hi) {  // to nearest, ties to even
    const bf16x2 v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}
__device__ inline float4 load4(const float* p, int64_t i4) { return reinterpret_cast<const float4*>(p)[i4]; }
__device__ inline float4 load4(const uint16_t* p, int64_t i4) {
    const uint2 w = reinterpret_cast<const uint2*>(p)[i4];
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
}
__device__ inline void store4(float* p, int64_t i4, const float4& v) { reinterpret_cast<float4*>(p)[i4] = v; }
__device__ inline void store4(uint16_t* p, int64_t i4, const float4& v) {
    reinterpret_cast<uint2*>(p)[i4] = make_uint2(bf16_pair(v.x, v.y), bf16_pair(v.z, v.w));
}
// The largest magnitude as the bits of a float: ordered as the numbers are, and an infinity and then NaN behind them all, which
// a maximum of floats would drop.
struct OpMostBits {
    __device__ int operator()(int a, int b) const { return a > b ? a : b; }
};
__device__ inline int most_bits(int m, float v) { return OpMostBits{}(m, __float_as_int(v) & 0x7fffffff); }
__device__ inline int most_bits(int m, const float4& v) {
    return most_bits(most_bits(most_bits(most_bits(m, v.x), v.y), v.z), v.w);
}
#endif

}  // namespace bl
