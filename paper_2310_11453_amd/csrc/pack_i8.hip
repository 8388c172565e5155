// The quantiser of 8-bit weights, a scale for each output channel:
//   m_n = max_k |W_nk|,  scale_n = m_n / 127,  code_nk = clamp(rne(W_nk * (127 / m_n)), -127, 127)
// into the tiles of i8.h, and back to the values that the codes stand for.
#include <type_traits>

#include "common.h"
#include "i8.h"
#include "rowops.h"

namespace bl {

// m below this has no 127 / m in fp32: its codes have a step of 2^-127
constexpr float kLeastMost = 127.f * 0x1p-127f;

template <typename T>
struct Four {  // four elements as they lie
    using Raw = std::conditional_t<sizeof(T) == 1, uint32_t, std::conditional_t<sizeof(T) == 2, uint2, float4>>;
};
__device__ inline float4 values(const float4& v) { return v; }
__device__ inline float4 values(const uint2& w) {
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                       __uint_as_float(w.y & 0xffff0000u));
}

// Eight rows, half a tile, a workgroup: WR waves a row, whose 16 float4 a lane lie in registers, so that rows of 4096 WR
// are read once; of longer ones all but the last chunk is read again, from the end, out of the caches.  The codes go
// through LDS and leave as whole lines of 128 bytes: eight rows of 16 columns.  Bound by HBM: 16384 x 4096 fp32
// 75 us (4.5 TB/s), bf16 35 us (5.7; 46 where the registers held it as fp32), 2048 x 8192 bf16 14 us (3.7); rows past
// registers, 4096 x 16384 fp32, 92 us (3.7).
template <typename T, int WR>
__global__ __launch_bounds__(512 * WR, sizeof(T) < 4 ? 8 : 4) void pack_i8_rows(PackI8Args a) {
    constexpr int NV = 16, LANES = 64 * WR, CHUNK = LANES * NV * 4;
    constexpr bool CODES = sizeof(T) == 1;
    using Raw = typename Four<T>::Raw;
    __shared__ __attribute__((aligned(16))) uint8_t codes[8][CHUNK + 16];
    __shared__ int most[8][WR];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), r = wave / WR;
    const int t = wave % WR * kWave + ((int)threadIdx.x & (kWave - 1));
    const int64_t K4 = a.K / 4, TK = i8_tiles_k(a.K), rows = tiles_n(a.N) * 16;
    const int chunks = (int)((a.K + CHUNK - 1) / CHUNK);
    for (int64_t n0 = (int64_t)blockIdx.x * 8; n0 < rows; n0 += (int64_t)gridDim.x * 8) {
        const int64_t n = n0 + r;
        const bool in = n < a.N;
        const T* src = static_cast<const T*>(a.W) + (in ? n : a.N - 1) * a.K;
        Raw v[NV];
        auto load = [&](int c) {
            const int64_t first = (int64_t)c * (CHUNK / 4);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (first + j * LANES < K4) {  // uniform
                    const int64_t i = first + j * LANES + t;
                    v[j] = reinterpret_cast<const Raw*>(src)[i < K4 ? i : K4 - 1];
                }
        };
        int bits = 0;
        for (int c = 0; c < chunks; ++c) {
            if (CODES && c < chunks - 1) continue;
            load(c);
            if constexpr (!CODES) {
                const int64_t first = (int64_t)c * (CHUNK / 4);
#pragma unroll
                for (int j = 0; j < NV; ++j)  // (the row's last element again past it)
                    if (first + j * LANES < K4) bits = most_bits(bits, values(v[j]));
            }
        }
        float up = 0.f;
        if constexpr (!CODES) {
            bits = wave_reduce(bits, OpMostBits{});
            if constexpr (WR > 1) {
                if ((threadIdx.x & (kWave - 1)) == 0) most[r][wave % WR] = bits;
                __syncthreads();
                bits = fold_slots<WR>(most[r], OpMostBits{});
            }
            float m = __int_as_float(bits);  // (a NaN stays one, and so does the scale)
            if (m > 0.f) m = fmaxf(m, kLeastMost);
            up = m > 0.f ? 127.0f / m : 0.f;
            if (t == 0 && in) a.scale[n] = m / 127.0f;
        }
        for (int c = chunks - 1; c >= 0; --c) {
            if (c < chunks - 1) load(c);
            const int64_t first = (int64_t)c * (CHUNK / 4);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (first + j * LANES < TK * 16) {  // uniform
                    uint32_t w;
                    if constexpr (CODES) {
                        w = v[j];
                    } else {
                        const float4 f = values(v[j]);
                        w = code_word(f.x * up, f.y * up, f.z * up, f.w * up, -127.f);
                    }
                    // zeros in what is filled up
                    *reinterpret_cast<uint32_t*>(&codes[r][(j * LANES + t) * 4]) = in && first + j * LANES + t < K4 ? w : 0u;
                }
            __syncthreads();
            const int64_t units = TK * 4 - (int64_t)c * (CHUNK / 16);
            uint8_t* dst = a.packed + (n0 / 16 * TK + (int64_t)c * (CHUNK / 64)) * 1024 + n0 % 16 * 16;
            for (int i = threadIdx.x; i < CHUNK / 16 * 8 && i / 8 < units; i += 512 * WR)
                *reinterpret_cast<uint4*>(dst + i / 8 * 256 + i % 8 * 16) =
                    *reinterpret_cast<const uint4*>(&codes[i % 8][i / 8 * 16]);
            __syncthreads();
        }
    }
}
template <typename T>
static void launch_pack_typed(const PackI8Args& a, hipStream_t s) {
    const int64_t wgs = tiles_n(a.N) * 2;
    const unsigned grid = (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
    if (a.K <= 4096) pack_i8_rows<T, 1><<<grid, 512, 0, s>>>(a);
    else pack_i8_rows<T, 2><<<grid, 1024, 0, s>>>(a);
}
hipError_t launch_pack_i8(const PackI8Args& a, hipStream_t s) {
    if (a.type == kF32) launch_pack_typed<float>(a, s);
    else if (a.type == kBF16) launch_pack_typed<uint16_t>(a, s);
    else launch_pack_typed<int8_t>(a, s);
    return hipGetLastError();
}

// A workgroup takes 2048 columns of the eight rows that share lines of 128 bytes, a wave a row: eight dwords a lane, all
// in flight before the first is used: 16384 x 4096 to bf16 32 us (6.3 TB/s).  (Rows dealt to workgroups without regard to
// the lines: with the quantiser 107 -> 131 us, 16384 x 4096.)
constexpr int kUnpackColumns = 2048;
template <int TYPE>
__global__ __launch_bounds__(512) void unpack_i8_rows(UnpackI8Args a, int64_t items, int64_t pieces) {
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x % kWave;
    const int64_t K4 = a.K / 4, TK = i8_tiles_k(a.K);
    for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
        const int64_t group = it / pieces, n = group * 8 + w, first = (it - group * pieces) * (kUnpackColumns / 4);
        if (n >= a.N) continue;
        const uint8_t* src = a.packed + (n / 16) * TK * 1024 + (n % 16) * 16;
        const float sc = TYPE == kI8 ? 0.f : a.scale[n];
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            int64_t i = first + j * kWave + l;
            if (i >= K4) i = K4 - 1;
            c[j] = *reinterpret_cast<const uint32_t*>(src + (i / 16) * 1024 + (i % 16 / 4) * 256 + (i % 4) * 4);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t i = first + j * kWave + l;
            if (i >= K4) continue;
            if constexpr (TYPE == kI8) {
                reinterpret_cast<uint32_t*>(static_cast<int8_t*>(a.out) + n * a.K)[i] = c[j];
            } else {
                const float4 v = make_float4((float)(int8_t)c[j] * sc, (float)(int8_t)(c[j] >> 8) * sc,
                                             (float)(int8_t)(c[j] >> 16) * sc, (float)(int8_t)(c[j] >> 24) * sc);
                if constexpr (TYPE == kF32) store4(static_cast<float*>(a.out) + n * a.K, i, v);
                else store4(static_cast<uint16_t*>(a.out) + n * a.K, i, v);
            }
        }
    }
}
hipError_t launch_unpack_i8(const UnpackI8Args& a, hipStream_t s) {
    const int64_t pieces = (a.K + kUnpackColumns - 1) / kUnpackColumns, items = (a.N + 7) / 8 * pieces;
    const unsigned grid = (unsigned)(items < (1 << 20) ? items : (1 << 20));
    if (a.type == kF32) unpack_i8_rows<kF32><<<grid, 512, 0, s>>>(a, items, pieces);
    else if (a.type == kBF16) unpack_i8_rows<kBF16><<<grid, 512, 0, s>>>(a, items, pieces);
    else unpack_i8_rows<kI8><<<grid, 512, 0, s>>>(a, items, pieces);
    return hipGetLastError();
}

}  // namespace bl
