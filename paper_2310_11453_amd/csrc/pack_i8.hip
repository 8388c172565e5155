// The quantiser of 8-bit weights, a scale for each output channel:
//   m_n = max_k |W_nk|,  scale_n = m_n / 127,  code_nk = clamp(rne(W_nk * (127 / m_n)), -127, 127)
// into the tiles of i8.h, and back to the values that the codes stand for.
#include "common.h"
#include "i8.h"
#include "rowops.h"

namespace bl {

// m below this has no 127 / m in fp32: its codes have a step of 2^-127
constexpr float kLeastMost = 127.f * 0x1p-127f;

// One wave a row, eight rows of a tile a workgroup: 128 bytes, a line, of every 16 columns.
template <typename T>
__global__ __launch_bounds__(512) void pack_i8_rows(PackI8Args a) {
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
    const int64_t K4 = a.K / 4, TK = i8_tiles_k(a.K), rows = tiles_n(a.N) * 16;
    for (int64_t n = (int64_t)blockIdx.x * 8 + w; n < rows; n += (int64_t)gridDim.x * 8) {
        const bool in = n < a.N;
        const T* src = static_cast<const T*>(a.W) + (in ? n : 0) * a.K;
        uint8_t* dst = a.packed + (n / 16) * TK * 1024 + (n % 16) * 16;
        float m = 0.f;
        if constexpr (sizeof(T) != 1) {
            for (int64_t i = l; i < K4; i += kWave) {
                const float4 v = load4(src, i);
                m = fmaxf(m, fmaxf(fmaxf(fabsf(v.x), fabsf(v.y)), fmaxf(fabsf(v.z), fabsf(v.w))));
            }
            m = wave_max(m);
        }
        if (m > 0.f) m = fmaxf(m, kLeastMost);
        const float up = m > 0.f ? 127.0f / m : 0.f;
        for (int64_t i = l; i < TK * 16; i += kWave) {
            uint32_t c = 0;
            if (in && i < K4) {
                if constexpr (sizeof(T) == 1) {
                    c = reinterpret_cast<const uint32_t*>(src)[i];
                } else {
                    const float4 v = load4(src, i);
                    c = code_word(v.x * up, v.y * up, v.z * up, v.w * up, -127.f);
                }
            }
            *reinterpret_cast<uint32_t*>(dst + (i / 16) * 1024 + (i % 16 / 4) * 256 + (i % 4) * 4) = c;
        }
        if constexpr (sizeof(T) != 1)
            if (l == 0 && in) a.scale[n] = m / 127.0f;
    }
}
hipError_t launch_pack_i8(const PackI8Args& a, hipStream_t s) {
    const int64_t wgs = tiles_n(a.N) * 2;
    const unsigned grid = (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
    if (a.type == kF32) pack_i8_rows<float><<<grid, 512, 0, s>>>(a);
    else if (a.type == kBF16) pack_i8_rows<uint16_t><<<grid, 512, 0, s>>>(a);
    else pack_i8_rows<int8_t><<<grid, 512, 0, s>>>(a);
    return hipGetLastError();
}

// One wave a row.
template <int TYPE>
__global__ __launch_bounds__(512) void unpack_i8_rows(UnpackI8Args a) {
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave;
    const int64_t K4 = a.K / 4, TK = i8_tiles_k(a.K);
    for (int64_t n = (int64_t)blockIdx.x * 8 + w; n < a.N; n += (int64_t)gridDim.x * 8) {
        const uint8_t* src = a.packed + (n / 16) * TK * 1024 + (n % 16) * 16;
        const float sc = TYPE == kI8 ? 0.f : a.scale[n];
        for (int64_t i = l; i < K4; i += kWave) {
            const uint32_t c = *reinterpret_cast<const uint32_t*>(src + (i / 16) * 1024 + (i % 16 / 4) * 256 + (i % 4) * 4);
            if constexpr (TYPE == kI8) {
                reinterpret_cast<uint32_t*>(static_cast<int8_t*>(a.out) + n * a.K)[i] = c;
            } else {
                const float4 v = make_float4((float)(int8_t)c * sc, (float)(int8_t)(c >> 8) * sc,
                                             (float)(int8_t)(c >> 16) * sc, (float)(int8_t)(c >> 24) * sc);
                if constexpr (TYPE == kF32) store4(static_cast<float*>(a.out) + n * a.K, i, v);
                else store4(static_cast<uint16_t*>(a.out) + n * a.K, i, v);
            }
        }
    }
}
hipError_t launch_unpack_i8(const UnpackI8Args& a, hipStream_t s) {
    const int64_t wgs = (a.N + 7) / 8;
    const unsigned grid = (unsigned)(wgs < (1 << 20) ? wgs : (1 << 20));
    if (a.type == kF32) unpack_i8_rows<kF32><<<grid, 512, 0, s>>>(a);
    else if (a.type == kBF16) unpack_i8_rows<kBF16><<<grid, 512, 0, s>>>(a);
    else unpack_i8_rows<kI8><<<grid, 512, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace bl
