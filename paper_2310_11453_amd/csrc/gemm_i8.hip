// int8 x int8 product with scales for each token and channel:
//   acc[m][n] = sum_k q[m][k] * w[n][k]  (int32, at most 2^14 K <= 2^30),   Y[m][n] = float(acc) * (scale_n * (gamma_m / 128))
#include "common.h"
#include "i8.h"
#include "kernels.h"
#include "ring.h"

namespace bl {

// ---- tiles ---------------------------------------------------------------------------------------------
// T x T of the output a workgroup, four waves of T/2 x T/2 on v_mfma_i32_32x32x32_i8, persistent over the tiles.  A stage is 64 k: a
// row of codes has 64 bytes of it, 16 channels a tile of the packed weights, both streamed global -> LDS by
// global_load_lds_dwordx4 into a ring of NS stages.  The 16-byte pieces of a row of codes are XOR-swizzled with (row / 4) % 4;
// the weights' tiles are the operands' own layout and need no swizzle.  The schedule is that of the bf16 product of backward.hip,
// whose operands and stages have the same bytes: a half-step (32 k) is one MFMA for each pair of blocks, the next one's operands
// are read behind the first row of them, and between the half-steps of stage st every wave waits for its own DMA of stage st + 1,
// meets the others at a bare barrier and requests stage st + NS - 1 into the buffer that stage st - 1 has left.
__device__ inline void i8_issue(v4i (&a)[4], v4i (&b)[4], uint32_t ad_a, uint32_t ad_b) {
    asm volatile(
        "ds_read_b128 %0, %8\n\t"
        "ds_read_b128 %1, %8 offset:2048\n\t"
        "ds_read_b128 %2, %8 offset:4096\n\t"
        "ds_read_b128 %3, %8 offset:6144\n\t"
        "ds_read_b128 %4, %9\n\t"
        "ds_read_b128 %5, %9 offset:2048\n\t"
        "ds_read_b128 %6, %9 offset:4096\n\t"
        "ds_read_b128 %7, %9 offset:6144"
        : "=&v"(a[0]), "=&v"(a[1]), "=&v"(a[2]), "=&v"(a[3]), "=&v"(b[0]), "=&v"(b[1]), "=&v"(b[2]), "=&v"(b[3])
        : "v"(ad_a), "v"(ad_b));
}
__device__ inline void i8_wait(v4i (&a)[4], v4i (&b)[4]) {
    asm volatile("s_waitcnt lgkmcnt(0)"
                 : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(b[0]), "+v"(b[1]), "+v"(b[2]), "+v"(b[3]));
}
__device__ inline void i8_issue(v4i (&a)[2], v4i (&b)[2], uint32_t ad_a, uint32_t ad_b) {
    asm volatile(
        "ds_read_b128 %0, %4\n\t"
        "ds_read_b128 %1, %4 offset:2048\n\t"
        "ds_read_b128 %2, %5\n\t"
        "ds_read_b128 %3, %5 offset:2048"
        : "=&v"(a[0]), "=&v"(a[1]), "=&v"(b[0]), "=&v"(b[1])
        : "v"(ad_a), "v"(ad_b));
}
__device__ inline void i8_wait(v4i (&a)[2], v4i (&b)[2]) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a[0]), "+v"(a[1]), "+v"(b[0]), "+v"(b[1]));
}

enum I8Out { kOutF32 = 0, kOutBF16 = 1, kOutAcc = 2, kOutPart = 3 };  // kOutPart: a slice's int32 sums
struct I8Plan {
    int tile, grid, gm, gn;  // rows and columns of tiles
    int splits, per;         // slices of K, of `per` stages
};

template <int T, int NS, int OUT>
__global__ __launch_bounds__(256, T == 256 ? 1 : 2) void gemm_i8_tiles(GemmI8Args a, I8Plan p) {
    constexpr int THREADS = 256, WT = T / 2, MI = T / 64, PA = T * 4 / THREADS, P = 2 * PA;
    constexpr int A_BYTES = T * 64, STAGE_BYTES = 2 * A_BYTES;
    constexpr bool SPLIT = OUT == kOutPart;
    static_assert((NS - 1) * P < 64, "vmcnt range");
    static_assert(PA == MI, "a piece of the codes and one of the weights for each row of MFMAs");
    __shared__ __attribute__((aligned(1024))) uint8_t sm[NS * STAGE_BYTES];
    __shared__ float sm_gamma[2][T];

    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x % kWave;
    const int wm = w / 2, wn = w % 2, j = l & 31, g2 = l >> 5;
    const int64_t K = a.K, TK = i8_tiles_k(K);
    const int nst_all = (int)TK;
    const bool odd = (K & 63) != 0;  // the last stage is half a stage
    int nst = nst_all, st0 = 0;
    int main_groups = 0;

    // An XCD's workgroups (every eighth) take a contiguous eighth of the items: slice by slice, in bands of H rows of
    // tiles with the rows fastest, so that what an XCD runs together is about square and shares its operands in one L2.
    const int ntiles = p.gm * p.gn, nitems = ntiles * (SPLIT ? p.splits : 1), G8 = (int)gridDim.x >> 3;
    const int x = (int)blockIdx.x & 7;
    const int first = (int)((int64_t)nitems * x / 8), len = (int)((int64_t)nitems * (x + 1) / 8) - first;
    int q_item = (int)blockIdx.x >> 3;
    if (q_item >= len) return;  // uniform for the whole workgroup
    int slice = 0;
    auto origin = [&](int item, int64_t& m0, int64_t& n0) {
        constexpr int H = 4;
        int tile = first + item;
        if constexpr (SPLIT) {
            slice = tile / ntiles;
            tile -= slice * ntiles;
            st0 = slice * p.per;
            nst = nst_all - st0 < p.per ? nst_all - st0 : p.per;
        }
        main_groups = nst >= 2 * NS - 1 ? (nst - (2 * NS - 1)) / NS + 1 : 0;
        const int band = tile / (H * p.gn), rem = tile - band * H * p.gn;
        const int rows = p.gm - band * H < H ? p.gm - band * H : H;
        m0 = (int64_t)(band * H + rem % rows) * T;
        n0 = (int64_t)(rem / rows) * T;
    };

    // thread -> PA pieces of 16 bytes of each operand.  Rows past the last token re-read it, tiles past the last one
    // that one: their results are never stored.
    uint32_t goffA[PA], goffB[PA];
    const uint8_t *baseA = nullptr, *baseB = nullptr;
    const int seg = (((int)threadIdx.x & 3) ^ (((int)threadIdx.x >> 4) & 3)) * 16;  // the same in all of a thread's rows
    auto setup_dma = [&](int64_t m0, int64_t n0) {
#pragma unroll
        for (int q = 0; q < PA; ++q) {
            int row = (q * THREADS + (int)threadIdx.x) >> 2;
            if (m0 + row > a.M - 1) row = (int)(a.M - 1 - m0);
            goffA[q] = (uint32_t)row * (uint32_t)K + (uint32_t)seg;
            int tile = q * 4 + w;
            const int last = (int)(tiles_n(a.N) - 1 - n0 / 16);
            if (tile > last) tile = last;
            goffB[q] = (uint32_t)tile * (uint32_t)(TK * 1024) + (uint32_t)l * 16;
        }
        baseA = reinterpret_cast<const uint8_t*>(a.codes) + m0 * K + (int64_t)st0 * 64;
        baseB = a.packed + (n0 / 16 * TK + st0) * 1024;
    };
    const uint32_t lds_wave = (uint32_t)(w * kWave * 16);
    // stage `st` into ring slot st % NS; `src` is the stage whose bytes are read (== st, or the last one when st does not
    // exist: the slot is filled with bytes nobody uses).  The second half of the odd last stage is behind the row: the
    // first half again, against zeros.
    auto issue_piece = [&](int st, int src, int q) {
        uint8_t* dst = sm + (st % NS) * STAGE_BYTES + lds_wave + q * THREADS * 16;
        uint32_t off = goffA[q];
        if (odd && st0 + src == nst_all - 1) off -= (uint32_t)(seg & 32);  // uniform
        __builtin_amdgcn_global_load_lds((const void*)(baseA + src * 64 + off),
                                         (__attribute__((address_space(3))) void*)dst, 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const void*)(baseB + src * 1024 + goffB[q]),
                                         (__attribute__((address_space(3))) void*)(dst + A_BYTES), 16, 0, 0);
    };
    auto issue_tile_start = [&]() {
#pragma unroll
        for (int s = 0; s < NS - 1; ++s)
#pragma unroll
            for (int q = 0; q < PA; ++q) issue_piece(s, s < nst ? s : nst - 1, q);
    };

    // lane's operand addresses inside a stage, for either half
    const uint32_t smb = (uint32_t)(uintptr_t)sm;
    const int sw = (j >> 2) & 3;
    const uint32_t a_row = smb + (wm * WT + j) * 64;
    const uint32_t a_lane[2] = {a_row + (g2 ^ sw) * 16, a_row + ((2 + g2) ^ sw) * 16};
    const uint32_t b_row = smb + A_BYTES + (wn * (WT / 16) + (j >> 4)) * 1024 + (j & 15) * 16;
    const uint32_t b_lane[2] = {b_row + g2 * 256, b_row + (2 + g2) * 256};
    auto ring = [&](int st) { return (uint32_t)((st % NS) * STAGE_BYTES); };

    v16i acc[MI][MI];
    v4i ax[MI], ay[MI], bx[MI], by[MI];
    auto half_step = [&](const v4i(&ac)[MI], const v4i(&bc)[MI], v4i(&an)[MI], v4i(&bn)[MI], uint32_t ad_a, uint32_t ad_b,
                         auto between) {
#pragma unroll
        for (int mi = 0; mi < MI; ++mi) {
#pragma unroll
            for (int s = 0; s < MI; ++s) acc[mi][s] = __builtin_amdgcn_mfma_i32_32x32x32_i8(ac[mi], bc[s], acc[mi][s], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (mi == 0) i8_issue(an, bn, ad_a, ad_b);
            between(mi);
            __builtin_amdgcn_sched_barrier(0);
        }
        i8_wait(an, bn);
    };
    // In: ax/bx = operands of (st, half 0).  Out: operands of (st + 1, half 0); for the last stage stale bytes that nobody uses.
    auto stage = [&](int st, bool ahead) {
        half_step(ax, bx, ay, by, a_lane[1] + ring(st), b_lane[1] + ring(st), [](int) {});
        if (ahead) wait_vmcnt<(NS - 3) * P>();  // younger than stage st + 1: stages st + 2 .. st + NS - 2
        else wait_vmcnt<0>();
        block_barrier();
        half_step(ay, by, ax, bx, a_lane[0] + ring(st + 1), b_lane[0] + ring(st + 1), [&](int mi) {
            if (ahead) issue_piece(st + NS - 1, st + NS - 1, mi);
        });
    };

    int64_t m0, n0;
    origin(q_item, m0, n0);
    setup_dma(m0, n0);
    issue_tile_start();
    int parity = 0;
    while (true) {
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int s = 0; s < MI; ++s)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mi][s][r] = 0;
        wait_vmcnt<(NS - 2) * P>();  // younger than stage 0: stages 1 .. NS - 2
        block_barrier();
        i8_issue(ax, bx, a_lane[0], b_lane[0]);
        i8_wait(ax, bx);

        for (int gidx = 0; gidx < main_groups; ++gidx)
            static_for<0, NS>([&](auto ic) { stage(gidx * NS + decltype(ic)::value, true); });
        for (int st = main_groups * NS; st < nst; ++st) stage(st, st + NS - 1 < nst);

        // the tile's factors, behind the waits of its stages
        if constexpr (OUT == kOutF32 || OUT == kOutBF16) {
            if (threadIdx.x < T) {
                const int64_t m = m0 + threadIdx.x;
                sm_gamma[parity][threadIdx.x] = (a.per_tensor ? *a.gamma : a.gamma[m < a.M ? m : a.M - 1]) * (1.0f / 128.0f);
            }
        }
        float sc[MI];
#pragma unroll
        for (int s = 0; s < MI; ++s) {
            const int64_t n = n0 + wn * WT + 32 * s + j;
            sc[s] = OUT == kOutF32 || OUT == kOutBF16 ? a.scale[n < a.N ? n : a.N - 1] : 0.f;
        }
        // every wave is done with the ring (and sees the factors): start the next tile's stream, then store
        __syncthreads();
        const int64_t mt = m0, nt = n0;
        const int sl = slice;
        q_item += G8;
        const bool more = q_item < len;
        if (more) {
            origin(q_item, m0, n0);
            setup_dma(m0, n0);
            issue_tile_start();
        }
        const int64_t mb = mt + __builtin_amdgcn_readfirstlane(wm * WT), nb = nt + __builtin_amdgcn_readfirstlane(wn * WT);
        const float* gm = sm_gamma[parity] + wm * WT + 4 * g2;
        if constexpr (OUT == kOutBF16) {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t m = mb + 32 * mi + 8 * (r >> 2) + 4 * g2 + (r & 3);
                    const float g = gm[32 * mi + 8 * (r >> 2) + (r & 3)];
                    if (m >= a.M) continue;
#pragma unroll
                    for (int s = 0; s < MI; ++s) {
                        const int64_t n = nb + 32 * s + j;
                        if (n < a.N)
                            static_cast<uint16_t*>(a.Y)[m * a.N + n] = (uint16_t)bf16_pair((float)acc[mi][s][r] * (sc[s] * g), 0.f);
                    }
                }
        } else {
#pragma unroll
            for (int mi = 0; mi < MI; ++mi)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t m = mb + 32 * mi + 8 * (r >> 2) + 4 * g2 + (r & 3);
                    const float g = OUT == kOutF32 ? gm[32 * mi + 8 * (r >> 2) + (r & 3)] : 0.f;
                    if (m >= a.M) continue;
#pragma unroll
                    for (int s = 0; s < MI; ++s) {
                        const int64_t n = nb + 32 * s + j;
                        if (n >= a.N) continue;
                        if constexpr (OUT == kOutPart) a.part[((int64_t)sl * a.M + m) * a.N + n] = acc[mi][s][r];
                        else if constexpr (OUT == kOutAcc) static_cast<int32_t*>(a.Y)[m * a.N + n] = acc[mi][s][r];
                        else __builtin_nontemporal_store((float)acc[mi][s][r] * (sc[s] * g), &static_cast<float*>(a.Y)[m * a.N + n]);
                    }
                }
        }
        if (!more) break;
        parity ^= 1;
    }
}

// ---- slices of K added, then scaled ----------------------------------------------------------------------
template <int OUT>
__global__ __launch_bounds__(256) void fold_i8(GemmI8Args a, int splits) {
    const int64_t count = a.M * a.N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        int32_t v = a.part[i];
        for (int s = 1; s < splits; ++s) v += a.part[s * count + i];
        if constexpr (OUT == kOutAcc) {
            static_cast<int32_t*>(a.Y)[i] = v;
        } else {
            const int64_t m = i / a.N, n = i - m * a.N;
            const float y = (float)v * (a.scale[n] * ((a.per_tensor ? *a.gamma : a.gamma[m]) * (1.0f / 128.0f)));
            if constexpr (OUT == kOutBF16) static_cast<uint16_t*>(a.Y)[i] = (uint16_t)bf16_pair(y, 0.f);
            else static_cast<float*>(a.Y)[i] = y;
        }
    }
}

// A wave takes 16 rows of weights and 16 tokens; both operands come from memory as the MFMA wants them.
__global__ __launch_bounds__(256) void gemm_i8_plain(GemmI8Args a, int64_t items, int64_t tn) {
    const int w = threadIdx.x / kWave, l = threadIdx.x % kWave, c = l & 15, g = l >> 4;
    const int64_t TK = i8_tiles_k(a.K);
    for (int64_t it = (int64_t)blockIdx.x * 4 + w; it < items; it += (int64_t)gridDim.x * 4) {
        const int64_t tile = it % tn, m0 = it / tn * 16;
        const int64_t m = m0 + c < a.M ? m0 + c : a.M - 1;
        const v4i* wt = reinterpret_cast<const v4i*>(a.packed + tile * TK * 1024) + l;
        const int8_t* q = a.codes + m * a.K;
        v4i acc = {0, 0, 0, 0};
        for (int64_t t = 0; t < TK; ++t) {
            int64_t k = t * 64 + 16 * g;
            if (k >= a.K) k = 0;  // the weights there are zeros
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(wt[t * 64], *reinterpret_cast<const v4i*>(q + k), acc, 0, 0, 0);
        }
        if (m0 + c >= a.M) continue;
        const float gm = a.out_acc ? 0.f : (a.per_tensor ? *a.gamma : a.gamma[m]) * (1.0f / 128.0f);  // (null with out_acc)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t n = tile * 16 + 4 * g + r;
            if (n >= a.N) continue;
            const int64_t at = m * a.N + n;
            if (a.out_acc) {
                static_cast<int32_t*>(a.Y)[at] = acc[r];
            } else {
                const float y = (float)acc[r] * (a.scale[n] * gm);
                if (a.y_bf16) static_cast<uint16_t*>(a.Y)[at] = (uint16_t)bf16_pair(y, 0.f);
                else static_cast<float*>(a.Y)[at] = y;
            }
        }
    }
}

// Cost in us of tiles in slices: rounds of workgroups, each of `per` stages.
static I8Plan i8_plan(int64_t M, int64_t N, int64_t K) {
    const Tuning& t = tuning();
    const int64_t cus = num_cus(), nst = i8_tiles_k(K);
    I8Plan best{};
    double least = 1e30;
    for (int T = 256; T >= 128; T /= 2) {
        if (t.i8_tile && t.i8_tile != (T == 256 ? 1 : 2)) continue;
        const int64_t gm = (M + T - 1) / T, gn = (N + T - 1) / T, tiles = gm * gn;
        const int64_t force = t.i8_splits > 0 ? t.i8_splits : 0;
        for (int64_t n = force ? force : 1; n <= (force ? force : 16); ++n) {
            const int64_t per = (nst + n - 1) / n, splits = (nst + per - 1) / per, items = tiles * splits;
            if (n > 1 && !force && (per < 4 || splits != n || items > 4 * cus)) continue;
            const double stage = T == 256 ? 0.62 : 0.22, item = T == 256 ? 12.0 : 4.5;
            const int64_t slots = T == 256 ? cus : items > cus ? 2 * cus : cus;
            const int64_t rounds = (items + slots - 1) / slots;
            double cost = (double)rounds * (stage * (slots > cus ? 1.75 : 1.0) * (double)per + item);
            if (splits > 1) cost += 4.0 + (double)(M * N) * 4.0 * (double)splits * 2e-6 / 5.0;
            if (cost < least) {
                least = cost;
                const int64_t cap = T == 256 ? cus : 2 * cus, up = (items + 7) / 8 * 8;
                best = I8Plan{T, (int)(up < cap ? up : cap), (int)gm, (int)gn, (int)splits, (int)per};
            }
        }
    }
    return best;
}
static I8Plan unsliced(I8Plan p, int64_t K) {
    const int64_t tiles = (int64_t)p.gm * p.gn, up = (tiles + 7) / 8 * 8;
    if (p.grid > up) p.grid = (int)up;
    p.splits = 1;
    p.per = (int)i8_tiles_k(K);
    return p;
}
static bool few_tokens(int64_t M) { return M <= 64; }

size_t gemm_i8_part_bytes(int64_t M, int64_t N, int64_t K) {
    if (M == 0 || few_tokens(M)) return 0;
    const I8Plan p = i8_plan(M, N, K);
    return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)N * 4 : 0;
}
hipError_t launch_gemm_i8(const GemmI8Args& a, hipStream_t s) {
    const int out = a.out_acc ? kOutAcc : a.y_bf16 ? kOutBF16 : kOutF32;
    if (few_tokens(a.M)) {
        const int64_t tn = tiles_n(a.N), items = tn * ((a.M + 15) / 16), wgs = (items + 3) / 4;
        gemm_i8_plain<<<(unsigned)(wgs < (1 << 20) ? wgs : (1 << 20)), 256, 0, s>>>(a, items, tn);
        return hipGetLastError();
    }
    I8Plan p = i8_plan(a.M, a.N, a.K);
    if (p.splits > 1 && (size_t)p.splits * (size_t)a.M * (size_t)a.N * 4 > a.part_bytes) p = unsliced(p, a.K);
    const int kind = p.splits > 1 ? kOutPart : out;
    auto pick = [&](auto t) {
        constexpr int T = decltype(t)::value;
        return kind == kOutPart ? gemm_i8_tiles<T, 4, kOutPart>
             : kind == kOutAcc  ? gemm_i8_tiles<T, 4, kOutAcc>
             : kind == kOutBF16 ? gemm_i8_tiles<T, 4, kOutBF16>
                                : gemm_i8_tiles<T, 4, kOutF32>;
    };
    const auto kernel = p.tile == 256 ? pick(std::integral_constant<int, 256>{}) : pick(std::integral_constant<int, 128>{});
    kernel<<<(unsigned)p.grid, 256, 0, s>>>(a, p);
    if (p.splits > 1) {
        const int64_t wgs = (a.M * a.N + 255) / 256;
        const auto fold = out == kOutAcc ? fold_i8<kOutAcc> : out == kOutBF16 ? fold_i8<kOutBF16> : fold_i8<kOutF32>;
        fold<<<(unsigned)(wgs < (1 << 16) ? wgs : (1 << 16)), 256, 0, s>>>(a, p.splits);
    }
    return hipGetLastError();
}

}  // namespace bl
