// int8 x int8 product with scales for each token and channel, and, in the same tiles, the bf16 products of its backward:
//   acc[m][n] = sum_k q[m][k] * w[n][k]  (int32, at most 2^14 K <= 2^30),   Y[m][n] = float(acc) * (scale_n * (gamma_m / 128))
#include <math.h>

#include "common.h"
#include "i8.h"
#include "kernels.h"
#include "ring.h"

namespace bl {

// ---- tiles ---------------------------------------------------------------------------------------------
// TM x TN of the output a workgroup, four waves of a quarter each on v_mfma_i32_32x32x32_i8, persistent over the tiles.
// A stage is 64 k: a row of codes has 64 bytes of it, 16 channels a tile of the packed weights, both streamed global ->
// LDS by global_load_lds_dwordx4 into a ring of NS stages.  The 16-byte pieces of a row of codes are XOR-swizzled with
// (row / 4) % 4; the weights' tiles are the operands' own layout and need no swizzle.  The schedule is that of the bf16
// product of backward.hip, whose operands and stages have the same bytes: a half-step (32 k) is one MFMA for each pair
// of blocks, the next one's operands are read one behind each of them (all behind the first ones they fill the LDS
// queue: 4096 x 4096 -> 16384 264 us, so 254), and between the half-steps of stage st every wave waits for its own DMA
// of stage st + 1, meets the others at a bare barrier and requests stage st + NS - 1 into the buffer that stage st - 1
// has left.  Measured, N x K: 8192 tokens, 8192 x 8192 447 us = 2.46 POP/s; 4096 tokens, 16384 x 4096, bf16 out 246 us =
// 2.23 POP/s, in four rounds of tiles whose starts and stores are a fifth of it; the matrix pipe is busy 56 % of the
// cycles at 1.83 GHz, without LDS bank conflicts.  bf16 operands, 8192 x 16384 x 4096: 1.28 PFLOP/s, busy 73 % at 1.63 GHz.
// One operand at a time, from block B of 32 rows (2 KiB in either operand); what waits for them is i8_wait.
template <int B>
__device__ inline void i8_read(v4i& x, uint32_t ad) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(x) : "v"(ad), "n"(B * 2048));
}
template <int MI, int NI>
__device__ inline void i8_wait(v4i (&a)[MI], v4i (&b)[NI]) {
    if constexpr (MI == 4 && NI == 4)
        asm volatile("s_waitcnt lgkmcnt(0)"
                     : "+v"(a[0]), "+v"(a[1]), "+v"(a[2]), "+v"(a[3]), "+v"(b[0]), "+v"(b[1]), "+v"(b[2]), "+v"(b[3]));
    else if constexpr (MI == 2)
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a[0]), "+v"(a[1]), "+v"(b[0]), "+v"(b[1]));
    else
        asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(a[0]), "+v"(b[0]), "+v"(b[1]));
}

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

enum I8Out { kOutF32 = 0, kOutBF16 = 1, kOutAcc = 2, kOutPart = 3 };  // kOutPart: a slice's sums
// What the tiles work on (REAL: bf16 operands, else int8).  A: 64 bytes of a row are a stage; B: 1 KiB of 16 rows.
struct TileArgs {
    const uint8_t *A, *B;
    int64_t a_pitch, a_step, b_pitch, b_step;  // bytes from row to row (tile to tile), from stage to stage
    int64_t M, N;
    int stages;
    bool odd;  // the last stage is half a stage: the second half of A is behind its rows, of B zeros
    // int8: Y = float(acc) * (scale[n] * (gamma[m] / 128)); REAL: acc * (*gamma (null: 1) * times)
    const float *gamma, *scale;
    bool per_tensor;
    float times;
    void *Y, *part;
};

// Stores a wave's blocks of 32 x 32: lane (j, g2) holds columns 32 s + j, rows 32 mi + 8 rq + 4 g2 + rr.  `rowp`, a
// scalar that is hidden from the optimiser (which would compute all the addresses ahead and spill), walks the rows; a
// lane's place in a row is one 32-bit offset.  With the rows' bounds, a 64-bit product and branches at every store the
// instructions around the stores took 12 us of a 256 x 256 tile.  bf16, two columns to a dword: a lane packs its values
// of two rows, exchanges with its neighbour and stores two columns of one of them, if rows begin at even elements of a
// 4-byte aligned output.  The output is streamed past the caches, where the operands are.
template <bool REAL, int OUT>
struct I8Store {
    typedef __attribute__((address_space(1))) uint8_t* gptr;
    static constexpr int ES = OUT == kOutBF16 ? 2 : 4;
    uint64_t first;
    int64_t pitch, rows, cols;
    int j, g2;
    bool pairs;
    __device__ I8Store(const TileArgs& a, int slice, int64_t mb, int64_t nb, int64_t rows_, int64_t cols_, int j_, int g2_)
        : pitch(a.N * ES), rows(rows_), cols(cols_), j(j_), g2(g2_) {
        uint8_t* base = OUT == kOutPart ? static_cast<uint8_t*>(a.part) + slice * a.M * a.N * 4 : static_cast<uint8_t*>(a.Y);
        const uint64_t at = (uint64_t)(uintptr_t)(base + mb * pitch + nb * ES);
        first = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)at) |
                (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) << 32;
        pairs = OUT == kOutBF16 && a.N % 2 == 0 && ((uintptr_t)a.Y & 3) == 0;
    }
    template <int MI, int NI, class GAMMA, class SC, class ACC>
    __device__ void all(GAMMA&& gamma, const SC& sc, const ACC& acc) const {
        const bool whole = rows >= 32 * MI && cols >= 32 * NI;  // uniform
        if constexpr (OUT == kOutBF16) {
            if (pairs) {
                if (whole) walk<MI, NI, false, true>(gamma, sc, acc);
                else walk<MI, NI, true, true>(gamma, sc, acc);
                return;
            }
        }
        if (whole) walk<MI, NI, false, false>(gamma, sc, acc);
        else walk<MI, NI, true, false>(gamma, sc, acc);
    }
    template <int MI, int NI, bool RAGGED, bool PAIRS, class GAMMA, class SC, class ACC>
    __device__ void walk(GAMMA&& gamma, const SC& sc, const ACC& acc) const {
        gptr rowp = (gptr)first;
        const int odd = PAIRS ? j & 1 : 0, col = j - odd;
        const int64_t lane = (4 * g2 + odd) * pitch + col * ES;
        const int mine = (int)(rows < 32 * MI ? rows : 32 * MI) - 4 * g2 - odd;  // this lane's rows end here
        const int last = (int)(cols < 32 * NI ? cols : 32 * NI) - col;           // and its columns
        // the neighbour's second row and its own; its own first and the neighbour's
        const uint32_t pick = odd ? 0x03020706u : 0x05040100u;
#pragma unroll
        for (int mi = 0; mi < MI; ++mi)
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
                v4f g{};
                if constexpr (!REAL && (OUT == kOutF32 || OUT == kOutBF16)) g = gamma(mi, rq);
                auto value = [&](int s, int rr) {
                    if constexpr (REAL) return acc[mi][s][4 * rq + rr] * sc[s];
                    else return (float)acc[mi][s][4 * rq + rr] * (sc[s] * g[rr]);
                };
#pragma unroll
                for (int rr = 0; rr < 4; rr += PAIRS ? 2 : 1) {
                    asm volatile("" : "+s"(rowp));
                    const bool in = !RAGGED || 32 * mi + 8 * rq + rr < mine;
#pragma unroll
                    for (int s = 0; s < NI; ++s) {
                        const int r = 4 * rq + rr;
                        if constexpr (PAIRS) {
                            const uint32_t p = bf16_pair(value(s, rr), value(s, rr + 1));
                            const uint32_t q = (uint32_t)__builtin_amdgcn_mov_dpp((int)p, 0xB1, 0xF, 0xF, true);
                            const uint32_t v = __builtin_amdgcn_perm(q, p, pick);
                            if (in && (!RAGGED || 32 * s < last))
                                __builtin_nontemporal_store(v, (__attribute__((address_space(1))) uint32_t*)(rowp + lane + 64 * s));
                        } else if (in && (!RAGGED || 32 * s < last)) {
                            const gptr at = rowp + lane + 32 * ES * s;
                            if constexpr (OUT == kOutBF16)
                                __builtin_nontemporal_store((uint16_t)bf16_pair(value(s, rr), 0.f),
                                                            (__attribute__((address_space(1))) uint16_t*)at);
                            else if constexpr (OUT == kOutF32)
                                __builtin_nontemporal_store(value(s, rr), (__attribute__((address_space(1))) float*)at);
                            else if constexpr (REAL) *(__attribute__((address_space(1))) float*)at = acc[mi][s][r];
                            else *(__attribute__((address_space(1))) int32_t*)at = acc[mi][s][r];
                        }
                    }
                    rowp += (PAIRS ? 2 : 1) * pitch;
                }
                rowp += 4 * pitch;
            }
    }
};

struct I8Plan {
    int tile, grid, gm, gn;  // which tile (kTiles); workgroups; rows and columns of tiles
    int splits, per;         // slices of K, of `per` stages
};

struct SecondProduct {
    TileArgs a;
    I8Plan p;
};
// SECOND: nothing, or a SecondProduct (REAL, into kOutF32, in one slice), whose workgroups are those behind the first p.grid.
template <bool REAL, int TM, int TN, int NS, int OUT, class... SECOND>
__global__ __launch_bounds__(256, NS * (TM + TN) * 64 > 80 * 1024 ? 1 : 2) void gemm_i8_tiles(
    TileArgs a, I8Plan p, SECOND... other) {
    constexpr int THREADS = 256, WTM = TM / 2, WTN = TN / 2, MI = WTM / 32, NI = WTN / 32;
    constexpr int PA = TM / 64, PB = TN / 64, P = PA + PB;
    constexpr int A_BYTES = TM * 64, STAGE_BYTES = A_BYTES + TN * 64;
    constexpr bool SPLIT = OUT == kOutPart;
    constexpr bool WHOLE = TM + TN < 512;         // a stage's operands in registers at once
    constexpr int AHEAD = WHOLE ? NS : NS - 1;    // stages requested ahead
    static_assert(AHEAD * P < 64, "vmcnt range");
    __shared__ __attribute__((aligned(1024))) uint8_t sm[NS * STAGE_BYTES];
    __shared__ __attribute__((aligned(16))) float sm_gamma[2][TM];

    constexpr bool TWO = sizeof...(SECOND) > 0;
    int block = (int)blockIdx.x, grid = (int)gridDim.x;
    bool second = false;
    if constexpr (TWO) {
        second = block >= p.grid;  // uniform
        if (second) {
            block -= p.grid;
            (..., (a = other.a, p = other.p));
        }
        grid = p.grid;
    }
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x % kWave;
    const int wm = w / 2, wn = w % 2, j = l & 31, g2 = l >> 5;
    const int nst_all = a.stages;
    const bool odd = !REAL && a.odd;
    int nst = nst_all, st0 = 0;
    int main_groups = 0;

    // An XCD's workgroups (every eighth) take a contiguous eighth of the items: slice by slice, in bands of H rows of
    // tiles with the rows fastest, so that what an XCD runs together is about square and shares its operands in one L2.
    const int ntiles = p.gm * p.gn, nitems = ntiles * (SPLIT ? p.splits : 1), G8 = grid >> 3;
    const int x = block & 7;
    const int first = (int)((int64_t)nitems * x / 8), len = (int)((int64_t)nitems * (x + 1) / 8) - first;
    int q_item = block >> 3;
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
        main_groups = nst >= NS + AHEAD ? (nst - NS - AHEAD) / NS + 1 : 0;  // of NS stages whose look-ahead exists
        const int band = tile / (H * p.gn), rem = tile - band * H * p.gn;
        const int rows = p.gm - band * H < H ? p.gm - band * H : H;
        m0 = (int64_t)(band * H + rem % rows) * TM;
        n0 = (int64_t)(rem / rows) * TN;
    };

    // thread -> PA + PB pieces of 16 bytes.  Rows past the last token re-read it, tiles past the last one
    // that one: their results are never stored.
    uint32_t goffA[PA], goffB[PB];
    const uint8_t *baseA = nullptr, *baseB = nullptr;
    const int seg = (((int)threadIdx.x & 3) ^ (((int)threadIdx.x >> 4) & 3)) * 16;  // the same in all of a thread's rows
    auto setup_dma = [&](int64_t m0, int64_t n0) {
#pragma unroll
        for (int q = 0; q < PA; ++q) {
            int row = (q * THREADS + (int)threadIdx.x) >> 2;
            if (m0 + row > a.M - 1) row = (int)(a.M - 1 - m0);
            goffA[q] = (uint32_t)row * (uint32_t)a.a_pitch + (uint32_t)seg;
        }
#pragma unroll
        for (int q = 0; q < PB; ++q) {
            int tile = q * 4 + w;
            const int last = (int)(tiles_n(a.N) - 1 - n0 / 16);
            if (tile > last) tile = last;
            goffB[q] = (uint32_t)tile * (uint32_t)a.b_pitch + (uint32_t)l * 16;
        }
        baseA = a.A + m0 * a.a_pitch + st0 * a.a_step;
        baseB = a.B + n0 / 16 * a.b_pitch + st0 * a.b_step;
    };
    const uint32_t lds_wave = (uint32_t)(w * kWave * 16);
    // stage `st` into ring slot st % NS; `src` is the stage whose bytes are read (== st, or the last one when st does not
    // exist: the slot is filled with bytes nobody uses).  The second half of the odd last stage is behind the row: the
    // first half again, against zeros.
    auto issue_piece = [&](int st, int src, int q) {
        uint8_t* dst = sm + (st % NS) * STAGE_BYTES + lds_wave;
        // in turn: codes, weights, codes, ... where there are as many of both
        const bool first_kind = PA == PB ? q % 2 == 0 : q < PA;
        const int b = PA == PB ? q / 2 : q < PA ? q : q - PA;
        if (first_kind) {
            uint32_t off = goffA[b < PA ? b : 0];
            if (odd && st0 + src == nst_all - 1) off -= (uint32_t)(seg & 32);  // uniform
            __builtin_amdgcn_global_load_lds((const void*)(baseA + src * a.a_step + off),
                                             (__attribute__((address_space(3))) void*)(dst + b * THREADS * 16), 16, 0, 0);
        } else {
            __builtin_amdgcn_global_load_lds((const void*)(baseB + src * a.b_step + goffB[b < PB ? b : 0]),
                                             (__attribute__((address_space(3))) void*)(dst + A_BYTES + b * THREADS * 16), 16, 0,
                                             0);
        }
    };
    auto issue_tile_start = [&]() {
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int q = 0; q < P; ++q) issue_piece(s, s < nst ? s : nst - 1, q);
    };

    // lane's operand addresses inside a stage, for either half
    const uint32_t smb = (uint32_t)(uintptr_t)sm;
    const int sw = (j >> 2) & 3;
    const uint32_t a_row = smb + (wm * WTM + j) * 64;
    const uint32_t a_lane[2] = {a_row + (g2 ^ sw) * 16, a_row + ((2 + g2) ^ sw) * 16};
    const uint32_t b_row = smb + A_BYTES + (wn * (WTN / 16) + (j >> 4)) * 1024 + (j & 15) * 16;
    const uint32_t b_lane[2] = {b_row + g2 * 256, b_row + (2 + g2) * 256};
    auto ring = [&](int st) { return (uint32_t)((st % NS) * STAGE_BYTES); };

    std::conditional_t<REAL, v16f, v16i> acc[MI][NI];
    auto mfma = [&](const v4i& x, const v4i& y, auto& c) {
        if constexpr (REAL)
            c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, y), c, 0, 0, 0);
        else
            c = __builtin_amdgcn_mfma_i32_32x32x32_i8(x, y, c, 0, 0, 0);
    };
    v4i ax[MI], ay[MI], bx[NI], by[NI];                              // of a half-step and the next
    v4i sa[WHOLE ? 2 : 1][2][MI], sb[WHOLE ? 2 : 1][2][NI];          // WHOLE: of the halves of a stage and of the next one
    // acc += ac x bc; an, bn = the operands at ad_a, ad_b, valid on return: one read behind each of the first MFMAs (all
    // behind one another they fill the LDS queue, and the wave's next MFMA waits for its place in it), then, one by one too,
    // between(q), the DMA of a stage
    auto half_step = [&](const v4i(&ac)[MI], const v4i(&bc)[NI], v4i(&an)[MI], v4i(&bn)[NI], uint32_t ad_a, uint32_t ad_b,
                         auto between) {
        constexpr int MFMAS = MI * NI, READS = MI + NI, PER = (READS + MFMAS - 1) / MFMAS, LATER = MFMAS - READS / PER;
        static_for<0, MFMAS>([&](auto ic) {
            constexpr int i = decltype(ic)::value, mi = i / NI, s = i % NI;
            mfma(ac[mi], bc[s], acc[mi][s]);
            __builtin_amdgcn_sched_barrier(0);
            static_for<i * PER, (i + 1) * PER>([&](auto rc) {
                constexpr int r = decltype(rc)::value;
                // in turn, so that the first MFMAs of the next half-step have both
                if constexpr (MI == NI) {
                    if constexpr (r < READS && r % 2 == 0) i8_read<r / 2>(an[r / 2], ad_a);
                    else if constexpr (r < READS) i8_read<r / 2>(bn[r / 2], ad_b);
                } else {
                    if constexpr (r < MI) i8_read<r>(an[r], ad_a);
                    else if constexpr (r < READS) i8_read<r - MI>(bn[r - MI], ad_b);
                }
            });
            if constexpr (LATER >= P) {
                if constexpr (i >= MFMAS - P) between(i - (MFMAS - P));
            } else {
#pragma unroll
                for (int q = i * P / MFMAS; q < (i + 1) * P / MFMAS; ++q) between(q);
            }
            __builtin_amdgcn_sched_barrier(0);
        });
        i8_wait(an, bn);
    };
    // the wait of a stage behind which nothing is requested any more: `younger` stages may still be on their way
    auto wait_last = [&](int younger) {
        bool waited = false;
        static_for<0, AHEAD - 1>([&](auto ic) {
            constexpr int y = AHEAD - 2 - decltype(ic)::value;
            if (!waited && younger >= y) {  // uniform
                wait_vmcnt<y * P>();
                waited = true;
            }
        });
        if (!waited) wait_vmcnt<0>();
    };
    // In: ax/bx = operands of (st, half 0).  Out: operands of (st + 1, half 0); for the last stage stale bytes that
    // nobody uses.
    auto stage = [&](int st, bool ahead) {
        half_step(ax, bx, ay, by, a_lane[1] + ring(st), b_lane[1] + ring(st), [](int) {});
        if (ahead) wait_vmcnt<(NS - 3) * P>();  // younger than stage st + 1: stages st + 2 .. st + NS - 2
        else wait_last(nst - 2 - st);
        block_barrier();
        half_step(ay, by, ax, bx, a_lane[0] + ring(st + 1), b_lane[0] + ring(st + 1), [&](int q) {
            if (ahead) issue_piece(st + NS - 1, st + NS - 1, q);
        });
    };

    // WHOLE: the operands of stage st are in registers F, those of st + 1 are read into 1 - F behind its MFMAs, and the stage
    // st + NS goes where st was, which every wave has read when it meets the others.  (With the operands of a half-step at a
    // time, 2 or 4 MFMAs do not hide a trip to LDS.)
    auto whole_stage = [&](auto fc, int st, bool ahead) {
        constexpr int F = decltype(fc)::value, G = 1 - F, MFMAS = 2 * MI * NI, READS = 2 * (MI + NI);
        constexpr int PER = (READS + MFMAS - 1) / MFMAS;
        if (ahead) wait_vmcnt<(NS - 2) * P>();  // younger than stage st + 1: stages st + 2 .. st + NS - 1
        else wait_last(nst - 2 - st);
        block_barrier();
        static_for<0, MFMAS>([&](auto ic) {
            constexpr int i = decltype(ic)::value, h = i / (MI * NI), mi = i % (MI * NI) / NI, s = i % NI;
            mfma(sa[F][h][mi], sb[F][h][s], acc[mi][s]);
            __builtin_amdgcn_sched_barrier(0);
            static_for<i * PER, (i + 1) * PER>([&](auto rc) {
                constexpr int r = decltype(rc)::value, hr = r / (MI + NI), k = r % (MI + NI);
                if constexpr (r < READS && k < MI) i8_read<k>(sa[G][hr][k], a_lane[hr] + ring(st + 1));
                else if constexpr (r < READS) i8_read<k - MI>(sb[G][hr][k - MI], b_lane[hr] + ring(st + 1));
            });
            if (ahead)
#pragma unroll
                for (int q = i * P / MFMAS; q < (i + 1) * P / MFMAS; ++q) issue_piece(st + NS, st + NS, q);
            __builtin_amdgcn_sched_barrier(0);
        });
        i8_wait(sa[G][0], sb[G][0]);
        i8_wait(sa[G][1], sb[G][1]);
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
            for (int s = 0; s < NI; ++s)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[mi][s][r] = 0;
        wait_vmcnt<(AHEAD - 1) * P>();  // younger than stage 0: stages 1 .. AHEAD - 1
        block_barrier();
        if constexpr (WHOLE) {
            static_for<0, 2>([&](auto hc) {
                constexpr int h = decltype(hc)::value;
                static_for<0, MI>([&](auto ic) { i8_read<decltype(ic)::value>(sa[0][h][decltype(ic)::value], a_lane[h]); });
                static_for<0, NI>([&](auto ic) { i8_read<decltype(ic)::value>(sb[0][h][decltype(ic)::value], b_lane[h]); });
            });
            i8_wait(sa[0][0], sb[0][0]);
            i8_wait(sa[0][1], sb[0][1]);
            static_assert(NS % 2 == 0, "the registers take turns");
            using Even = std::integral_constant<int, 0>;
            using Odd = std::integral_constant<int, 1>;
            for (int gidx = 0; gidx < main_groups; ++gidx)
                static_for<0, NS>([&](auto ic) {
                    whole_stage(std::integral_constant<int, decltype(ic)::value % 2>{}, gidx * NS + decltype(ic)::value, true);
                });
            int st = main_groups * NS;
            for (; st + 1 < nst; st += 2) {
                whole_stage(Even{}, st, st + NS < nst);
                whole_stage(Odd{}, st + 1, st + 1 + NS < nst);
            }
            if (st < nst) whole_stage(Even{}, st, false);
        } else {
            static_for<0, MI>([&](auto ic) { i8_read<decltype(ic)::value>(ax[decltype(ic)::value], a_lane[0]); });
            static_for<0, NI>([&](auto ic) { i8_read<decltype(ic)::value>(bx[decltype(ic)::value], b_lane[0]); });
            i8_wait(ax, bx);
            for (int gidx = 0; gidx < main_groups; ++gidx)
                static_for<0, NS>([&](auto ic) { stage(gidx * NS + decltype(ic)::value, true); });
            for (int st = main_groups * NS; st < nst; ++st) stage(st, st + NS - 1 < nst);
        }

        // the tile's factors, behind the waits of its stages
        if constexpr (!REAL && (OUT == kOutF32 || OUT == kOutBF16)) {
            if (threadIdx.x < TM) {
                const int64_t m = m0 + threadIdx.x;
                sm_gamma[parity][threadIdx.x] = (a.per_tensor ? *a.gamma : a.gamma[m < a.M ? m : a.M - 1]) * (1.0f / 128.0f);
            }
        }
        float sc[NI];
#pragma unroll
        for (int s = 0; s < NI; ++s) {
            const int64_t n = n0 + wn * WTN + 32 * s + j;
            if constexpr (REAL) sc[s] = (a.gamma ? *a.gamma : 1.0f) * a.times;
            else sc[s] = OUT == kOutF32 || OUT == kOutBF16 ? a.scale[n < a.N ? n : a.N - 1] : 0.f;
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
        const int64_t mb = mt + __builtin_amdgcn_readfirstlane(wm * WTM), nb = nt + __builtin_amdgcn_readfirstlane(wn * WTN);
        const float* gm = sm_gamma[parity] + wm * WTM + 4 * g2;
        auto store = [&](auto out) {
            I8Store<REAL, decltype(out)::value> st(a, sl, mb, nb, a.M - mb, a.N - nb, j, g2);
            st.template all<MI, NI>([&](int mi, int rq) { return *reinterpret_cast<const v4f*>(gm + 32 * mi + 8 * rq); }, sc, acc);
        };
        if (TWO && second) store(std::integral_constant<int, kOutF32>{});
        else store(std::integral_constant<int, OUT>{});
        if (!more) break;
        parity ^= 1;
    }
}

// ---- slices of K added, then scaled ----------------------------------------------------------------------
// A thread takes four channels of a token (VEC: 16 bytes of every slice, N a multiple of 4), all slices' loads in flight.
template <bool REAL, int OUT, bool VEC>
__global__ __launch_bounds__(256) void fold_i8(TileArgs a, int splits) {
    constexpr int E = VEC ? 4 : 1;
    using Sum = std::conditional_t<REAL, float, int32_t>;
    typedef Sum Sums __attribute__((ext_vector_type(4)));
    const Sum* const part = static_cast<const Sum*>(a.part);
    const int64_t count = a.M * a.N, n = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E;
    if (n >= a.N) return;
    for (int64_t m = blockIdx.y; m < a.M; m += gridDim.y) {
        const int64_t i = m * a.N + n;
        Sum v[E];
        if constexpr (VEC) {
            Sums t = *reinterpret_cast<const Sums*>(part + i);
#pragma unroll 4
            for (int s = 1; s < splits; ++s) t += *reinterpret_cast<const Sums*>(part + s * count + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = t[e];
        } else {
            v[0] = part[i];
            for (int s = 1; s < splits; ++s) v[0] += part[s * count + i];
        }
        if constexpr (OUT == kOutAcc) {
#pragma unroll
            for (int e = 0; e < E; ++e) static_cast<int32_t*>(a.Y)[i + e] = (int32_t)v[e];
        } else {
            float y[E];
            if constexpr (REAL) {
                const float sc = (a.gamma ? *a.gamma : 1.0f) * a.times;
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = v[e] * sc;
            } else {
                const float gm = (a.per_tensor ? *a.gamma : a.gamma[m]) * (1.0f / 128.0f);
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = (float)v[e] * (a.scale[n + e] * gm);
            }
#pragma unroll
            for (int e = 0; e < E; ++e)
                if constexpr (OUT == kOutBF16) static_cast<uint16_t*>(a.Y)[i + e] = (uint16_t)bf16_pair(y[e], 0.f);
                else static_cast<float*>(a.Y)[i + e] = y[e];
        }
    }
}

// ---- up to 32 tokens: the weights' stream ------------------------------------------------------------------
// Bound by reading the weights once.  A workgroup takes TN rows of tiles (16 TN channels) and all of K, or a slice of
// it; its W waves share the tiles of K evenly.  A wave loads S tiles of each row with 16 bytes a lane, which is the
// operand of v_mfma_i32_16x16x64_i8 as it lies, and the codes of MB blocks of 16 tokens beside them (from L2), while it
// multiplies the ones before.  The waves' sums meet in LDS.  A lane has four consecutive channels of one token.
// One token, 28672 x 7168, weights that no cache holds: 35 us = 5.8 TB/s; 16 tokens 45, 32 tokens 53; 8192 x 2048, one token:
// 4.7 us, an empty launch and two trips to memory.
template <int TN, int MB, int S, int W>
__global__ __launch_bounds__(W * 64, W * TN * MB <= 32 ? 4 : 2) void gemm_i8_stream(GemmI8Args a, int out) {
    __shared__ v4i red[W][TN * MB][kWave];
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), l = threadIdx.x % kWave, c = l & 15, g = l >> 4;
    const int K = (int)a.K, TK = (int)i8_tiles_k(K);
    const int64_t rows = tiles_n(a.N);
    const int ns = (int)gridDim.y, from_s = TK * (int)blockIdx.y / ns, in_s = TK * ((int)blockIdx.y + 1) / ns - from_s;
    const int from = from_s + in_s * w / W, to = from_s + in_s * (w + 1) / W;
    uint32_t row[MB];
#pragma unroll
    for (int b = 0; b < MB; ++b) row[b] = (uint32_t)(16 * b + c < (int)a.M ? 16 * b + c : (int)a.M - 1) * (uint32_t)K;
    const bool odd = (K & 63) != 0;  // the last tile's second half is behind K

    // (one item a workgroup but for more channels than a launch takes)
    for (int64_t tile0 = (int64_t)blockIdx.x * TN; tile0 < rows; tile0 += (int64_t)gridDim.x * TN) {
    const uint8_t* wt[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t) wt[t] = a.packed + (tile0 + t < rows ? tile0 + t : rows - 1) * TK * 1024;
    struct Step {
        v4i w[S][TN], q[S][MB];
    } A, B;
    v4i acc[TN][MB];
#pragma unroll
    for (int t = 0; t < TN; ++t)
#pragma unroll
        for (int b = 0; b < MB; ++b) acc[t][b] = v4i{0, 0, 0, 0};
    auto load = [&](Step& x, int at) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int t = at + s < to ? at + s : to - 1;
#pragma unroll
            for (int r = 0; r < TN; ++r)
                x.w[s][r] = __builtin_nontemporal_load(reinterpret_cast<const v4i*>(wt[r] + (uint32_t)t * 1024u) + l);
            const uint32_t k = (uint32_t)t * 64 + (odd && t == TK - 1 ? 16 * (g & 1) : 16 * g);  // (against zeros)
#pragma unroll
            for (int b = 0; b < MB; ++b) x.q[s][b] = *reinterpret_cast<const v4i*>(a.codes + (row[b] + k));
        }
    };
    auto multiply = [&](const Step& x, int at) {
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (at + s < to) {  // uniform
#pragma unroll
                for (int r = 0; r < TN; ++r)
#pragma unroll
                    for (int b = 0; b < MB; ++b)
                        acc[r][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(x.w[s][r], x.q[s][b], acc[r][b], 0, 0, 0);
            }
    };
    if (from < to) {
        int at = from;
        load(A, at);
        for (; at + 2 * S < to; at += 2 * S) {
            load(B, at + S);
            multiply(A, at);
            load(A, at + 2 * S);
            multiply(B, at + S);
        }
        if (at + S < to) {
            load(B, at + S);
            multiply(A, at);
            multiply(B, at + S);
        } else {
            multiply(A, at);
        }
    }
#pragma unroll
    for (int r = 0; r < TN; ++r)
#pragma unroll
        for (int b = 0; b < MB; ++b) red[w][r * MB + b][l] = acc[r][b];
    __syncthreads();
    for (int i = threadIdx.x; i < TN * MB * kWave; i += W * kWave) {
        const int slot = i / kWave, r = slot / MB, m = 16 * (slot % MB) + (i & 15);
        const int64_t n = (tile0 + r) * 16 + 4 * (i % kWave >> 4);
        v4i v = red[0][slot][i % kWave];
#pragma unroll
        for (int k = 1; k < W; ++k) v += red[k][slot][i % kWave];
        if (m >= (int)a.M || n >= a.N) continue;
        const int64_t o = (int64_t)m * a.N + n;
        const int left = a.N - n < 4 ? (int)(a.N - n) : 4;
        if (out == kOutPart || out == kOutAcc) {
            int32_t* y = out == kOutPart ? a.part + (int64_t)blockIdx.y * a.M * a.N + o : static_cast<int32_t*>(a.Y) + o;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < left) y[e] = v[e];
            continue;
        }
        const float gm = (a.per_tensor ? *a.gamma : a.gamma[m]) * (1.0f / 128.0f);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) {
                const float y = (float)v[e] * (a.scale[n + e] * gm);
                if (out == kOutBF16) static_cast<uint16_t*>(a.Y)[o + e] = (uint16_t)bf16_pair(y, 0.f);
                else static_cast<float*>(a.Y)[o + e] = y;
            }
    }
    __syncthreads();
    }
}

// The tiles: 256 x 256 with one workgroup a CU, 128 x 128 and 64 x 128 with two.  What a call costs, in us: rounds of
// workgroups with `per` stages each (`two` us a stage with all of a CU's workgroups, `one` with a single one) and their
// start and stores (`item`), or the operands and the output at the memory's rate; slices of K, their launch and their
// sums.  The constants were fitted by what the choice costs, over 300 shapes of 65 to 8192 tokens, K to 16384, N to
// 28672: 0.6 % slower than the best of 18 variants on average, 22 % at most; over 150 others 0.7 % and 14 %.  They serve 33 to
// 64 tokens too, where the choice is 4.5 % and 51 % slower (36 x 15360 -> 12084, left uncut, 68 us, two slices 45): one rate of
// the memory for any number of workgroups is too low with all CUs at work and too high with few.  Any one tile less costs 1.4
// to 10 % on average; 256 x 256 in slices would gain 0.1 %.
struct I8Tile {
    int tm, tn, wgs;  // wgs: a CU's
    double two, one, item, item_one;
};
constexpr I8Tile kTiles[3] = {{256, 256, 1, 0.679, 0.539, 9.7, 15.4}, {128, 128, 2, 0.485, 0.26, 2.96, 2.75},
                              {64, 128, 2, 0.339, 0.138, 1.41, 1.75}};
constexpr double kCallUs = 2.61, kTrafficPerUs = 3.56e6, kFoldUs = 1.78, kFoldSliceUs = 0.26, kFoldPerByte = 3.86e-7;
constexpr int kMostSlices = 8;
static double fold_us(double outputs, int64_t splits) {
    return splits > 1 ? kFoldUs + (double)splits * (kFoldSliceUs + outputs * 4.0 * kFoldPerByte) : 0.0;
}
static I8Plan i8_plan(int64_t M, int64_t N, int64_t nst, double bytes, double* us = nullptr, int only = -1) {
    const Tuning& t = tuning();
    if (only < 0 && t.i8_tile >= 1 && t.i8_tile <= 3) only = t.i8_tile - 1;
    const int64_t cus = num_cus();
    const double outputs = (double)M * (double)N, floor = bytes / kTrafficPerUs;
    I8Plan best{};
    double least = 1e300;
    for (int k = 0; k < 3; ++k) {
        if (only >= 0 ? only != k : k == 0 && M <= 192) continue;
        const I8Tile& T = kTiles[k];
        const int64_t gm = (M + T.tm - 1) / T.tm, gn = (N + T.tn - 1) / T.tn, tiles = gm * gn;
        const int64_t force = t.i8_splits > 0 ? t.i8_splits : 0;
        for (int64_t n = force ? force : 1; n <= (force ? force : kMostSlices); ++n) {
            const int64_t per = (nst + n - 1) / n, splits = k == 0 ? 1 : (nst + per - 1) / per, items = tiles * splits;
            if (n > 1 && !force && (k == 0 || per < 3 || splits != n || items > 4 * cus)) continue;
            const int64_t slots = T.wgs * cus, full = items / slots, rest = items % slots, stages = k == 0 ? nst : per;
            double cost = (double)full * (T.two * (double)stages + T.item);
            if (rest) cost += rest > cus ? T.two * (double)stages + T.item : T.one * (double)stages + T.item_one;
            cost = kCallUs + (cost > floor ? cost : floor) + fold_us(outputs, splits);
            if (cost < least) {
                least = cost;
                const int64_t up = (items + 7) / 8 * 8;
                best = I8Plan{k, (int)(up < slots ? up : slots), (int)gm, (int)gn, (int)splits, (int)stages};
            }
        }
    }
    if (us) *us = least;
    return best;
}
static I8Plan i8_plan_of(int64_t M, int64_t N, int64_t K, double* us = nullptr) {
    const double m = (double)M, n = (double)N, k = (double)K;
    return i8_plan(M, N, i8_tiles_k(K), (m + n) * k + 2.0 * m * n, us);
}
static I8Plan bf16_plan(int64_t M, int64_t N, int64_t stages, int only = -1) {
    const double m = (double)M, n = (double)N;
    return i8_plan(M, N, stages, (m + n) * 64.0 * (double)stages + 4.0 * m * n, nullptr, only);
}
static I8Plan unsliced(I8Plan p, int stages) {
    const int64_t tiles = (int64_t)p.gm * p.gn, up = (tiles + 7) / 8 * 8;
    if (p.grid > up) p.grid = (int)up;
    p.splits = 1;
    p.per = stages;
    return p;
}
struct StreamPlan {
    int tn, mb, slices;  // rows of tiles a workgroup (0: tiles it is, of i8_plan), blocks of 16 tokens, slices of K
};
// Up to 32 tokens: the stream with the rows of tiles and slices that cost least, or tiles where those do.  us: `call`,
// and `tile` for each tile of K that a wave has, (workgroups / CUs)^power where there are more than CUs; or the weights
// at `rate` MB/us.  Fitted to 126 shapes of 1 to 32 tokens: 2.4 % slower than the best of 20 variants on average, 44 %
// at most; over 126 others 3.7 % and 61 %; the 52 shapes of 17 to 32 tokens among them alone 8.3 % and 61 %, those of 1 to 16
// 1.8 % and 34 %.  From 17 tokens on there are no two rows a workgroup: 26 registers spill in the
// stream's loop (32 x 8384 -> 14656 44 us, four rows 28, one 46), and of 300000 shapes to N = 2 * 10^6 none took them.
struct StreamCost {
    double call, tile, rate, power;
};
constexpr StreamCost kStream[2][3] = {{{4.336, 0.231, 5.265, 1.41}, {4.187, 0.394, 5.77, 1.63}, {3.993, 0.716, 5.32, 1.03}},
                                      {{4.631, 0.055, 2.953, 1.82}, {}, {4.004, 1.05, 3.83, 0.81}}};
static StreamPlan stream_plan(int64_t M, int64_t N, int64_t K) {
    const Tuning& t = tuning();
    StreamPlan p{};
    if (M > 32 || (t.i8_tile >= 1 && t.i8_tile <= 3)) return p;
    const int64_t rows = tiles_n(N), TK = i8_tiles_k(K), cus = num_cus();
    const int mb = M > 16 ? 2 : 1;
    double least = 1e300;
    const int only = t.i8_rows == 1 || t.i8_rows == 4 || (t.i8_rows == 2 && mb == 1) ? t.i8_rows : 0;
    for (int r = 0; r < 3; ++r) {
        if (only ? only != 1 << r : r == 1 && mb == 2) continue;
        const StreamCost& c = kStream[mb - 1][r];
        const int64_t force = t.i8_splits > 0 ? (t.i8_splits < TK ? t.i8_splits : TK) : 0, wgs = (rows + (1 << r) - 1) >> r;
        for (int64_t n = force ? force : 1; n <= (force ? force : 8); n *= 2) {
            if (n > 1 && !force && (wgs * n > 2 * cus || TK < 8 * n)) break;
            const double load = (double)(wgs * n) / (double)cus, tiles = (double)((TK + 8 * n - 1) / (8 * n));
            double cost = c.tile * tiles * (load > 1.0 ? pow(load, c.power) : 1.0);
            const double bytes = (double)N * (double)K * 1e-6 / c.rate;
            cost = c.call + (cost > bytes ? cost : bytes);
            if (n > 1) cost += 1.09 + (double)n * (0.23 + (double)M * (double)N * 4.85e-6);
            if (cost < least) least = cost, p = StreamPlan{1 << r, mb, (int)n};
        }
    }
    double tiles_us;
    if (t.i8_tile != 4 && t.i8_rows == 0 && rows > 8) {
        i8_plan_of(M, N, K, &tiles_us);
        if (tiles_us < least) p.tn = 0;
    }
    return p;
}
static void launch_stream(const GemmI8Args& a, const StreamPlan& p, int out, hipStream_t s) {
    const int64_t wgs = (tiles_n(a.N) + p.tn - 1) / p.tn;
    const dim3 grid((unsigned)(wgs < (1 << 18) ? wgs : (1 << 18)), (unsigned)p.slices);
    auto go = [&](auto tn, auto mb) {
        constexpr int TN = decltype(tn)::value, MB = decltype(mb)::value, S = 8 / TN < 4 ? 8 / TN : 4;
        gemm_i8_stream<TN, MB, S, 8><<<grid, 512, 0, s>>>(a, out);
    };
    auto rows = [&](auto tn) {
        if (p.mb == 1) go(tn, std::integral_constant<int, 1>{});
        else go(tn, std::integral_constant<int, 2>{});
    };
    if (p.tn == 1) rows(std::integral_constant<int, 1>{});
    else if (p.tn == 2) go(std::integral_constant<int, 2>{}, std::integral_constant<int, 1>{});
    else rows(std::integral_constant<int, 4>{});
}

static size_t slices_bytes(int64_t slices, int64_t M, int64_t N) { return slices > 1 ? (size_t)slices * M * N * 4 : 0; }

size_t gemm_i8_part_bytes(int64_t M, int64_t N, int64_t K) {
    if (M == 0) return 0;
    const StreamPlan p = stream_plan(M, N, K);
    return slices_bytes(p.tn ? p.slices : i8_plan_of(M, N, K).splits, M, N);
}
template <bool REAL>
static void launch_fold(const TileArgs& a, int splits, int out, hipStream_t s) {
    const bool vec = a.N % 4 == 0;
    const int64_t per = vec ? 1024 : 256;
    const dim3 grid((unsigned)((a.N + per - 1) / per), (unsigned)(a.M < 32768 ? a.M : 32768));
    auto pick = [&](auto v) {
        constexpr bool VEC = decltype(v)::value;
        if constexpr (!REAL)
            if (out == kOutAcc) return fold_i8<REAL, kOutAcc, VEC>;
        return out == kOutBF16 ? fold_i8<REAL, kOutBF16, VEC> : fold_i8<REAL, kOutF32, VEC>;
    };
    const auto fold = vec ? pick(std::true_type{}) : pick(std::false_type{});
    fold<<<grid, 256, 0, s>>>(a, splits);
}
template <bool REAL>
static hipError_t launch_tiles(const TileArgs& a, I8Plan p, int out, size_t part_bytes, hipStream_t s) {
    if (slices_bytes(p.splits, a.M, a.N) > part_bytes) p = unsliced(p, a.stages);
    const int kind = p.splits > 1 ? kOutPart : out;
    auto pick = [&](auto tm, auto tn) {
        constexpr int TM = decltype(tm)::value, TN = decltype(tn)::value;
        if constexpr (TM < 256)
            if (kind == kOutPart) return gemm_i8_tiles<REAL, TM, TN, 4, kOutPart>;
        if constexpr (!REAL)
            if (kind == kOutAcc) return gemm_i8_tiles<REAL, TM, TN, 4, kOutAcc>;
        return kind == kOutBF16 ? gemm_i8_tiles<REAL, TM, TN, 4, kOutBF16> : gemm_i8_tiles<REAL, TM, TN, 4, kOutF32>;
    };
    using std::integral_constant;
    const auto kernel =
        p.tile == 0   ? pick(integral_constant<int, 256>{}, integral_constant<int, 256>{})
        : p.tile == 1 ? pick(integral_constant<int, 128>{}, integral_constant<int, 128>{})
                      : pick(integral_constant<int, 64>{}, integral_constant<int, 128>{});
    kernel<<<(unsigned)p.grid, 256, 0, s>>>(a, p);
    if (p.splits > 1) launch_fold<REAL>(a, p.splits, out, s);
    return hipGetLastError();
}

hipError_t launch_gemm_i8(const GemmI8Args& a, hipStream_t s) {
    const int out = a.out_acc ? kOutAcc : a.y_bf16 ? kOutBF16 : kOutF32;
    const int64_t TK = i8_tiles_k(a.K);
    TileArgs t{reinterpret_cast<const uint8_t*>(a.codes), a.packed, a.K, 64, TK * 1024, 1024, a.M, a.N, (int)TK, (a.K & 63) != 0,
               a.gamma, a.scale, a.per_tensor, 1.0f, a.Y, a.part};
    if (StreamPlan p = stream_plan(a.M, a.N, a.K); p.tn) {
        if (slices_bytes(p.slices, a.M, a.N) > a.part_bytes) p.slices = 1;
        launch_stream(a, p, p.slices > 1 ? kOutPart : out, s);
        if (p.slices > 1) launch_fold<false>(t, p.slices, out, s);
        return hipGetLastError();
    }
    return launch_tiles<false>(t, i8_plan_of(a.M, a.N, a.K), out, a.part_bytes, s);
}

size_t gemm_bf16_part_bytes(int64_t M, int64_t N, int64_t stages) {
    if (M <= 0 || stages <= 0) return 0;
    const size_t alone = slices_bytes(bf16_plan(M, N, stages).splits, M, N);
    const size_t beside = slices_bytes(bf16_plan(M, N, stages, 2).splits, M, N);
    return alone > beside ? alone : beside;
}
static TileArgs tile_args(const GemmBF16Args& a) {
    return TileArgs{static_cast<const uint8_t*>(a.A), static_cast<const uint8_t*>(a.B), a.a_pitch, a.a_step, 1024, a.N / 16 * 1024,
                    a.M, a.N, a.stages, false, a.factor, nullptr, false, a.times, a.Y, a.part};
}
hipError_t launch_gemm_bf16(const GemmBF16Args& a, hipStream_t s) {
    return launch_tiles<true>(tile_args(a), bf16_plan(a.M, a.N, a.stages), a.y_bf16 ? kOutBF16 : kOutF32, a.part_bytes, s);
}
// One launch for both, in tiles that both take, where together they are at most two rounds of workgroups: 333 x 2048 x
// 2048 (M, N, K of the layer) 31.4 -> 28.5 us, 1000 x 1024 x 1024 25.1 -> 18.3, 64 x 2048 x 2048 24.2 -> 20.7; up to
// four rounds it costs: 333 x 4096 x 4096 64.5 -> 67.0, 256 x 8192 x 4096 91 -> 96.
hipError_t launch_gemm_bf16_two(const GemmBF16Args& a, const GemmBF16Args& a2, hipStream_t s) {
    I8Plan p = bf16_plan(a.M, a.N, a.stages), p2 = bf16_plan(a2.M, a2.N, a2.stages);
    if (p.tile + p2.tile == 3) {  // 128 x 128 and 64 x 128
        p = bf16_plan(a.M, a.N, a.stages, 2);
        p2 = bf16_plan(a2.M, a2.N, a2.stages, 2);
    }
    if (slices_bytes(p.splits, a.M, a.N) > a.part_bytes) p = unsliced(p, a.stages);
    const int64_t slots = (int64_t)num_cus() * kTiles[p.tile].wgs;
    const int64_t items = (int64_t)p.gm * p.gn * p.splits + (int64_t)p2.gm * p2.gn;
    if (p.tile == 0 || p.tile != p2.tile || p2.splits > 1 || a2.y_bf16 || items > 2 * slots) {
        if (const hipError_t e = launch_gemm_bf16(a, s); e != hipSuccess) return e;
        return launch_gemm_bf16(a2, s);
    }
    const TileArgs t = tile_args(a);
    const SecondProduct t2{tile_args(a2), p2};
    const int out = a.y_bf16 ? kOutBF16 : kOutF32, kind = p.splits > 1 ? kOutPart : out;
    auto pick = [&](auto tm) {
        constexpr int TM = decltype(tm)::value;
        return kind == kOutPart   ? gemm_i8_tiles<true, TM, 128, 4, kOutPart, SecondProduct>
               : kind == kOutBF16 ? gemm_i8_tiles<true, TM, 128, 4, kOutBF16, SecondProduct>
                                  : gemm_i8_tiles<true, TM, 128, 4, kOutF32, SecondProduct>;
    };
    const auto kernel = p.tile == 1 ? pick(std::integral_constant<int, 128>{}) : pick(std::integral_constant<int, 64>{});
    kernel<<<(unsigned)(p.grid + p2.grid), 256, 0, s>>>(t, p, t2);
    if (p.splits > 1) launch_fold<true>(t, p.splits, out, s);
    return hipGetLastError();
}

}  // namespace bl
