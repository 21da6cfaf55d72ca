// The contraction of 8-bit integers (gemm_i8.hip) for problems of more than a few rows: gemm_wide.h's schedule on the same bytes.  A slab of K is 128 bytes a row, two k-steps of the
// 16x16x64 instruction, which reads the registers and takes the time (16 clocks) of the bf16 one of 16x16x32: tiles, ring, swizzles and fragments are those of GemmWide.
// What differs: sums are whole numbers, so that halves of K add up exactly in any order; K is any multiple of 16 (a last slab's requests stay inside the row, and the fragments of one operand are
// zeros from K on: whatever the other one holds there adds nothing); the epilogue scales by row and column.
//
// What bounds it.  Long K: 256x256 takes 1.4 to 1.6 us a slab (2.7 POP/s, at which the clock settles near 2 GHz): the matrix pipes 2050 of its 3000 clocks, and LDS as many (192 KB of fragments read
// and 64 KB written by the requests, at 128 bytes a clock); neither is free while the other is not.  The block's K of 768 to 1280 are 6 to 10 slabs, and there a round's ends weigh as much: first slabs
// from memory 2 us, and C, which is twice the bytes of A and W together.  So
//   * results go through LDS and out in whole pieces of rows (64 to 192 bytes by lanes in order): straight from the accumulators 16 lanes write 16 bytes into each of 16 rows;
//   * past the caches: C is as large as the L2s in every round, and pushed A and W out.  32768 x 3840 x 1280 as gemm_wide.h does it 192 us, with both 165 (skipping the stores: 140); one of the two alone 178.  What
//     reads C next does not miss it: fc1, rows in 8 bits, fc2, LayerNorm of 13104 x 1280 x 5120 267 -> 237 us, of 1638 rows 52 -> 49;
//   * tiles that are not a whole round are cut in pieces, half of them in front (192 -> 184 us before the stores were changed).
// Measured (us; int8 library product, no scales nor bias, for comparison): 32768 x 3840 x 1280 160 in a loop, 173 the median of traced launches, the least of which is 165 (217), 13104 x 5120 x 1280 94, + GELU 114 (119), 13104 x 1280 x 5120 87 (99), + scatter-add 91, 4900 x 1280 x 1280 + scatter-add 16.1,
// 4096 x 2304 x 768 12.8.  GELU costs 4.5 us a round of 256x256: its arithmetic, which nothing runs beside.  Not faster: results by whole lines of 128 bytes after an exchange between lanes (8 rows an
// instruction, 30 % slower); two workgroups to a CU, of which one writes while the other multiplies: 128x128 in 128 registers 194 us of the first, 128x256 of four waves 187 (GELU as fast as now): they pull
// twice and one and a half times the bytes of 256x256 from the L2.
#pragma once

#include "gemm_wide.h"

typedef int i32x4 __attribute__((ext_vector_type(4)));

struct GemmI8Args {
    const unsigned char *A, *W;
    const float *a_scales, *w_scales, *bias;
    bf16 *C;
    int M, N, K;
    GemmLd ld;
    GemmRowMap rm;
};

constexpr int GEMM_I8_BK = 2 * GEMM_BK;       // bytes of K in a slab

// Sum, scales and bias of a value of C.
template <int EPI>
__device__ __forceinline__ float gemm_i8_value(int acc, float w_scale, float a_scale, float bias)
{
    const float v = fmaf((float)acc * w_scale, a_scale, bias);
    return EPI == SSAM_EPI_BIAS_GELU ? gelu_erf(v) : v;
}

// Destination row of row m of the product, -1: none.
template <int EPI>
__device__ __forceinline__ int gemm_i8_row(const GemmI8Args &a, int m)
{
    if (m >= a.M) return -1;
    if constexpr (EPI != SSAM_EPI_BIAS_SCATTER_ADD && EPI != SSAM_EPI_BIAS_SCATTER) return m;
    const int b = m / a.rm.rows_per_batch;
    const int idx = a.rm.map[(long)b * a.rm.map_batch_stride + (m - b * a.rm.rows_per_batch)];
    return (unsigned)idx < (unsigned)a.rm.dst_rows_per_batch ? b * a.rm.dst_rows_per_batch + idx : -1;
}

// The workgroup's tile from row m0 and column n0 on.
template <int BM, int BN, int WGK, int EPI>
__device__ __forceinline__ void gemm_i8_tile(const GemmI8Args &a, int m0, int n0, unsigned char *smem)
{
    using G = GemmWide<BM, BN, WGK>;
    constexpr int WGN = G::WGN, MT = G::MT, NT = G::NT, NP = NT / 2, WM = MT * 16, WN = NT * 16, SA = G::SA, SW = G::SW, L = G::L;
    constexpr bool ADD = EPI == SSAM_EPI_BIAS_SCATTER_ADD, EARLY = MT * NT < 24 && !(ADD && WGK == 2 && NT == 3);       // registers for what the epilogue reads before the last slabs
    static_assert(!EARLY || G::EARLY, "and LDS for the row map");
    // WGK == 1: SA slabs of A, then SW of W; 2: slab by slab, A then W
    constexpr int STRIDE_A = WGK == 1 ? G::AB : G::AB + G::WB, STRIDE_W = WGK == 1 ? G::WB : G::AB + G::WB, W0 = WGK == 1 ? SA * G::AB : G::AB;
    unsigned char *as = smem, *ws = smem + W0;
    using std::integral_constant;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wk = wave * WGK >> 3, wt = wave & (8 / WGK - 1), wm = wt / WGN * WM, wn = wt % WGN * WN;
    const int l16 = lane & 15, quad = lane >> 4;
    const int n = (a.K + GEMM_I8_BK - 1) / GEMM_I8_BK, last = (a.K - (n - 1) * GEMM_I8_BK) / 16;      // slabs, and 16-byte chunks of the last one

    // column of C (from the wave's first) of operand row l of its MFMA tile j: a lane then holds 8 consecutive columns of a pair of tiles
    auto perm = [](int j, int l) { return j < 2 * NP ? 32 * (j >> 1) + (l >> 2) * 8 + (j & 1) * 4 + (l & 3) : 16 * j + l; };

    // ---- requests: 1 KB each, A's of a slab, then W's; wave w takes w, w + 8, ...  Rows past the end repeat the last one; nothing of them is stored.
    static_assert(G::QA % 2 == 0, "a wave's requests all have the same swizzle");
    const int chunk = (lane & 7) ^ ((4 * (wave & 1) + (lane >> 4)) & 7);                    // of a row's slab, that this lane asks for
    const uint32_t back = (uint32_t)(chunk - min(chunk, last - 1)) * 16;                    // by so much further in front in the last slab
    uint32_t off[L], dst[L];
    const unsigned char *base[L];
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)smem);
    auto is_a = [&](int i) { return WGK == 1 ? i < G::QA / 8 : i * 8 + wave < G::QA; };
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int f = i * 8 + wave;
        if (is_a(i)) {
            off[i] = (uint32_t)(min(m0 + f * 8 + (lane >> 3), a.M - 1) - m0) * (uint32_t)a.ld.a + chunk * 16;
            base[i] = a.A + (long)m0 * a.ld.a;
            dst[i] = lds0 + f * 1024;
        } else {
            const int w = f - G::QA, row = w * 8 + (lane >> 3), h = row / WN, q = row % WN;
            off[i] = (uint32_t)(min(n0 + h * WN + perm(q >> 4, q & 15), a.N - 1) - n0) * (uint32_t)a.ld.w + chunk * 16;
            base[i] = a.W + (long)n0 * a.ld.w;
            dst[i] = lds0 + W0 + w * 1024;
        }
    }
    const bool all = G::LREST == 0 || wave < G::LREST;              // this wave has an L-th request
    auto request = [&](int i, int sa, int sw) {
        if (G::LREST != 0 && i == L - 1 && !all) return;
        gemm_load_lds16_s(dst[i] + (WGK == 1 && i >= G::QA / 8 ? sw * STRIDE_W : sa * STRIDE_A), off[i], base[i]);
        base[i] += GEMM_I8_BK;
    };
    // in front of the requests [from, to) of slab t
    auto ahead = [&](int t, int from, int to) {
        if (t != n - 1) return;
#pragma unroll
        for (int i = 0; i < L; ++i)
            if (i >= from && i < to) off[i] -= back;
    };
    // waits until the slab before the last `rem` requested ones has landed; MAX: the most that rem can be
    auto wait_slabs = [&](int rem, auto max_) {
        constexpr int MAX = decltype(max_)::value;
        auto out = [&](auto slabs) {                // no more than the requests of `slabs` slabs still out (of W's at most MAX - (SA - SW))
            constexpr int s = decltype(slabs)::value, w = s < MAX - (SA - SW) ? s : MAX - (SA - SW);
            if constexpr (WGK == 1) gemm_wait_vm<G::QA / 8 * s + G::QW / 8 * w>();
            else if (G::LREST != 0 && !all) gemm_wait_vm<(L - 1) * s>();
            else gemm_wait_vm<L * s>();
        };
        if (rem >= MAX) out(integral_constant<int, MAX>{});
        else if (MAX > 2 && rem >= 2) out(integral_constant<int, 2>{});
        else if (MAX > 1 && rem >= 1) out(integral_constant<int, 1>{});
        else gemm_wait_vm<0>();
    };
    constexpr int LA = G::QA / 8, LW = G::QW / 8;   // WGK == 1: requests per wave of A and of W

    // ---- fragments: operand a = 16 columns of C (rows of W), operand b = 16 rows
    const uint32_t fa0 = (wm + l16) * 128 + ((quad ^ ((l16 >> 1) & 7)) << 4), fw0 = (wn + l16) * 128 + ((quad ^ ((l16 >> 1) & 7)) << 4);
    i32x4 fa[2][MT], fw[2][NT], acc[MT][NT] = {};
    // read q of k-step s of a slab into set b, in the order its MFMAs want them
    auto read = [&](int q, int b, int s, int sa, int sw) {
        if (q == 0 || q > NT) {
            const int i = q == 0 ? 0 : q - NT;
            fa[b][i] = *reinterpret_cast<const i32x4 *>(as + sa * STRIDE_A + (fa0 ^ (s * 64)) + i * 2048);
        } else {
            fw[b][q - 1] = *reinterpret_cast<const i32x4 *>(ws + sw * STRIDE_W + (fw0 ^ (s * 64)) + (q - 1) * 2048);
        }
    };
    // of the last slab: what lies past K is zeros in one operand
    auto cut = [&](int b, int s) {
        if (last == 8) return;
        const bool past = 4 * s + quad >= last;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) fw[b][j][e] = past ? 0 : fw[b][j][e];
    };
    constexpr int NM = MT * NT, NR = MT + NT;
    auto mfma = [&](int m, int b) {
        const int i = m / NT, j = m % NT;
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[b][j], fa[b][i], acc[i][j], 0, 0, 0);
    };

    // ---- what the epilogue reads (group wk of two finishes rows i of its MTH, from wk * MTH on): requested before the last slabs, the row map in front of the first one,
    // since a wait for an ordinary load also waits for every request in front of it
    constexpr int MTH = (MT + WGK - 1) / WGK, NB = NP * 2 + NT % 2;          // NB: groups of 4 columns
    constexpr bool MAPPED = ADD || EPI == SSAM_EPI_BIAS_SCATTER;
    const int ncol = n0 + wn + quad * 8, ncol1 = n0 + wn + 32 * NP + quad * 4;      // first column of pair 0, of the odd tile
    if constexpr (MAPPED && EARLY) {
        if (wave * 64 < BM) {
            const int m = min(m0 + wave * 64 + lane, a.M - 1), b = m / a.rm.rows_per_batch;
            gemm_load_lds4(lds0 + (uint32_t)G::ring + wave * 256, a.rm.map + (long)b * a.rm.map_batch_stride + (m - b * a.rm.rows_per_batch));
        }
    }
    int drow[MTH];                                // destination rows, -1: not stored
    float rs[MTH];
    f32x4 bv[NB], cs[NB];
    // Results go to memory through LDS, where lanes that follow each other take 16 bytes that follow each other: slot (row, chunk of 8 columns) = lane + 64 j of GK * 16 rows.  Straight from the
    // accumulators 16 lanes write 16 rows, 16 bytes each.
    constexpr int CH = 2 * NT, GK = NT == 3 ? 2 : 1, J = GK * 16 * CH / 64, PITCH = CH * (ADD ? 32 : 16) + 16;
    static_assert(GK * 16 * CH % 64 == 0 && MTH % GK == 0, "whole requests");
    static_assert(8 * GK * 16 * PITCH <= G::ring, "the ring's LDS");
    static_assert(WGK == 1 || 4 * 2 * MTH * NT * 64 * sizeof(i32x4) <= G::ring, "the halves are added in the ring's LDS");
    unsigned char *const stage = smem + wave * (GK * 16 * PITCH);
    constexpr int AHEAD = !ADD ? 1 : J * MTH <= 16 * GK ? MTH / GK : 16 / J;      // groups of rows whose old values are requested ahead
    uint4 old[ADD ? AHEAD * J : 1];
    auto slot_row = [&](int j) { return (lane + 64 * j) / CH; };
    auto slot_col = [&](int j) { return n0 + wn + (lane + 64 * j) % CH * 8; };
    // destination row of slot j of the group that begins with row k of MTH, from the lanes that hold the rows'
    auto slot_to = [&](int k, int j) {
        const int r = slot_row(j);
        const int one = __shfl(drow[k], r & 15, 64);
        if constexpr (GK == 1) return one;
        const int two = __shfl(drow[k + GK - 1], r & 15, 64);
        return r < 16 ? one : two;
    };
    auto load_old = [&](int g) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int to = slot_to(g * GK, j), col = slot_col(j);
            old[g % AHEAD * J + j] = *reinterpret_cast<const uint4 *>(a.C + (long)max(to, 0) * a.ld.c + (col < a.N ? col : 0));      // a row that is not stored reads row 0 and drops the value
        }
    };
    auto load_epilogue = [&]() {
#pragma unroll
        for (int k = 0; k < MTH; ++k) {
            const int i = wk * MTH + k, row = wm + 16 * i + l16, m = m0 + row;
            if constexpr (MAPPED && EARLY) {
                const int b = min(m, a.M - 1) / a.rm.rows_per_batch, idx = reinterpret_cast<const int32_t *>(smem + G::ring)[row < BM ? row : 0];
                drow[k] = m < a.M && (unsigned)idx < (unsigned)a.rm.dst_rows_per_batch ? b * a.rm.dst_rows_per_batch + idx : -1;
            } else {
                drow[k] = gemm_i8_row<EPI>(a, m);
            }
            if (MTH * WGK != MT && i >= MT) drow[k] = -1;
            rs[k] = a.a_scales[min(m, a.M - 1)];
        }
        if constexpr (ADD) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) load_old(k);
        }
#pragma unroll
        for (int g = 0; g < NB; ++g) {
            int c = g < 2 * NP ? ncol + 32 * (g >> 1) + 4 * (g & 1) : ncol1;
            c = c < a.N ? c : 0;
            bv[g] = *reinterpret_cast<const f32x4 *>(a.bias + c);
            cs[g] = *reinterpret_cast<const f32x4 *>(a.w_scales + c);
        }
    };

    // ---- ring
    int sa = 0, sw = 0;                          // stages of slab t
    if constexpr (WGK == 1) {
        // iteration t of the loop requests W of slab t + SW, then A of slab t + SA; here those of t = -SA .. -1
#pragma unroll
        for (int t = -SA; t < 0; ++t) {
            if (t + SW >= 0 && t + SW < n) {
                ahead(t + SW, LA, L);
#pragma unroll
                for (int i = LA; i < L; ++i) request(i, 0, t + SW);
            }
            if (t + SA < n) {
                ahead(t + SA, 0, LA);
#pragma unroll
                for (int i = 0; i < LA; ++i) request(i, t + SA, 0);
            }
        }
        wait_slabs(n - 1, integral_constant<int, SA - 1>{});
        LDS_BARRIER();
#pragma unroll
        for (int q = 0; q < NR; ++q) read(q, 0, 0, 0, 0);
        auto slab = [&](int t, auto full) {
            constexpr bool FULL = decltype(full)::value;
            const int sa1 = sa + 1 == SA ? 0 : sa + 1, sw1 = sw + 1 == SW ? 0 : sw + 1;
            if constexpr (FULL) {
                ahead(t + SW, LA, L);
                ahead(t + SA, 0, LA);
            } else if (t == n - 1) {
                cut(0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                mfma(m, 0);
#pragma unroll
                for (int q = m * NR / NM; q < (m + 1) * NR / NM; ++q) read(q, 1, 1, sa, sw);
                __builtin_amdgcn_sched_barrier(0);
            }
            // slab t + 1 has landed when no more than the requests behind it are out; every wave has read all of slab t
            wait_slabs(FULL ? SA : n - 2 - t, integral_constant<int, SA - 2>{});
            LDS_BARRIER();
            if constexpr (FULL) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = 0; m < NM; ++m) {
                    mfma(m, 1);
#pragma unroll
                    for (int q = m * NR / NM; q < (m + 1) * NR / NM; ++q) read(q, 0, 0, sa1, sw1);
#pragma unroll
                    for (int q = m * L / NM; q < (m + 1) * L / NM; ++q) request(q < LW ? LA + q : q - LW, sa, sw);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                if (t + SW < n) {
                    ahead(t + SW, LA, L);
#pragma unroll
                    for (int i = LA; i < L; ++i) request(i, sa, sw);
                }
                if (t == n - 1) cut(1, 1);
                if (t + 1 < n)
#pragma unroll
                    for (int q = 0; q < NR; ++q) read(q, 0, 0, sa1, sw1);
#pragma unroll
                for (int m = 0; m < NM; ++m) mfma(m, 1);
            }
            sa = sa1;
            sw = sw1;
        };
        int t = 0;
        for (; t < n - SA; ++t) slab(t, std::true_type{});
        if (EARLY) load_epilogue();
#pragma unroll 1
        for (; t < n; ++t) slab(t, std::false_type{});
    } else {
        constexpr int S = SA;
#pragma unroll
        for (int t = 0; t < S; ++t)
            if (t < n) {
                ahead(t, 0, L);
#pragma unroll
                for (int i = 0; i < L; ++i) request(i, t, t);
            }
        wait_slabs(n - 1, integral_constant<int, S - 1>{});
        LDS_BARRIER();
#pragma unroll
        for (int q = 0; q < NR; ++q) read(q, 0, wk, 0, 0);
        // slab t from set B; its stage, which every wave has read, takes slab t + S
        auto slab = [&](int t, auto set, auto full) {
            constexpr bool FULL = decltype(full)::value;
            constexpr int B = decltype(set)::value;
            const int s1 = sa + 1 == S ? 0 : sa + 1;
            if constexpr (FULL) ahead(t + S, 0, L);
            else if (t == n - 1) cut(B, wk);
            wait_slabs(FULL ? S : n - 2 - t, integral_constant<int, S - 2>{});
            LDS_BARRIER();
            if constexpr (FULL) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int m = 0; m < NM; ++m) {
                    mfma(m, B);
#pragma unroll
                    for (int q = m * NR / NM; q < (m + 1) * NR / NM; ++q) read(q, B ^ 1, wk, s1, s1);
#pragma unroll
                    for (int q = m * L / NM; q < (m + 1) * L / NM; ++q) request(q, sa, sa);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                if (t + 1 < n)
#pragma unroll
                    for (int q = 0; q < NR; ++q) read(q, B ^ 1, wk, s1, s1);
#pragma unroll
                for (int m = 0; m < NM; ++m) mfma(m, B);
            }
            sa = s1;
        };
        int t = 0;
        for (; t < n - S; t += 2) {
            slab(t, integral_constant<int, 0>{}, std::true_type{});
            if (t + 1 >= n - S) break;
            slab(t + 1, integral_constant<int, 1>{}, std::true_type{});
        }
        t = n > S ? n - S : 0;
        if (EARLY) load_epilogue();
#pragma unroll 1
        for (; t < n; ++t) {
            if (t & 1) slab(t, integral_constant<int, 1>{}, std::false_type{});
            else slab(t, integral_constant<int, 0>{}, std::false_type{});
        }
    }
    if (!EARLY) load_epilogue();

    // ---- epilogue: lane (l16, quad) holds row 16*i + l16, columns 8*quad .. + 7 of every pair of tiles
    i32x4 fin[MTH][NT];
    if constexpr (WGK == 2) {
        // the halves of K: either group sends the rows that the other one finishes, through the ring, whose last slab every wave had read at the last barrier
        i32x4 *x = reinterpret_cast<i32x4 *>(smem) + wt * (2 * MTH * NT * 64) + lane;
#pragma unroll
        for (int k = 0; k < MTH; ++k)
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int hi = MTH + k < MT ? MTH + k : MT - 1;
                x[((wk ^ 1) * MTH + k) * NT * 64 + j * 64] = wk ? acc[k][j] : acc[hi][j];
                fin[k][j] = wk ? acc[hi][j] : acc[k][j];
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MTH; ++k)
#pragma unroll
            for (int j = 0; j < NT; ++j) fin[k][j] += x[(wk * MTH + k) * NT * 64 + j * 64];
        LDS_BARRIER();                           // results are staged where other waves' halves lie
    } else {
#pragma unroll
        for (int k = 0; k < MTH; ++k)
#pragma unroll
            for (int j = 0; j < NT; ++j) fin[k][j] = acc[k][j];
    }
#pragma unroll
    for (int g = 0; g < MTH / GK; ++g) {
#pragma unroll
        for (int i = 0; i < GK; ++i) {
            const int k = g * GK + i;
            unsigned char *const at = stage + (16 * i + l16) * PITCH;
            auto value = [&](int j, int e) { return gemm_i8_value<EPI>(fin[k][j][e], cs[j][e], rs[k], bv[j][e]); };
            auto packed = [&](int j) { return make_uint2(pack_bf16x2(value(j, 0), value(j, 1)), pack_bf16x2(value(j, 2), value(j, 3))); };
            // of a pair of tiles the first has columns 0 to 3 and the second 4 to 7 of chunk 4 * (pair) + quad; of an odd one two quads share a chunk
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const int four = j < 2 * NP ? 2 * (4 * (j / 2) + quad) + j % 2 : 8 * NP + quad;
                if constexpr (ADD) *reinterpret_cast<f32x4 *>(at + 16 * four) = f32x4{ value(j, 0), value(j, 1), value(j, 2), value(j, 3) };
                else if (j >= 2 * NP) *reinterpret_cast<uint2 *>(at + 8 * four) = packed(j);
                else if (j % 2 == 0) {
                    const uint2 lo = packed(j), hi = packed(j + 1 < NT ? j + 1 : j);
                    *reinterpret_cast<uint4 *>(at + 8 * four) = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
            }
        }
        wave_lds_fence();
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int to = slot_to(g * GK, j), col = slot_col(j);
            const unsigned char *const from = stage + slot_row(j) * PITCH + (lane + 64 * j) % CH * (ADD ? 32 : 16);
            uint4 out;
            if constexpr (ADD) {
                float v[8], o[8];
                unpack_bf16x8(old[g % AHEAD * J + j], o);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = reinterpret_cast<const float *>(from)[e] + o[e];
                out = pack_bf16x8(v);
            } else {
                out = *reinterpret_cast<const uint4 *>(from);
            }
            // (past the caches: what was there stays)
            if (to >= 0 && col < a.N) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, out), reinterpret_cast<u32x4 *>(a.C + (long)to * a.ld.c + col));      // N % 8 == 0
        }
        wave_lds_fence();
        if constexpr (ADD) if (g + AHEAD < MTH / GK) load_old(g + AHEAD);
    }
}

template <int BM, int BN, int WGK, int EPI>
__global__ void __launch_bounds__(512, 1)
gemm_i8_wide_kernel(GemmI8Args a, GemmTileRange tr)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int per_xcd = (tr.tile_count + 7) / 8, tl = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (tl >= tr.tile_count) return;
    int m0, n0;
    gemm_tile_origin(tr, tl, 0, 1, 1, BM, BN, m0, n0);
    gemm_i8_tile<BM, BN, WGK, EPI>(a, m0, n0, smem);
}

// Several rounds of workgroups, of which the last would be a part: tiles from tr.tile_begin on are cut into SUB_M x SUB_N pieces.  Half of the pieces come first and half last: every CU has
// as much to do, and CUs that began with a piece are out of step with the others, so that what some write at the end of a tile goes to memory under the products of the rest.
template <int BM, int BN, int SUB_M, int SUB_N, int EPI>
__global__ void __launch_bounds__(512, 1)
gemm_i8_wide_cut_kernel(GemmI8Args a, GemmTileRange tr)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    constexpr int SUBS = SUB_M * SUB_N;
    const int xcd = blockIdx.x & 7, i = blockIdx.x >> 3;
    const int whole = tr.tile_begin, pieces = (tr.tile_count - whole) * SUBS;
    auto share = [](int n, int x) { return (int)((long)n * x / 8); };                     // of n tiles, XCD x takes [share(n, x), share(n, x + 1))
    const int w0 = share(whole, xcd), ws = share(whole, xcd + 1) - w0, p0 = share(pieces, xcd), ps = share(pieces, xcd + 1) - p0, first = ps / 2;
    int m0, n0;
    if (i >= first && i < first + ws) {
        gemm_tile_origin(tr, w0 + i - first, 0, 1, 1, BM, BN, m0, n0);
        gemm_i8_tile<BM, BN, 1, EPI>(a, m0, n0, smem);
        return;
    }
    const int p = i < first ? i : i - ws;
    if (p >= ps) return;
    gemm_tile_origin(tr, whole + (p0 + p) / SUBS, (p0 + p) % SUBS, SUB_M, SUB_N, BM / SUB_M, BN / SUB_N, m0, n0);
    if (m0 >= a.M || n0 >= a.N) return;
    gemm_i8_tile<BM / SUB_M, BN / SUB_N, 1, EPI>(a, m0, n0, smem);
}

template <class Kernel>
int gemm_i8_launch_kernel(Kernel kern, int workgroups, size_t lds, const GemmI8Args &a, const GemmTileRange &tr, hipStream_t st)
{
    // more than 64 KiB of LDS per workgroup needs the per-kernel opt-in (idempotent, host-side only)
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return SSAM_EHIP;
    hipLaunchKernelGGL(kern, dim3(workgroups), dim3(512), lds, st, a, tr);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}

template <int BM, int BN, int WGK, int EPI>
int gemm_i8_launch_tile(const GemmI8Args &a, hipStream_t st)
{
    GemmTileRange tr = { ssam_div_up(a.M, BM), ssam_div_up(a.N, BN), 0, 0 };
    tr.tile_count = tr.tiles_m * tr.tiles_n;
    return gemm_i8_launch_kernel(gemm_i8_wide_kernel<BM, BN, WGK, EPI>, ssam_div_up(tr.tile_count, 8) * 8, GemmWide<BM, BN, WGK>::lds_bytes, a, tr, st);
}

// Tiles of so many that are cut: those past whole rounds of 256, unless their pieces are more than a round.
inline int gemm_i8_cut_tiles(int tiles, int subs)
{
    const int rem = tiles % 256;
    return rem * subs <= 256 ? rem : 0;
}

// Workgroups of a launch of so many tiles: on every XCD its share of the whole ones and of the pieces.
inline int gemm_i8_cut_workgroups(int tiles, int subs)
{
    const int cut = gemm_i8_cut_tiles(tiles, subs);
    return 8 * (ssam_div_up(tiles - cut, 8) + ssam_div_up((long)cut * subs, 8));
}

template <int BM, int BN, int SUB_M, int SUB_N, int EPI>
int gemm_i8_launch_cut(const GemmI8Args &a, hipStream_t st)
{
    constexpr size_t lds0 = GemmWide<BM, BN, 1>::lds_bytes, lds1 = GemmWide<BM / SUB_M, BN / SUB_N, 1>::lds_bytes;
    GemmTileRange tr = { ssam_div_up(a.M, BM), ssam_div_up(a.N, BN), 0, 0 };
    tr.tile_count = tr.tiles_m * tr.tiles_n;
    tr.tile_begin = tr.tile_count - gemm_i8_cut_tiles(tr.tile_count, SUB_M * SUB_N);
    return gemm_i8_launch_kernel(gemm_i8_wide_cut_kernel<BM, BN, SUB_M, SUB_N, EPI>, gemm_i8_cut_workgroups(tr.tile_count, SUB_M * SUB_N), lds0 > lds1 ? lds0 : lds1, a, tr, st);
}

// Tiles, in the order of their index in the time model (gemm_i8.hip).
#define GEMM_I8_TILES(X)                                                                                       \
    X(0, 64, 64, 2) X(1, 96, 64, 2) X(2, 96, 96, 2) X(3, 64, 128, 2) X(4, 128, 128, 1) X(5, 128, 192, 1)         \
    X(6, 192, 128, 1) X(7, 256, 128, 1) X(8, 192, 192, 1) X(9, 192, 256, 1) X(10, 256, 192, 1) X(11, 256, 256, 1)
#define GEMM_I8_CUT_TILES(X) X(12, 256, 256, 1, 2) X(13, 192, 256, 1, 2) X(14, 256, 192, 2, 1)
constexpr int GEMM_I8_TILE_COUNT = 12, GEMM_I8_COUNT = 15;

template <int EPI>
int gemm_i8_launch(int tile, const GemmI8Args &a, hipStream_t st)
{
    switch (tile) {
#define X(id, bm, bn, wgk) case id: return gemm_i8_launch_tile<bm, bn, wgk, EPI>(a, st);
    GEMM_I8_TILES(X)
#undef X
#define X(id, bm, bn, sm, sn) case id: return gemm_i8_launch_cut<bm, bn, sm, sn, EPI>(a, st);
    GEMM_I8_CUT_TILES(X)
#undef X
    default: return SSAM_EINVAL;
    }
}
