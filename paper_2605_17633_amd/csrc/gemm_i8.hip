// The block's contractions on 8-bit integers: C = epilogue((A W^T) * w_scales * a_scales + bias), A and W codes with a scale for each row, sums exact in 32 bits.
// Which kernel, and the one for few rows; tiles of more are in gemm_i8.h.
#include "gemm_i8.h"

int ssam_gemm_i8_bias(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_gelu(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_add(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_scatter(int tile, const GemmI8Args &a, hipStream_t st);

namespace {

constexpr int I8_MOST_LD = 1 << 22;

// Few rows: 16 columns a workgroup, whose waves share K and add up in LDS.  Codes go from memory to the matrix unit's registers, past no barrier.
template <int MT, int WAVES, int EPI>
__global__ void __launch_bounds__(64 * WAVES)
gemm_i8_few_kernel(GemmI8Args a)
{
    constexpr int U = 2;                      // k-steps that are requested together
    __shared__ i32x4 sums[WAVES > 1 ? (WAVES - 1) * MT * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, quad = lane >> 4;
    const int n0 = blockIdx.x * 16, m0 = blockIdx.y * MT * 16, steps = (a.K + 63) / 64;
    const unsigned char *w = a.W + (long)min(n0 + l16, a.N - 1) * a.ld.w, *row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) row[i] = a.A + (long)min(m0 + 16 * i + l16, a.M - 1) * a.ld.a;
    i32x4 acc[MT] = {};
    const int first = (int)((long)steps * wave / WAVES), end = (int)((long)steps * (wave + 1) / WAVES);
    for (int s = first; s < end; s += U) {
        i32x4 fw[U], fa[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + u) * 64 + quad * 16, at = min(k, a.K - 16);
            fw[u] = *reinterpret_cast<const i32x4 *>(w + at);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[u][i] = *reinterpret_cast<const i32x4 *>(row[i] + at);
            if (k >= a.K || s + u >= end) fw[u] = i32x4{ 0, 0, 0, 0 };
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fa[u][i], acc[i], 0, 0, 0);
    }
    // wave i % WAVES finishes rows i, which the others send it
    if constexpr (WAVES > 1) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int to = i % WAVES;
            if (wave != to) sums[((wave < to ? wave : wave - 1) * MT + i) * 64 + lane] = acc[i];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        if (wave != i % WAVES) continue;
#pragma unroll
        for (int o = 0; o < WAVES - 1; ++o) acc[i] += sums[(o * MT + i) * 64 + lane];
        const int m = m0 + 16 * i + l16, c = n0 + quad * 4;
        const int to = gemm_i8_row<EPI>(a, m);
        if (to < 0 || c >= a.N) continue;
        uint2 *at = reinterpret_cast<uint2 *>(a.C + (long)to * a.ld.c + c);
        const f32x4 cs = *reinterpret_cast<const f32x4 *>(a.w_scales + c), bias = *reinterpret_cast<const f32x4 *>(a.bias + c);
        const float rs = a.a_scales[m];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = gemm_i8_value<EPI>(acc[i][e], cs[e], rs, bias[e]);
        if constexpr (EPI == SSAM_EPI_BIAS_SCATTER_ADD) {
            const uint2 old = *at;
            v[0] += __uint_as_float(old.x << 16); v[1] += __uint_as_float(old.x & 0xffff0000u);
            v[2] += __uint_as_float(old.y << 16); v[3] += __uint_as_float(old.y & 0xffff0000u);
        }
        *at = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
}

template <int EPI>
int launch_few(int mt, const GemmI8Args &a, hipStream_t st)
{
    constexpr int WAVES = 8;
    auto kern = mt == 1 ? gemm_i8_few_kernel<1, WAVES, EPI> : mt == 2 ? gemm_i8_few_kernel<2, WAVES, EPI> : gemm_i8_few_kernel<4, WAVES, EPI>;
    hipLaunchKernelGGL(kern, dim3(ssam_div_up(a.N, 16), ssam_div_up(a.M, 16 * mt)), dim3(64 * WAVES), 0, st, a);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}

// A launch of r rounds (one workgroup per CU at a time) takes t0 + r * (t_round + t_slab per slab, t_gelu and t_add behind those epilogues) + t_mb per megabyte of C.
struct I8Tile { int bm, bn; double t0, t_round, t_slab, t_gelu, t_add, t_mb; };
constexpr I8Tile i8_tiles[12] = {
    { 64, 64, 3.7, 0, 0.16, 0.262, 0, 0.326 },
    { 96, 64, 0, 4.18, 0.207, 0.375, 0.03, 0.246 },
    { 96, 96, 0, 4.66, 0.251, 0.336, 0.504, 0.223 },
    { 64, 128, 0, 4.27, 0.228, 0.614, 0.075, 0.354 },
    { 128, 128, 1.14, 2.89, 0.382, 1.2, 0, 0.153 },
    { 128, 192, 0.896, 4.09, 0.498, 1.31, 0, 0.205 },
    { 192, 128, 0.478, 3.86, 0.505, 1.71, 0, 0.183 },
    { 256, 128, 0.243, 4.64, 0.623, 2.1, 0, 0.2 },
    { 192, 192, 0.697, 5.38, 0.668, 1.56, 0, 0.22 },
    { 192, 256, 1.07, 4.83, 0.85, 3.16, 0, 0.197 },
    { 256, 192, 0.964, 5, 0.838, 3.1, 0, 0.194 },
    { 256, 256, 1.7, 4.96, 1.09, 4.28, 0, 0.207 } };

constexpr int I8_FEW = 32;                    // forms: tiles by their index, and 32 + 0, 1, 2: few rows, 16, 32 or 64 a workgroup

int pick_form(int M, int N, int K, int epilogue)
{
    if (M <= 64) return I8_FEW + (M <= 16 ? 0 : M <= 32 ? 1 : 2);
    const int slabs = ssam_div_up(K, GEMM_I8_BK);
    int best = 0;
    double best_us = 1e30;
    for (int i = 0; i < 12; ++i) {
        const I8Tile &t = i8_tiles[i];
        const long rounds = ((long)ssam_div_up(M, t.bm) * ssam_div_up(N, t.bn) + 255) / 256;
        const double us = t.t0 + rounds * (t.t_round + t.t_slab * slabs + (epilogue == SSAM_EPI_BIAS_GELU ? t.t_gelu : epilogue == SSAM_EPI_BIAS_SCATTER_ADD ? t.t_add : 0.0))
                        + t.t_mb * 2e-6 * M * N;
        if (us < best_us) { best_us = us; best = i; }
    }
    return best;
}

template <int EPI>
int launch(int form, const GemmI8Args &a, hipStream_t st)
{
    if (form >= I8_FEW) return launch_few<EPI>(1 << (form - I8_FEW), a, st);
    if constexpr (EPI == SSAM_EPI_BIAS) return ssam_gemm_i8_bias(form, a, st);
    else if constexpr (EPI == SSAM_EPI_BIAS_GELU) return ssam_gemm_i8_gelu(form, a, st);
    else if constexpr (EPI == SSAM_EPI_BIAS_SCATTER_ADD) return ssam_gemm_i8_add(form, a, st);
    else return ssam_gemm_i8_scatter(form, a, st);
}

int linear_i8(const void *A, int lda, const float *a_scales, const void *W, int ldw, const float *w_scales, const float *bias, void *C, int ldc, int M, int N, int K, int epilogue,
              const int32_t *row_map, int rows_per_batch, int map_batch_stride, int dst_rows_per_batch, int form, void *stream)
{
    if (!A || !a_scales || !W || !w_scales || !bias || !C || M <= 0 || N <= 0 || K <= 0) return SSAM_EINVAL;
    if (!ssam_aligned16(A) || !ssam_aligned16(W) || !ssam_aligned16(a_scales) || !ssam_aligned16(w_scales) || !ssam_aligned16(bias) || !ssam_aligned16(C)) return SSAM_EINVAL;
    if (lda < K || ldw < K || ldc < N || lda % 16 || ldw % 16 || ldc % 8) return SSAM_EINVAL;
    const bool mapped = epilogue == SSAM_EPI_BIAS_SCATTER_ADD || epilogue == SSAM_EPI_BIAS_SCATTER;
    if (epilogue < 0 || epilogue > SSAM_EPI_BIAS_SCATTER) return SSAM_EINVAL;
    if (mapped && (!row_map || rows_per_batch <= 0 || map_batch_stride < 0 || dst_rows_per_batch <= 0)) return SSAM_EINVAL;
    if (N % 8 != 0 || K % 16 != 0 || K >= 131072 || lda > I8_MOST_LD || ldw > I8_MOST_LD || (long)M * N >= 1L << 40) return SSAM_EUNSUPPORTED;
    if (mapped && (long)ssam_div_up(M, rows_per_batch) * dst_rows_per_batch > 0x7fffffffL) return SSAM_EUNSUPPORTED;
    const GemmI8Args a = { (const unsigned char *)A, (const unsigned char *)W, a_scales, w_scales, bias, (bf16 *)C, M, N, K, { lda, ldw, ldc },
                           { row_map, rows_per_batch, map_batch_stride, dst_rows_per_batch } };
    if (form < 0) form = pick_form(M, N, K, epilogue);
    else if (form >= GEMM_I8_COUNT && (form < I8_FEW || form > I8_FEW + 2 || M > 64)) return SSAM_EUNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    switch (epilogue) {
    case SSAM_EPI_BIAS: return launch<SSAM_EPI_BIAS>(form, a, st);
    case SSAM_EPI_BIAS_GELU: return launch<SSAM_EPI_BIAS_GELU>(form, a, st);
    case SSAM_EPI_BIAS_SCATTER_ADD: return launch<SSAM_EPI_BIAS_SCATTER_ADD>(form, a, st);
    default: return launch<SSAM_EPI_BIAS_SCATTER>(form, a, st);
    }
}

}  // namespace

extern "C" int ssam_linear_i8(const void *A, int lda, const float *a_scales, const void *W, int ldw, const float *w_scales, const float *bias, void *C, int ldc,
                              int M, int N, int K, int epilogue, const int32_t *row_map, int rows_per_batch, int map_batch_stride, int dst_rows_per_batch, void *stream)
{
    return linear_i8(A, lda, a_scales, W, ldw, w_scales, bias, C, ldc, M, N, K, epilogue, row_map, rows_per_batch, map_batch_stride, dst_rows_per_batch, -1, stream);
}

// The same with its form forced, and the form that a call takes: for tests and tuning; not part of the interface.
extern "C" int ssam_linear_i8_as(const void *A, int lda, const float *a_scales, const void *W, int ldw, const float *w_scales, const float *bias, void *C, int ldc, int M, int N, int K, int epilogue,
                                 const int32_t *row_map, int rows_per_batch, int map_batch_stride, int dst_rows_per_batch, int form, void *stream)
{
    return form < 0 ? SSAM_EINVAL : linear_i8(A, lda, a_scales, W, ldw, w_scales, bias, C, ldc, M, N, K, epilogue, row_map, rows_per_batch, map_batch_stride, dst_rows_per_batch, form, stream);
}

extern "C" int ssam_linear_i8_form(int M, int N, int K, int epilogue) { return pick_form(M, N, K, epilogue); }
