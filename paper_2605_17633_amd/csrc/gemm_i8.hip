// The block's contractions on 8-bit integers: C = epilogue((A W^T) * w_scales * a_scales + bias), A and W codes with a scale for each row, sums exact in 32 bits.
// Which kernel, and the one for few rows; tiles of more are in gemm_i8.h.
#include "gemm_i8.h"

int ssam_gemm_i8_bias(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_gelu(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_add(int tile, const GemmI8Args &a, hipStream_t st);
int ssam_gemm_i8_scatter(int tile, const GemmI8Args &a, hipStream_t st);

namespace {

constexpr int I8_MOST_LD = 1 << 22, I8_MOST = 0x7fff0000;        // row and column indices and a tile more stay in 32 bits
constexpr int I8_MOST_WORKGROUPS = (1 << 23) - 64;                 // of a launch, which has less than 2^32 threads

// Few rows: 16 columns a workgroup, whose eight waves share K and add up in LDS.  Codes go from memory to the matrix unit's registers, past no barrier: latency and the weight's bytes are all there
// is.  One row (us, launches of a graph, an empty one 2.6): 1280 x 1280 3.2, 3840 x 1280 3.8, 5120 x 1280 4.6, 1280 x 5120 5.3; 16 rows 3.6, 4.2, 5.3, 7.1 (64x64 tiles 5.6, 6.3, 6.4, 10.9).  Two k-steps in flight a wave: four, or
// sixteen waves, ask for more at once than a CU takes in order (up to twice the time at 5120 columns).
template <int MT, int WAVES, int EPI>
__global__ void __launch_bounds__(64 * WAVES)
gemm_i8_few_kernel(GemmI8Args a)
{
    __shared__ i32x4 sums[WAVES > 1 ? (WAVES - 1) * MT * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, quad = lane >> 4;
    const int across = (a.N + 15) / 16, n0 = (int)(blockIdx.x % across) * 16, m0 = (int)(blockIdx.x / across) * MT * 16, steps = (a.K + 63) / 64;
    const unsigned char *w = a.W + (long)min(n0 + l16, a.N - 1) * a.ld.w, *row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) row[i] = a.A + (long)min(m0 + 16 * i + l16, a.M - 1) * a.ld.a;
    i32x4 acc[MT] = {};
    const int first = (int)((long)steps * wave / WAVES), end = (int)((long)steps * (wave + 1) / WAVES);
    auto multiply = [&](int s, auto steps_) {          // k-steps s, s + 1, ...: requested together
        constexpr int U = decltype(steps_)::value;
        i32x4 fw[U], fa[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s + u) * 64 + quad * 16, at = min(k, a.K - 16);
            fw[u] = *reinterpret_cast<const i32x4 *>(w + at);
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[u][i] = *reinterpret_cast<const i32x4 *>(row[i] + at);
            if (k >= a.K) fw[u] = i32x4{ 0, 0, 0, 0 };
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fa[u][i], acc[i], 0, 0, 0);
    };
    int s = first;
    for (; s + 2 <= end; s += 2) multiply(s, std::integral_constant<int, 2>{});
    if (s < end) multiply(s, std::integral_constant<int, 1>{});
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
    auto kern = mt == 1 ? gemm_i8_few_kernel<1, WAVES, EPI> : gemm_i8_few_kernel<2, WAVES, EPI>;
    hipLaunchKernelGGL(kern, dim3(ssam_div_up(a.N, 16) * ssam_div_up(a.M, 16 * mt)), dim3(64 * WAVES), 0, st, a);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}

// A launch of r rounds (one workgroup per CU at a time) takes t0 + r * (t_round + t_slab per slab, t_gelu and t_add behind those epilogues) + (t_mb, and of a scatter-add t_add_mb) per megabyte
// of C.  Of tiles that are cut, the last round is one of their pieces' (`piece`, an index).  Fitted to 850 shapes (M 65 to 33000, N 64 to 5120, K 64 to 5120) with a standard error of 5 %; what is taken
// is 0.6 % on average from the fastest form, 20 % at most (16384 x 4096 x 352, whole rounds of 256x256: 102 us, 192x256 85).
struct I8Tile { int bm, bn; double t0, t_round, t_slab, t_gelu, t_add, t_mb, t_add_mb; };
constexpr I8Tile i8_tiles[GEMM_I8_TILE_COUNT] = {
    { 64, 64, 3.14, 0.661, 0.197, 0.259, 0.259, 0.23, 0.0912 },
    { 96, 64, 1.78, 2.38, 0.269, 0.781, 0.63, 0.165, 0.0568 },
    { 96, 96, 2.43, 2.36, 0.304, 1.16, 0.735, 0.307, 0.0131 },
    { 64, 128, 2.01, 2.54, 0.291, 0.748, 0.559, 0.199, 0.0621 },
    { 128, 128, 2.15, 1.92, 0.411, 1.57, 0.594, 0.132, 0.15 },
    { 128, 192, 2.35, 2.39, 0.513, 2.14, 0.958, 0.173, 0.102 },
    { 192, 128, 2.13, 2.39, 0.516, 2.37, 0.891, 0.11, 0.148 },
    { 256, 128, 1.88, 2.97, 0.665, 3.14, 1.27, 0.0964, 0.143 },
    { 192, 192, 2.32, 2.93, 0.665, 3.02, 1.81, 0.197, 0.0572 },
    { 192, 256, 1.87, 3.93, 0.902, 4.48, 2.51, 0.0808, 0.152 },
    { 256, 192, 1.61, 4.5, 0.836, 4.27, 2.46, 0.0981, 0.125 },
    { 256, 256, 1.49, 5.09, 1.14, 6.16, 3.57, 0.0797, 0.146 } };
struct I8Cut { int tile, subs, piece; };
constexpr I8Cut i8_cuts[GEMM_I8_COUNT - GEMM_I8_TILE_COUNT] = { { 11, 2, 7 }, { 9, 2, 6 }, { 10, 2, 5 } };

// Few rows, 16 or 32 of them and 16 columns a workgroup: t0, and for 512 of K (64 of a wave) and each 16 rows what a workgroup takes alone, and what w / 256 workgroups a CU take.  Fitted
// to 650 shapes (M 1 to 160, N 64 to 5120, K 64 to 5120), standard error 9 %; of all forms what is taken is 1 % on average from the fastest, 30 % at most (78 x 4096 x 576: 5.1 us, 3.9).
struct I8Few { double t0, k, k_rows, w, wk, wk_rows; };
constexpr I8Few i8_few[2] = { { 2.638, 0.243, 0.062, 0.057, 0.166, 0.219 }, { 2.638, 0.305, 0.101, 0.091, 0.112, 0.164 } };

constexpr int I8_FEW = 32;                    // forms: tiles by their index, and 32, 33: few rows, 16 or 32 a workgroup

// Workgroups of a form's launch.
long form_workgroups(int form, int M, int N)
{
    if (form >= I8_FEW) return (long)ssam_div_up(N, 16) * ssam_div_up(M, 16 << (form - I8_FEW));
    const I8Cut *cut = form < GEMM_I8_TILE_COUNT ? nullptr : &i8_cuts[form - GEMM_I8_TILE_COUNT];
    const I8Tile &t = i8_tiles[cut ? cut->tile : form];
    const int tiles = ssam_div_up(M, t.bm) * ssam_div_up(N, t.bn);                          // (M * N < 2^38)
    return cut ? gemm_i8_cut_workgroups(tiles, cut->subs) : ssam_div_up(tiles, 8) * 8;
}

int pick_form(int M, int N, int K, int epilogue)
{
    const int slabs = ssam_div_up(K, GEMM_I8_BK);
    auto round = [&](const I8Tile &t) { return t.t_round + t.t_slab * slabs + (epilogue == SSAM_EPI_BIAS_GELU ? t.t_gelu : epilogue == SSAM_EPI_BIAS_SCATTER_ADD ? t.t_add : 0.0); };
    int best = GEMM_I8_TILE_COUNT - 1;        // 256x256: within the limit of workgroups at any size that is taken
    double best_us = 1e30;
    for (int form = 0; form < GEMM_I8_COUNT; ++form) {
        const I8Cut *cut = form < GEMM_I8_TILE_COUNT ? nullptr : &i8_cuts[form - GEMM_I8_TILE_COUNT];
        const I8Tile &t = i8_tiles[cut ? cut->tile : form];
        const long tiles = (long)ssam_div_up(M, t.bm) * ssam_div_up(N, t.bn);
        if (form_workgroups(form, M, N) > I8_MOST_WORKGROUPS || (cut && (tiles < 256 || gemm_i8_cut_tiles((int)tiles, cut->subs) == 0))) continue;
        const double us = t.t0 + (cut ? tiles / 256 * round(t) + round(i8_tiles[cut->piece]) : (tiles + 255) / 256 * round(t))
                        + (t.t_mb + (epilogue == SSAM_EPI_BIAS_SCATTER_ADD ? t.t_add_mb : 0.0)) * 2e-6 * M * N;
        if (us < best_us) { best_us = us; best = form; }
    }
    for (int i = 0; i < 2; ++i) {
        const int rows = 16 << i;
        const double w = (double)ssam_div_up(N, 16) * ssam_div_up(M, rows) / 256, k = K / 512.0, r = (M < rows ? M : rows) / 16.0;
        const I8Few &t = i8_few[i];
        const double us = t.t0 + k * (t.k + t.k_rows * r) + w * (t.w + k * (t.wk + t.wk_rows * r));
        if (us < best_us && form_workgroups(I8_FEW + i, M, N) <= I8_MOST_WORKGROUPS) { best_us = us; best = I8_FEW + i; }
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
    if (N % 8 != 0 || K % 16 != 0 || K >= 131072 || lda > I8_MOST_LD || ldw > I8_MOST_LD || (long)M * N >= 1L << 38 || M > I8_MOST || N > I8_MOST) return SSAM_EUNSUPPORTED;
    if (mapped && (long)ssam_div_up(M, rows_per_batch) * dst_rows_per_batch > 0x7fffffffL) return SSAM_EUNSUPPORTED;
    const GemmI8Args a = { (const unsigned char *)A, (const unsigned char *)W, a_scales, w_scales, bias, (bf16 *)C, M, N, K, { lda, ldw, ldc },
                           { row_map, rows_per_batch, map_batch_stride, dst_rows_per_batch } };
    if (form < 0) form = pick_form(M, N, K, epilogue);
    else if ((form >= GEMM_I8_COUNT && (form < I8_FEW || form > I8_FEW + 1)) || form_workgroups(form, M, N) > I8_MOST_WORKGROUPS) return SSAM_EUNSUPPORTED;
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
