// The block's contractions on 8-bit integers: C = epilogue((A W^T) * w_scales * a_scales + bias), A and W codes with a scale for each row, sums exact in 32 bits.
#include "gemm_kernel.h"

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int I8_MOST_LD = 1 << 22;

struct I8Args {
    const unsigned char *A, *W;
    const float *a_scales, *w_scales, *bias;
    bf16 *C;
    int M, N, K;
    GemmLd ld;
    GemmRowMap rm;
};

// Destination row of row m of the product, -1: none.
template <int EPI>
__device__ __forceinline__ long i8_row(const I8Args &a, int m)
{
    if (m >= a.M) return -1;
    if (EPI != SSAM_EPI_BIAS_SCATTER_ADD && EPI != SSAM_EPI_BIAS_SCATTER) return m;
    const int b = m / a.rm.rows_per_batch;
    const int idx = a.rm.map[(long)b * a.rm.map_batch_stride + (m - b * a.rm.rows_per_batch)];
    return (unsigned)idx < (unsigned)a.rm.dst_rows_per_batch ? (long)b * a.rm.dst_rows_per_batch + idx : -1;
}

// Tiles of 64 x 64, 2 x 2 waves of 32 x 32, slabs of 64 of K through LDS.
template <int EPI>
__global__ void __launch_bounds__(256)
gemm_i8_kernel(I8Args a)
{
    constexpr int PITCH = 80;
    __shared__ __attribute__((aligned(16))) unsigned char sa[64 * PITCH], sw[64 * PITCH];
    const int m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, quad = lane >> 4;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const int row = tid >> 2, c = (tid & 3) * 16;
    const unsigned char *ga = a.A + (long)min(m0 + row, a.M - 1) * a.ld.a + c, *gw = a.W + (long)min(n0 + row, a.N - 1) * a.ld.w + c;
    i32x4 acc[2][2] = {};
    for (int k = 0; k < a.K; k += 64) {
        const u32x4 zero = { 0, 0, 0, 0 };
        const u32x4 va = k + c < a.K ? *reinterpret_cast<const u32x4 *>(ga + k) : zero, vw = k + c < a.K ? *reinterpret_cast<const u32x4 *>(gw + k) : zero;
        __syncthreads();
        *reinterpret_cast<u32x4 *>(sa + row * PITCH + c) = va;
        *reinterpret_cast<u32x4 *>(sw + row * PITCH + c) = vw;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4 *>(sw + (wn + 16 * j + l16) * PITCH + quad * 16),
                                                                  *reinterpret_cast<const i32x4 *>(sa + (wm + 16 * i + l16) * PITCH + quad * 16), acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int m = m0 + wm + 16 * i + l16;
        const long to = i8_row<EPI>(a, m);
        if (to < 0) continue;
        const float as = a.a_scales[m];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int n = n0 + wn + 16 * j + quad * 4;
            if (n >= a.N) continue;
            uint2 *at = reinterpret_cast<uint2 *>(a.C + to * a.ld.c + n);
            const f32x4 ws = *reinterpret_cast<const f32x4 *>(a.w_scales + n), bias = *reinterpret_cast<const f32x4 *>(a.bias + n);
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = fmaf((float)acc[i][j][e] * ws[e], as, bias[e]);
                if (EPI == SSAM_EPI_BIAS_GELU) v[e] = gelu_erf(v[e]);
            }
            if (EPI == SSAM_EPI_BIAS_SCATTER_ADD) {
                const uint2 old = *at;
                v[0] += __uint_as_float(old.x << 16); v[1] += __uint_as_float(old.x & 0xffff0000u);
                v[2] += __uint_as_float(old.y << 16); v[3] += __uint_as_float(old.y & 0xffff0000u);
            }
            *at = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
    }
}

}  // namespace

extern "C" int ssam_linear_i8(const void *A, int lda, const float *a_scales, const void *W, int ldw, const float *w_scales, const float *bias, void *C, int ldc,
                              int M, int N, int K, int epilogue, const int32_t *row_map, int rows_per_batch, int map_batch_stride, int dst_rows_per_batch, void *stream)
{
    if (!A || !a_scales || !W || !w_scales || !bias || !C || M <= 0 || N <= 0 || K <= 0) return SSAM_EINVAL;
    if (!ssam_aligned16(A) || !ssam_aligned16(W) || !ssam_aligned16(a_scales) || !ssam_aligned16(w_scales) || !ssam_aligned16(bias) || !ssam_aligned16(C)) return SSAM_EINVAL;
    if (lda < K || ldw < K || ldc < N || lda % 16 || ldw % 16 || ldc % 8) return SSAM_EINVAL;
    const bool mapped = epilogue == SSAM_EPI_BIAS_SCATTER_ADD || epilogue == SSAM_EPI_BIAS_SCATTER;
    if (epilogue < 0 || epilogue > SSAM_EPI_BIAS_SCATTER) return SSAM_EINVAL;
    if (mapped && (!row_map || rows_per_batch <= 0 || map_batch_stride < 0 || dst_rows_per_batch <= 0)) return SSAM_EINVAL;
    if (N % 8 != 0 || K % 16 != 0 || K >= 131072 || lda > I8_MOST_LD || ldw > I8_MOST_LD || (long)M * N >= 1L << 45) return SSAM_EUNSUPPORTED;
    const I8Args a = { (const unsigned char *)A, (const unsigned char *)W, a_scales, w_scales, bias, (bf16 *)C, M, N, K, { lda, ldw, ldc },
                       { row_map, rows_per_batch, map_batch_stride, dst_rows_per_batch } };
    auto kern = epilogue == SSAM_EPI_BIAS ? gemm_i8_kernel<SSAM_EPI_BIAS> : epilogue == SSAM_EPI_BIAS_GELU ? gemm_i8_kernel<SSAM_EPI_BIAS_GELU>
              : epilogue == SSAM_EPI_BIAS_SCATTER_ADD ? gemm_i8_kernel<SSAM_EPI_BIAS_SCATTER_ADD> : gemm_i8_kernel<SSAM_EPI_BIAS_SCATTER>;
    hipLaunchKernelGGL(kern, dim3(ssam_div_up(N, 64), ssam_div_up(M, 64)), dim3(256), 0, (hipStream_t)stream, a);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}
