// The 8-bit contraction's tiles, epilogue SSAM_EPI_BIAS_SCATTER.
#include "gemm_i8.h"

int ssam_gemm_i8_scatter(int tile, const GemmI8Args &a, hipStream_t st) { return gemm_i8_launch<SSAM_EPI_BIAS_SCATTER>(tile, a, st); }
