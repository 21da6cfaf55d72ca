// The 8-bit contraction's tiles, epilogue SSAM_EPI_BIAS_GELU.
#include "gemm_i8.h"

int ssam_gemm_i8_gelu(int tile, const GemmI8Args &a, hipStream_t st) { return gemm_i8_launch<SSAM_EPI_BIAS_GELU>(tile, a, st); }
