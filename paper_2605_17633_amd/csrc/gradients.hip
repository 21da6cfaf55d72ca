// What a training step of the block needs beside attention's gradient: the gradient of the LayerNorm of gathered rows, and
// activations that are kept in 8 bits between the forward and the backward pass, with the GELU that reads them.
// All of it is bound by HBM: one pass over the data, 16 bytes of bf16 per lane and request.
#include "rows8.h"

namespace {

// ---------------------------------------------------------------- LayerNorm + gather, backward
// y = gamma * h + beta with h = (x - mean) * rstd.  With g = dy * gamma, over the features of a row:
//   dx = rstd * (g - mean(g) - h * mean(g * h)),   dgamma = sum over rows of dy * h,   dbeta = sum over rows of dy.
// A row's statistics are taken again from x, which the gradient has to read anyway: nothing is kept by the forward call.
// One wave per row, the row in registers; waves walk the rows and keep their share of dgamma and dbeta in registers too.  The four waves
// of a workgroup add theirs up in LDS, a second launch adds the workgroups' up, both in a fixed order: no atomics, same bits every time.
// Bound by HBM: 32768 rows of 1280 in window order, added to dx (336 MB): 66 us, 5.0 TB/s, and 5 for the weights' sums; 313 kept rows of 768: 5.6 + 3.4 us, 22 with the host's part of the call.
constexpr int LNB_WAVES = 4;

template <int MAXC, bool ACCUMULATE, bool WEIGHTS>
__global__ void __launch_bounds__(256)
ln_gather_backward_kernel(const uint4 *__restrict__ x, const int32_t *__restrict__ idx, int idx_batch_stride,
                          const float *__restrict__ gamma, float eps, const uint4 *__restrict__ dy, uint4 *dx,
                          float *__restrict__ parts, int B, int Nin, int Nout, int chunks)
{
    __shared__ float4 lds[WEIGHTS ? LNB_WAVES * 64 * 2 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rows = B * Nout, stride = (int)gridDim.x * LNB_WAVES;
    const float over_D = 1.f / (float)(chunks * 8);
    int at[MAXC];                                // a chunk past the row re-reads its last one and is masked in the arithmetic
    bool in[MAXC];
    float gm[MAXC][8], sg[MAXC][8], sb[MAXC][8];
#pragma unroll
    for (int i = 0; i < MAXC; ++i) {
        in[i] = lane + 64 * i < chunks;
        at[i] = min(lane + 64 * i, chunks - 1);
        const float4 *g4 = reinterpret_cast<const float4 *>(gamma) + 2 * at[i];
        const float4 lo = g4[0], hi = g4[1];
        const float v[8] = { lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w };
#pragma unroll
        for (int e = 0; e < 8; ++e) { gm[i][e] = in[i] ? v[e] : 0.f; sg[i][e] = sb[i][e] = 0.f; }
    }
    auto source = [&](int row) -> long {         // row of x and dx, -1: none
        if ((unsigned)row >= (unsigned)rows) return -1;
        const int b = row / Nout, p = row - b * Nout;
        const int src = idx[(long)b * idx_batch_stride + p];
        return src < 0 || src >= Nin ? -1 : (long)b * Nin + src;
    };
    int row = (int)blockIdx.x * LNB_WAVES + wave;
    long src = source(row);
    for (; row < rows; row += stride) {          // (rows + stride stays below 2^31)
        const long here = src;
        uint4 rx[MAXC], ry[MAXC], ro[MAXC];
        if (here >= 0) {
            const uint4 *xr = x + here * chunks, *yr = dy + (long)row * chunks;
#pragma unroll
            for (int i = 0; i < MAXC; ++i) { rx[i] = xr[at[i]]; ry[i] = yr[at[i]]; }
            if constexpr (ACCUMULATE)
#pragma unroll
                for (int i = 0; i < MAXC; ++i) ro[i] = dx[here * chunks + at[i]];
        }
        src = source(row + stride);              // one row ahead: its own round trip is hidden behind this row's
        if (here < 0) continue;
        float v[MAXC][8], d[MAXC][8];
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            unpack_bf16x8(rx[i], v[i]);
            unpack_bf16x8(ry[i], d[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s += in[i] ? v[i][e] : 0.f;
        }
        const float mean = wave_sum(s) * over_D;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[i][e] -= mean; q += in[i] ? v[i][e] * v[i][e] : 0.f; }
        const float rstd = rsqrtf(wave_sum(q) * over_D + eps);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] *= rstd;
                if constexpr (WEIGHTS) {          // of lanes past the row these are never stored
                    sg[i][e] = fmaf(d[i][e], v[i][e], sg[i][e]);
                    sb[i][e] += d[i][e];
                }
                d[i][e] *= gm[i][e];
                s1 += in[i] ? d[i][e] : 0.f;
                s2 += in[i] ? d[i][e] * v[i][e] : 0.f;
            }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) { s1 += __shfl_xor(s1, o, 64); s2 += __shfl_xor(s2, o, 64); }
        s1 *= over_D;
        s2 *= over_D;
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            if (!in[i]) continue;
            float o[8], old[8];
            if constexpr (ACCUMULATE) unpack_bf16x8(ro[i], old);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                o[e] = rstd * (d[i][e] - s1 - v[i][e] * s2);
                if constexpr (ACCUMULATE) o[e] += old[e];
            }
            dx[here * chunks + lane + 64 * i] = pack_bf16x8(o);
        }
    }
    if constexpr (WEIGHTS) {
        // the waves' sums of 8 columns at a time, [wave][which half][lane]: every lane then adds up one float4 of four waves
        float *mine = parts + (long)blockIdx.x * 2 * chunks * 8;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const float *f = w ? sb[i] : sg[i];
                __syncthreads();
                lds[(wave * 2 + 0) * 64 + lane] = make_float4(f[0], f[1], f[2], f[3]);
                lds[(wave * 2 + 1) * 64 + lane] = make_float4(f[4], f[5], f[6], f[7]);
                __syncthreads();
                if (wave < 2 && in[i]) {
                    float4 a = lds[wave * 64 + lane];
#pragma unroll
                    for (int o = 1; o < LNB_WAVES; ++o) {
                        const float4 t = lds[(o * 2 + wave) * 64 + lane];
                        a.x += t.x; a.y += t.y; a.z += t.z; a.w += t.w;
                    }
                    reinterpret_cast<float4 *>(mine + (long)w * chunks * 8)[2 * (lane + 64 * i) + wave] = a;
                }
            }
    }
}

// [n][2 D] -> the column sums: dgamma in the first D, dbeta in the rest.  A workgroup adds up 32 columns: eight lanes with 16 bytes each, 32 slices of the rows.
__global__ void __launch_bounds__(256)
ln_weight_sums_kernel(const float4 *__restrict__ parts, int n, int D, float *__restrict__ dgamma, float *__restrict__ dbeta)
{
    __shared__ float4 lds[256];
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3, quads = 2 * D / 4;
    const int col = blockIdx.x * 8 + c;
    const bool in = col < quads;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int r = slice; r < n; r += 32) {
        const float4 t = parts[(long)r * quads + min(col, quads - 1)];
        a.x += t.x; a.y += t.y; a.z += t.z; a.w += t.w;
    }
    a = sum_of_shares(a, lds);
    if (slice == 0 && in) *reinterpret_cast<float4 *>(4 * col < D ? dgamma + 4 * col : dbeta + 4 * col - D) = a;
}

// Workgroups of the first launch, and rows of sums that it leaves: two waves to a SIMD of 256 CUs, which keep enough requests in flight.  (Rows above 1536, added, with the weights'
// gradients take 269 registers, one wave to a SIMD, and run in two rounds: 32768 rows of 2048 at 4.4 TB/s, 121 us.  Held to 256 registers they spill 13 and take 140.)
inline int ln_backward_workgroups(long rows) { return (int)(rows < 4L * 512 ? (rows + 3) / 4 : 512); }

template <int MAXC, bool ACCUMULATE, bool WEIGHTS>
int launch_ln_backward(const void *x, const int32_t *idx, int idx_batch_stride, const float *gamma, float eps, const void *dy, void *dx,
                       float *dgamma, float *dbeta, int B, int Nin, int Nout, int D, float *parts, hipStream_t st)
{
    const int n = ln_backward_workgroups((long)B * Nout);
    hipLaunchKernelGGL((ln_gather_backward_kernel<MAXC, ACCUMULATE, WEIGHTS>), dim3(n), dim3(256), 0, st, (const uint4 *)x, idx, idx_batch_stride, gamma, eps,
                       (const uint4 *)dy, (uint4 *)dx, parts, B, Nin, Nout, D / 8);
    SSAM_CHECK_LAUNCH();
    if (WEIGHTS) {
        hipLaunchKernelGGL(ln_weight_sums_kernel, dim3(ssam_div_up(2 * D, 32)), dim3(256), 0, st, (const float4 *)parts, n, D, dgamma, dbeta);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int MAXC>
int launch_ln_backward(bool accumulate, const void *x, const int32_t *idx, int idx_batch_stride, const float *gamma, float eps, const void *dy, void *dx,
                       float *dgamma, float *dbeta, int B, int Nin, int Nout, int D, float *parts, hipStream_t st)
{
    auto go = accumulate ? (dgamma ? launch_ln_backward<MAXC, true, true> : launch_ln_backward<MAXC, true, false>)
                         : (dgamma ? launch_ln_backward<MAXC, false, true> : launch_ln_backward<MAXC, false, false>);
    return go(x, idx, idx_batch_stride, gamma, eps, dy, dx, dgamma, dbeta, B, Nin, Nout, D, parts, st);
}

// ---------------------------------------------------------------- 8 bits
// 64 columns of a row share a scale, their largest magnitude / 127; a value is held as the nearest whole multiple of it (ties to even), off by
// at most 1/254 of that magnitude.  Eight lanes with eight values each hold a block.  Held in fp32, the scale costs 1/16 byte a value.
//   all zero: codes 0.  Scales below 2^-126 (subnormal) become 2^-126: such values are off by 2^-127 at most.
//   infinity or NaN in a block: its scale is NaN, and so is all that comes back of it.  A multiple of an infinite scale would be NaN too (0 * inf),
//   and a clamped infinity would hide what went wrong.
constexpr int CKPT_COLS = 64;

// slot -> row and chunk: division by the slots of a row (8 a block), exact below 2^31
struct FastDiv {
    uint32_t d, m;
    int shift;
    explicit FastDiv(uint32_t d_) : d(d_), shift(0)
    {
        while ((1ull << shift) < d) ++shift;
        m = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> shift; }
};

struct Quantised { uint2 codes; float scale; };
// v: this lane's eight values of a block (zeros past the row); all eight lanes of the block call it
__device__ __forceinline__ Quantised quantise_block(const uint4 &v)
{
    uint32_t top = top_of_bf16x8(v);
    top = max(top >> 16, top & 0xffffu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    Quantised r = { make_uint2(0, 0), __uint_as_float(0x7fc00000u) };
    if (top >= 0x7f80u) return r;
    const RowScale s = row_scale(bf16_bits_to_float(top));
    r.scale = s.scale;
    float f[8];
    unpack_bf16x8(v, f);
    r.codes = codes_of(f, s.inv);
    return r;
}

__device__ __forceinline__ void restore_block(const uint2 &codes, float scale, float *f)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)(int8_t)((e < 4 ? codes.x : codes.y) >> (8 * (e & 3))) * scale;
}

// Phi(t) and t Phi(t) = gelu(t) with the approximation of gelu_erf, and the derivative Phi(t) + t exp(-t^2 / 2) / sqrt(2 pi)
__device__ __forceinline__ void gelu_slope(float t, float &gelu, float &slope)
{
    const float a = fabsf(t);
    const float u = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752440f, a, 1.0f));
    const float poly = half_erfc_poly(u);
    const float s = a * 0.84932180028801904272f;               // sqrt(log2(e) / 2)
    const float e = __builtin_amdgcn_exp2f(-s * s);
    const float tail = u * poly * e;                            // 1 - Phi(|t|)
    gelu = fmaf(-a, tail, fmaxf(t, 0.0f));
    slope = fmaf(t * 0.39894228040143267794f, e, t < 0.f ? tail : 1.f - tail);
}

// Bound by HBM: 32768 x 1280 stored in 21 us and restored in 20 (128 MB each, 6.1 and 6.4 TB/s: the codes are still in the cache); GELU of 13104 x 5120 64 to 72 us forward and 90 backward,
// 150 both (814 MB together, 5.4 TB/s).  Small ones cost what their launches do, 3 to 4 us, and twice that on the host.
enum CkptOp { CKPT_STORE, CKPT_RESTORE, CKPT_GELU, CKPT_GELU_BACKWARD };

// A thread has the slots i and i + half of the launch: both are requested before the first is used, or anything stored (out may be in).
template <CkptOp OP>
__global__ void __launch_bounds__(256)
checkpoint_kernel(const uint4 *in, uint4 *out, uint2 *codes, float *scales, uint4 *again,
                  uint32_t slots, uint32_t half, int chunks, FastDiv per_row)
{
    constexpr bool READS = OP == CKPT_RESTORE || OP == CKPT_GELU_BACKWARD;      // codes and scales are inputs
    const uint32_t blocks = per_row.d / 8;
    uint32_t row[2], chunk[2];
    bool ok[2];
    uint4 v[2];
    uint2 c[2];
    float s[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t i = blockIdx.x * 256u + threadIdx.x + j * half;
        row[j] = per_row.div(i);
        chunk[j] = i - row[j] * per_row.d;
        ok[j] = i < slots && chunk[j] < (uint32_t)chunks;
        v[j] = make_uint4(0, 0, 0, 0);
        if (ok[j]) {
            const size_t at = (size_t)row[j] * chunks + chunk[j];
            if constexpr (OP != CKPT_RESTORE) v[j] = in[at];
            if constexpr (READS) { c[j] = codes[at]; s[j] = scales[(size_t)row[j] * blocks + chunk[j] / 8]; }
        }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const size_t at = (size_t)row[j] * chunks + chunk[j];
        if constexpr (!READS) {
            const Quantised q = quantise_block(v[j]);               // whole blocks of lanes: slots are counted in them
            if (ok[j]) {
                codes[at] = q.codes;
                if (chunk[j] % 8 == 0) scales[(size_t)row[j] * blocks + chunk[j] / 8] = q.scale;
                if constexpr (OP == CKPT_GELU) {
                    float f[8];
                    unpack_bf16x8(v[j], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = gelu_erf(f[e]);
                    out[at] = pack_bf16x8(f);
                }
            }
        } else if (ok[j]) {
            float t[8];
            restore_block(c[j], s[j], t);
            if constexpr (OP == CKPT_RESTORE) {
                out[at] = pack_bf16x8(t);
            } else {
                float d[8];
                unpack_bf16x8(v[j], d);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float slope;
                    gelu_slope(t[e], t[e], slope);
                    d[e] *= slope;
                }
                out[at] = pack_bf16x8(d);
                if (again) again[at] = pack_bf16x8(t);
            }
        }
    }
}

template <CkptOp OP>
int launch_checkpoint(const void *in, void *out, void *codes, float *scales, void *again, long rows, int D, hipStream_t st)
{
    const int chunks = D / 8, blocks = ssam_div_up(D, CKPT_COLS);
    const FastDiv per_row((uint32_t)blocks * 8);
    const long some = (1L << 30) / (blocks * 8);                   // rows of a launch: 2^30 slots at most
    for (long r = 0; r < rows; r += some) {
        const long n = rows - r < some ? rows - r : some;
        const uint32_t slots = (uint32_t)(n * blocks * 8), half = (slots / 2 + 255) / 256 * 256;
        const size_t at = (size_t)r * chunks;
        hipLaunchKernelGGL((checkpoint_kernel<OP>), dim3(half / 256), dim3(256), 0, st, in ? (const uint4 *)in + at : nullptr, out ? (uint4 *)out + at : nullptr,
                           (uint2 *)codes + at, scales + (size_t)r * blocks, again ? (uint4 *)again + at : nullptr, slots, half, chunks, per_row);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

int check_checkpoint(const void *codes, const float *scales, long rows, int D)
{
    if (!codes || !scales || rows <= 0 || D <= 0 || D % 8 != 0 || !ssam_aligned16(codes) || !ssam_aligned16(scales)) return SSAM_EINVAL;
    return D > 1 << 24 ? SSAM_EUNSUPPORTED : SSAM_OK;
}

}  // namespace

extern "C" size_t ssam_ln_gather_backward_workspace_bytes(int B, int Nout, int D)
{
    if (B <= 0 || Nout <= 0 || D <= 0) return 0;
    return (size_t)ln_backward_workgroups((long)B * Nout) * 2 * D * sizeof(float);
}

extern "C" int ssam_ln_gather_backward(const void *x, const int32_t *idx, int idx_batch_stride, const float *gamma, float eps, const void *dy,
                                       void *dx, int accumulate, float *dgamma, float *dbeta, int B, int Nin, int Nout, int D,
                                       void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x || !idx || !gamma || !dy || !dx || (!dgamma) != (!dbeta) || B <= 0 || Nin <= 0 || Nout <= 0 || D <= 0 || D % 8 != 0) return SSAM_EINVAL;
    if (idx_batch_stride != 0 && idx_batch_stride < Nout) return SSAM_EINVAL;
    if (!ssam_aligned16(x) || !ssam_aligned16(gamma) || !ssam_aligned16(dy) || !ssam_aligned16(dx)) return SSAM_EINVAL;
    if (D > 2048 || (long)B * Nout > 0x7fff0000L) return SSAM_EUNSUPPORTED;
    if (dgamma) {
        if (!workspace || !ssam_aligned16(workspace) || !ssam_aligned16(dgamma) || !ssam_aligned16(dbeta)) return SSAM_EINVAL;
        if (workspace_bytes < ssam_ln_gather_backward_workspace_bytes(B, Nout, D)) return SSAM_EWORKSPACE;
    }
    const int maxc = ssam_div_up(D / 8, 64);
    auto go = maxc == 1 ? launch_ln_backward<1> : maxc == 2 ? launch_ln_backward<2> : maxc == 3 ? launch_ln_backward<3> : launch_ln_backward<4>;
    return go(accumulate != 0, x, idx, idx_batch_stride, gamma, eps, dy, dx, dgamma, dbeta, B, Nin, Nout, D, (float *)workspace, (hipStream_t)stream);
}

extern "C" int ssam_checkpoint_store(const void *x, void *codes, float *scales, long rows, int D, void *stream)
{
    if (!x || !ssam_aligned16(x)) return SSAM_EINVAL;
    if (int rc = check_checkpoint(codes, scales, rows, D); rc != SSAM_OK) return rc;
    return launch_checkpoint<CKPT_STORE>(x, nullptr, codes, scales, nullptr, rows, D, (hipStream_t)stream);
}

extern "C" int ssam_checkpoint_restore(const void *codes, const float *scales, void *x, long rows, int D, void *stream)
{
    if (!x || !ssam_aligned16(x)) return SSAM_EINVAL;
    if (int rc = check_checkpoint(codes, scales, rows, D); rc != SSAM_OK) return rc;
    return launch_checkpoint<CKPT_RESTORE>(nullptr, x, const_cast<void *>(codes), const_cast<float *>(scales), nullptr, rows, D, (hipStream_t)stream);
}

extern "C" int ssam_gelu_checkpoint(const void *h, void *a, void *codes, float *scales, long rows, int D, void *stream)
{
    if (!h || !a || !ssam_aligned16(h) || !ssam_aligned16(a)) return SSAM_EINVAL;
    if (int rc = check_checkpoint(codes, scales, rows, D); rc != SSAM_OK) return rc;
    return launch_checkpoint<CKPT_GELU>(h, a, codes, scales, nullptr, rows, D, (hipStream_t)stream);
}

extern "C" int ssam_gelu_backward(const void *codes, const float *scales, const void *da, void *dh, void *a, long rows, int D, void *stream)
{
    if (!da || !dh || !ssam_aligned16(da) || !ssam_aligned16(dh) || !ssam_aligned16(a)) return SSAM_EINVAL;
    if (int rc = check_checkpoint(codes, scales, rows, D); rc != SSAM_OK) return rc;
    return launch_checkpoint<CKPT_GELU_BACKWARD>(da, dh, const_cast<void *>(codes), const_cast<float *>(scales), a, rows, D, (hipStream_t)stream);
}
