// The step between two halves of a block, forward and backward, and rows in 8 bits: the branch behind its own LayerNorm and a gate joins the scaled residual
// stream, whose LayerNorm goes to the rows that the next half reads, in bf16 or in 8 bits.  All of it is bound by HBM: one pass over the data, 16 bytes of bf16 per
// lane and request.
#include "rows8.h"

namespace {

constexpr int WAVES = 4;                      // of a workgroup
constexpr long MOST_ROWS = 0x7fff0000L;       // row indices and what is added to them stay in 32 bits

// The 16-byte chunks of a row that a lane has: lane, lane + 64, ...; one past the row re-reads the last one and is masked in the arithmetic.
template <int MAXC>
struct Chunks {
    int at[MAXC];
    bool in[MAXC];
    float over_D;
    __device__ __forceinline__ Chunks(int chunks)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            in[i] = lane + 64 * i < chunks;
            at[i] = min(lane + 64 * i, chunks - 1);
        }
        over_D = 1.f / (float)(chunks * 8);
    }
    __device__ __forceinline__ void load(const uint4 *row, uint4 (&r)[MAXC]) const
    {
#pragma unroll
        for (int i = 0; i < MAXC; ++i) r[i] = row[at[i]];
    }
    __device__ __forceinline__ void store(uint4 *row, const float (&v)[MAXC][8]) const
    {
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
            if (in[i]) row[at[i]] = pack_bf16x8(v[i]);
    }
    __device__ __forceinline__ void unpack(const uint4 (&r)[MAXC], float (&v)[MAXC][8]) const
    {
#pragma unroll
        for (int i = 0; i < MAXC; ++i) unpack_bf16x8(r[i], v[i]);
    }
    // eight values of an fp32 vector [D]
    __device__ __forceinline__ void values(const float *p, int i, float (&v)[8]) const
    {
        const float4 lo = reinterpret_cast<const float4 *>(p)[2 * at[i]], hi = reinterpret_cast<const float4 *>(p)[2 * at[i] + 1];
        v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
    }
    // v -> (v - mean) / deviation; returns one over the deviation.  Two passes over the registers, fp32.
    __device__ __forceinline__ float normalise(float (&v)[MAXC][8], float eps) const
    {
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += in[i] ? v[i][e] : 0.f;
        const float mean = wave_sum(s) * over_D;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[i][e] -= mean; q += in[i] ? v[i][e] * v[i][e] : 0.f; }
        const float rstd = rsqrtf(wave_sum(q) * over_D + eps);
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= rstd;
        return rstd;
    }
    // The gradient of normalise: g -> rstd (g - mean(g) - h mean(g h))
    __device__ __forceinline__ void normalise_back(float (&g)[MAXC][8], const float (&h)[MAXC][8], float rstd) const
    {
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s1 += in[i] ? g[i][e] : 0.f;
                s2 += in[i] ? g[i][e] * h[i][e] : 0.f;
            }
        s1 = wave_sum(s1) * over_D;
        s2 = wave_sum(s2) * over_D;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) g[i][e] = rstd * (g[i][e] - s1 - h[i][e] * s2);
    }
};

// Which rows of the branch (p) and of y (q) belong to token t of image b; -1: none.
struct TokenRows {
    const int32_t *src, *dst;
    int src_stride, dst_stride, No, Ny;       // No, Ny 0: no branch, no second LayerNorm
    __device__ __forceinline__ int branch(int b, int t) const { return of(src, src_stride, No, b, t); }
    __device__ __forceinline__ int out(int b, int t) const { return of(dst, dst_stride, Ny, b, t); }
    __device__ __forceinline__ static int of(const int32_t *map, int stride, int rows, int b, int t)
    {
        if (rows == 0) return -1;
        const int r = map ? map[(long)b * stride + t] : t;
        return (unsigned)r < (unsigned)rows ? r : -1;
    }
};

struct StepArgs {
    const uint4 *x;
    uint4 *x_out;
    const uint4 *o;
    TokenRows rows;
    const float *post_g, *post_b, *gate, *pre_g, *pre_b;
    int gate_stride;
    float alpha, eps;
    void *y;
    float *scales;
    int tokens, N, chunks;
};

enum StepOut { STEP_NONE, STEP_BF16, STEP_8BIT };

// One wave per token, its row and the branch's in registers.
template <int MAXC, bool POST, StepOut OUT>
__global__ void __launch_bounds__(256)
residual_norm_kernel(StepArgs a)
{
    const int row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.tokens) return;
    const int b = row / a.N, t = row - b * a.N;
    const int p = a.rows.branch(b, t), q = OUT == STEP_NONE ? -1 : a.rows.out(b, t);
    const bool writes = a.x_out && (p >= 0 || a.x_out != a.x);
    if (q < 0 && !writes) return;
    const Chunks<MAXC> ch(a.chunks);
    uint4 raw[MAXC];
    ch.load(a.x + (long)row * a.chunks, raw);
    float v[MAXC][8];
    if (p >= 0) {
        uint4 other[MAXC];
        ch.load(a.o + ((long)b * a.rows.No + p) * a.chunks, other);
        float n[MAXC][8];
        ch.unpack(raw, v);
        ch.unpack(other, n);
        if constexpr (POST) ch.normalise(n, a.eps);
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            float g[8], s[8];
            if constexpr (POST) {
                ch.values(a.post_g, i, g);
                ch.values(a.post_b, i, s);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[i][e] = fmaf(n[i][e], g[e], s[e]);
            }
            if (a.gate) {
                ch.values(a.gate + (long)b * a.gate_stride, i, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) n[i][e] *= g[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = fmaf(a.alpha, v[i][e], n[i][e]);
            raw[i] = pack_bf16x8(v[i]);
        }
    }
    if (writes) {
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
            if (ch.in[i]) a.x_out[(long)row * a.chunks + ch.at[i]] = raw[i];
    }
    if constexpr (OUT != STEP_NONE) {
        if (q < 0) return;
        ch.unpack(raw, v);                       // the stream as it is stored
        ch.normalise(v, a.eps);
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            float g[8], s[8];
            ch.values(a.pre_g, i, g);
            ch.values(a.pre_b, i, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e], g[e], s[e]);
        }
        const long to = (long)b * a.rows.Ny + q;
        if constexpr (OUT == STEP_BF16) {
            ch.store((uint4 *)a.y + to * a.chunks, v);
        } else {
            // magnitudes order as their bits do, infinities and NaN highest (lanes past the row repeat its last values)
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[i][e]) & 0x7fffffffu);
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
            const bool finite = top < 0x7f800000u;
            const RowScale s = row_scale(finite ? __uint_as_float(top) : 0.f);
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
                if (ch.in[i]) ((uint2 *)a.y)[to * a.chunks + ch.at[i]] = finite ? codes_of(v[i], s.inv) : make_uint2(0, 0);
            if ((threadIdx.x & 63) == 0) a.scales[to] = finite ? s.scale : __uint_as_float(0x7fc00000u);
        }
    }
}

template <int MAXC>
int launch_step(const StepArgs &a, bool post, StepOut out, hipStream_t st)
{
    auto go = post ? (out == STEP_NONE ? residual_norm_kernel<MAXC, true, STEP_NONE> : out == STEP_BF16 ? residual_norm_kernel<MAXC, true, STEP_BF16> : residual_norm_kernel<MAXC, true, STEP_8BIT>)
                   : (out == STEP_NONE ? residual_norm_kernel<MAXC, false, STEP_NONE> : out == STEP_BF16 ? residual_norm_kernel<MAXC, false, STEP_BF16> : residual_norm_kernel<MAXC, false, STEP_8BIT>);
    hipLaunchKernelGGL(go, dim3(ssam_div_up(a.tokens, WAVES)), dim3(64 * WAVES), 0, st, a);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}

int launch_step(const StepArgs &a, bool post, StepOut out, hipStream_t st)
{
    const int maxc = ssam_div_up(a.chunks, 64);
    return maxc == 1 ? launch_step<1>(a, post, out, st) : maxc == 2 ? launch_step<2>(a, post, out, st) : maxc == 3 ? launch_step<3>(a, post, out, st) : launch_step<4>(a, post, out, st);
}

// ---------------------------------------------------------------- backward
// A token's G = dx_out + gradient of the second LayerNorm is all that the rest needs, and stays in registers:
//   dx = alpha G (G without a branch),  dn = gate G,  do = gradient of the first LayerNorm (dn).
// The weights' gradients come from sums over tokens of at most four vectors: G, G h, dy h_x and dy (h, h_x: the normalised rows; h = o without a first LayerNorm):
//   dgate = post_g sum(G h) + post_b sum(G) or sum(G o),  dpost_g = gate sum(G h),  dpost_b = gate sum(G);  with a gate of every image the first two are summed per image.
// Waves walk the tokens and keep their share of the sums in registers; the four waves of a workgroup add theirs up in LDS, a second launch adds
// the workgroups' up, a third the images', all in a fixed order: no atomics, the same bits every time.
struct BackArgs {
    const uint4 *x_out, *o, *dy, *dx_out;
    uint4 *dx, *d_o;
    TokenRows rows;
    const float *post_g, *gate, *pre_g;
    int gate_stride;
    float alpha, eps;
    float *parts;                             // [images or 1][workgroups][NV][D]
    int tokens, N, chunks;                    // tokens: of a group (gridDim.y groups)
};

// Sums of a launch: vectors of them, and where each is
template <bool POST, bool PRE>
struct Sums {
    static constexpr int GH = 0, G = 1, DYH = 1 + POST, DY = 2 + POST, NV = 1 + POST + 2 * PRE;
};

template <int MAXC, bool POST, bool PRE, bool WEIGHTS>
__global__ void __launch_bounds__(256)
residual_norm_backward_kernel(BackArgs a)
{
    using V = Sums<POST, PRE>;
    __shared__ float4 lds[WEIGHTS ? WAVES * 64 * 2 : 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const Chunks<MAXC> ch(a.chunks);
    float sums[WEIGHTS ? V::NV : 1][MAXC][8];
    if constexpr (WEIGHTS)
#pragma unroll
        for (int w = 0; w < V::NV; ++w)
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[w][i][e] = 0.f;
    for (int r = blockIdx.x * WAVES + wave; r < a.tokens; r += gridDim.x * WAVES) {
        const int row = blockIdx.y * a.tokens + r, b = row / a.N, t = row - b * a.N;
        const int p = a.rows.branch(b, t), q = PRE ? a.rows.out(b, t) : -1;
        const long at = (long)row * a.chunks, branch = ((long)b * a.rows.No + p) * a.chunks;
        uint4 rg[MAXC], ro[MAXC], rx[MAXC], ry[MAXC];
        if (a.dx_out) ch.load(a.dx_out + at, rg);
        if (p >= 0) ch.load(a.o + branch, ro);
        if (PRE && q >= 0) {
            ch.load(a.x_out + at, rx);
            ch.load(a.dy + ((long)b * a.rows.Ny + q) * a.chunks, ry);
        }
        float g[MAXC][8];
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            if (!a.dx_out) rg[i] = make_uint4(0, 0, 0, 0);
            unpack_bf16x8(rg[i], g[i]);
        }
        if (PRE && q >= 0) {
            float h[MAXC][8], d[MAXC][8];
            ch.unpack(rx, h);
            ch.unpack(ry, d);
            const float rstd = ch.normalise(h, a.eps);
#pragma unroll
            for (int i = 0; i < MAXC; ++i) {
                float w[8];
                ch.values(a.pre_g, i, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (WEIGHTS && PRE) {          // of lanes past the row these are never stored
                        sums[V::DYH][i][e] = fmaf(d[i][e], h[i][e], sums[V::DYH][i][e]);
                        sums[V::DY][i][e] += d[i][e];
                    }
                    d[i][e] *= w[e];
                }
            }
            ch.normalise_back(d, h, rstd);
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[i][e] += d[i][e];
        }
        if (p >= 0) {
            float h[MAXC][8], d[MAXC][8];
            ch.unpack(ro, h);
            float rstd = 1.f;
            if constexpr (POST) rstd = ch.normalise(h, a.eps);
#pragma unroll
            for (int i = 0; i < MAXC; ++i) {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (WEIGHTS) {
                        sums[V::GH][i][e] = fmaf(g[i][e], h[i][e], sums[V::GH][i][e]);
                        if constexpr (POST) sums[V::G][i][e] += g[i][e];
                    }
                    d[i][e] = g[i][e];
                    g[i][e] *= a.alpha;
                }
                if (a.gate) {
                    ch.values(a.gate + (long)b * a.gate_stride, i, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[i][e] *= w[e];
                }
                if constexpr (POST) {
                    ch.values(a.post_g, i, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[i][e] *= w[e];
                }
            }
            if constexpr (POST) ch.normalise_back(d, h, rstd);
            ch.store(a.d_o + branch, d);
        }
        ch.store(a.dx + at, g);
    }
    if constexpr (WEIGHTS) {
        // the waves' sums of 8 columns at a time, [wave][which half][lane]: every lane then adds up one float4 of four waves
        float *mine = a.parts + ((long)blockIdx.y * gridDim.x + blockIdx.x) * V::NV * a.chunks * 8;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int w = 0; w < V::NV; ++w) {
                const float *f = sums[w][i];
                __syncthreads();
                lds[(wave * 2 + 0) * 64 + lane] = make_float4(f[0], f[1], f[2], f[3]);
                lds[(wave * 2 + 1) * 64 + lane] = make_float4(f[4], f[5], f[6], f[7]);
                __syncthreads();
                if (wave < 2 && ch.in[i]) {
                    float4 s = lds[wave * 64 + lane];
#pragma unroll
                    for (int o = 1; o < WAVES; ++o) {
                        const float4 t = lds[(o * 2 + wave) * 64 + lane];
                        s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
                    }
                    reinterpret_cast<float4 *>(mine + (long)w * a.chunks * 8)[2 * (lane + 64 * i) + wave] = s;
                }
            }
    }
}

struct WeightGrads {
    const float *post_g, *post_b, *gate;
    int gate_stride;
    float *dgate, *dpost_g, *dpost_b, *dpre_g, *dpre_b;
    int D;
};

__device__ __forceinline__ float4 mul4(float4 a, float4 b) { return make_float4(a.x * b.x, a.y * b.y, a.z * b.z, a.w * b.w); }
__device__ __forceinline__ float4 add4(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// The sums of a group of tokens, of four columns -> the gradients
template <bool POST, bool PRE>
__device__ __forceinline__ void gate_gradient(const WeightGrads &w, int image, int quad, const float4 *s)
{
    using V = Sums<POST, PRE>;
    float4 d = s[V::GH];
    if constexpr (POST) d = add4(mul4(reinterpret_cast<const float4 *>(w.post_g)[quad], s[V::GH]), mul4(reinterpret_cast<const float4 *>(w.post_b)[quad], s[V::G]));
    if (w.dgate) reinterpret_cast<float4 *>(w.dgate + (long)image * w.D)[quad] = d;
}

template <bool POST, bool PRE>
__device__ __forceinline__ void norm_gradients(const WeightGrads &w, int quad, const float4 *s)      // s: the gate is in it
{
    using V = Sums<POST, PRE>;
    auto put = [&](float *to, const float4 &v) { if (to) reinterpret_cast<float4 *>(to)[quad] = v; };
    if constexpr (POST) { put(w.dpost_g, s[V::GH]); put(w.dpost_b, s[V::G]); }
    if constexpr (PRE) { put(w.dpre_g, s[V::DYH]); put(w.dpre_b, s[V::DY]); }
}

template <bool POST, bool PRE>
__device__ __forceinline__ void times_gate(const WeightGrads &w, int image, int quad, float4 *s)
{
    using V = Sums<POST, PRE>;
    if (!POST || !w.gate) return;
    const float4 g = reinterpret_cast<const float4 *>(w.gate + (long)image * w.gate_stride)[quad];
    s[V::GH] = mul4(s[V::GH], g);
    if constexpr (POST) s[V::G] = mul4(s[V::G], g);
}

// [groups][n][NV][D] -> sums over n.  A workgroup adds up 32 columns of a group: eight lanes with 16 bytes each, 32 slices of the rows.  One group: the gradients; more: the
// gate's of the group, and its sums, gate in them, to `images` [groups][NV][D].
template <bool POST, bool PRE>
__global__ void __launch_bounds__(256)
residual_weight_sums_kernel(const float4 *__restrict__ parts, int n, WeightGrads w, float4 *images)
{
    constexpr int NV = Sums<POST, PRE>::NV;
    __shared__ float4 lds[256];
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3, quads = w.D / 4, quad = blockIdx.x * 8 + c, at = min(quad, quads - 1), group = blockIdx.y;
    parts += (long)group * n * NV * quads;
    float4 s[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int r = slice; r < n; r += 32)
#pragma unroll
        for (int k = 0; k < NV; ++k) s[k] = add4(s[k], parts[((long)r * NV + k) * quads + at]);
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] = sum_of_shares(s[k], lds);
    if (slice != 0 || quad >= quads) return;
    gate_gradient<POST, PRE>(w, group, quad, s);
    times_gate<POST, PRE>(w, group, quad, s);
    if (gridDim.y == 1) {
        norm_gradients<POST, PRE>(w, quad, s);
        return;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) images[((long)group * NV + k) * quads + quad] = s[k];
}

template <bool POST, bool PRE>
__global__ void __launch_bounds__(64)
residual_image_sums_kernel(const float4 *__restrict__ images, int groups, WeightGrads w)
{
    constexpr int NV = Sums<POST, PRE>::NV;
    const int quads = w.D / 4, quad = blockIdx.x * 64 + threadIdx.x;
    if (quad >= quads) return;
    float4 s[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) s[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int g = 0; g < groups; ++g)
#pragma unroll
        for (int k = 0; k < NV; ++k) s[k] = add4(s[k], images[((long)g * NV + k) * quads + quad]);
    norm_gradients<POST, PRE>(w, quad, s);
}

// Workgroups that a group of tokens is dealt to: two waves to a SIMD of 256 CUs over all groups.
inline int backward_workgroups(long tokens, int groups)
{
    const long most = ssam_div_up(512, groups), need = (tokens + WAVES - 1) / WAVES;
    return (int)(need < most ? need : most);
}

template <int MAXC, bool POST, bool PRE>
int launch_backward(const BackArgs &a, const WeightGrads &w, bool weights, int groups, hipStream_t st)
{
    const int n = backward_workgroups(a.tokens, groups);
    const dim3 grid(n, groups);
    hipLaunchKernelGGL((weights ? residual_norm_backward_kernel<MAXC, POST, PRE, true> : residual_norm_backward_kernel<MAXC, POST, PRE, false>), grid, dim3(64 * WAVES), 0, st, a);
    SSAM_CHECK_LAUNCH();
    if (!weights) return SSAM_OK;
    float4 *images = reinterpret_cast<float4 *>(a.parts + (size_t)groups * n * Sums<POST, PRE>::NV * w.D);
    hipLaunchKernelGGL((residual_weight_sums_kernel<POST, PRE>), dim3(ssam_div_up(w.D, 32), groups), dim3(256), 0, st, (const float4 *)a.parts, n, w, images);
    SSAM_CHECK_LAUNCH();
    if (groups > 1) {
        hipLaunchKernelGGL((residual_image_sums_kernel<POST, PRE>), dim3(ssam_div_up(w.D, 256)), dim3(64), 0, st, (const float4 *)images, groups, w);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int MAXC>
int launch_backward(const BackArgs &a, const WeightGrads &w, bool post, bool pre, bool weights, int groups, hipStream_t st)
{
    auto go = post ? (pre ? launch_backward<MAXC, true, true> : launch_backward<MAXC, true, false>) : (pre ? launch_backward<MAXC, false, true> : launch_backward<MAXC, false, false>);
    return go(a, w, weights, groups, st);
}

// ---------------------------------------------------------------- rows in 8 bits
// One wave per row: its largest magnitude, then its codes.  Rows of up to 64 * 8 * MAXC features stay in registers in between; MAXC = 0: longer ones are read twice.
template <int MAXC>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const uint4 *__restrict__ x, uint2 *__restrict__ codes, float *__restrict__ scales, long rows, int chunks)
{
    const long row = (long)blockIdx.x * WAVES + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (row >= rows) return;
    x += row * chunks;
    codes += row * chunks;
    uint4 v[MAXC ? MAXC : 1];
    uint32_t top = 0;
    if constexpr (MAXC != 0) {
#pragma unroll
        for (int i = 0; i < MAXC; ++i) v[i] = x[min(lane + 64 * i, chunks - 1)];
#pragma unroll
        for (int i = 0; i < MAXC; ++i) top = max_u16x2(top, top_of_bf16x8(v[i]));
    } else {
        for (int c = lane; c < chunks; c += 64) top = max_u16x2(top, top_of_bf16x8(x[c]));
    }
    top = max(top >> 16, top & 0xffffu);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    const bool finite = top < 0x7f80u;
    const RowScale s = row_scale(finite ? bf16_bits_to_float(top) : 0.f);
    auto put = [&](int c, const uint4 &r) {
        float f[8];
        unpack_bf16x8(r, f);
        codes[c] = finite ? codes_of(f, s.inv) : make_uint2(0, 0);
    };
    if constexpr (MAXC != 0) {
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
            if (lane + 64 * i < chunks) put(lane + 64 * i, v[i]);
    } else {
        for (int c = lane; c < chunks; c += 64) put(c, x[c]);
    }
    if (lane == 0) scales[row] = finite ? s.scale : __uint_as_float(0x7fc00000u);
}

// ---------------------------------------------------------------- inverse tables
__global__ void __launch_bounds__(256)
fill_rows_kernel(int32_t *inv, int n)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) inv[i] = -1;
}

int check_step(const void *o, const int32_t *src, int src_stride, const float *post_g, const float *post_b, const float *gate, int gate_stride, const float *pre_g,
               const int32_t *dst, int dst_stride, int B, int N, int No, int Ny, int D)
{
    if (B <= 0 || N <= 0 || D <= 0 || D % 8 != 0) return SSAM_EINVAL;
    if (!post_g && post_b) return SSAM_EINVAL;
    if (!ssam_aligned16(o) || !ssam_aligned16(post_g) || !ssam_aligned16(post_b) || !ssam_aligned16(gate) || !ssam_aligned16(pre_g)) return SSAM_EINVAL;
    if (o) {
        if (No <= 0 || (!src && No != N) || (src && src_stride != 0 && src_stride < N)) return SSAM_EINVAL;
    } else if (src || post_g || gate) {
        return SSAM_EINVAL;
    }
    if (gate && gate_stride != 0 && (gate_stride < D || gate_stride % 4)) return SSAM_EINVAL;
    if (pre_g) {
        if (Ny <= 0 || (!dst && Ny != N) || (dst && dst_stride != 0 && dst_stride < N)) return SSAM_EINVAL;
    } else if (dst) {
        return SSAM_EINVAL;
    }
    if (!o && !pre_g) return SSAM_EINVAL;
    return D > 2048 || (long)B * N > MOST_ROWS ? SSAM_EUNSUPPORTED : SSAM_OK;
}

int step(const void *x, void *x_out, const void *o, const int32_t *src, int src_stride, const float *post_g, const float *post_b, const float *gate, int gate_stride, float alpha,
         const float *pre_g, const float *pre_b, const int32_t *dst, int dst_stride, float eps, void *y, float *scales, StepOut out, int B, int N, int No, int Ny, int D, void *stream)
{
    if (!x || !ssam_aligned16(x) || !ssam_aligned16(x_out) || !ssam_aligned16(y) || !ssam_aligned16(scales) || !ssam_aligned16(pre_b)) return SSAM_EINVAL;
    if ((!post_g) != (!post_b) || (!pre_g) != (!pre_b) || (!pre_g) != (!y) || !(eps > 0.f)) return SSAM_EINVAL;
    if (o ? !x_out : x_out && x_out != x) return SSAM_EINVAL;
    if (int rc = check_step(o, src, src_stride, post_g, post_b, gate, gate_stride, pre_g, dst, dst_stride, B, N, No, Ny, D); rc != SSAM_OK) return rc;
    const TokenRows rows = { src, dst, src_stride, dst_stride, o ? No : 0, pre_g ? Ny : 0 };
    const StepArgs a = { (const uint4 *)x, (uint4 *)x_out, (const uint4 *)o, rows, post_g, post_b, gate, pre_g, pre_b, gate_stride, alpha, eps, y, scales, B * N, N, D / 8 };
    return launch_step(a, post_g != nullptr, out, (hipStream_t)stream);
}

}  // namespace

int ssam_invert_table(const int32_t *table, int table_batch_stride, int B, int Nout, int N, int32_t *inv, hipStream_t st);        // movers.hip

extern "C" int ssam_invert_rows(const int32_t *idx, int idx_batch_stride, int32_t *inv, int B, int Nout, int N, void *stream)
{
    if (!idx || !inv || B <= 0 || Nout <= 0 || N <= 0 || (idx_batch_stride != 0 && idx_batch_stride < Nout)) return SSAM_EINVAL;
    if ((long)B * N > MOST_ROWS || (long)B * Nout > MOST_ROWS) return SSAM_EUNSUPPORTED;
    hipLaunchKernelGGL(fill_rows_kernel, dim3(ssam_div_up((long)B * N, 256)), dim3(256), 0, (hipStream_t)stream, inv, B * N);
    SSAM_CHECK_LAUNCH();
    return ssam_invert_table(idx, idx_batch_stride, B, Nout, N, inv, (hipStream_t)stream);
}

extern "C" int ssam_quantize_rows(const void *x, void *codes, float *scales, long rows, int D, void *stream)
{
    if (!x || !codes || !scales || rows <= 0 || D <= 0 || !ssam_aligned16(x) || !ssam_aligned16(codes) || !ssam_aligned16(scales)) return SSAM_EINVAL;
    if (D % 16 != 0 || D >= 131072 || rows > 4 * 0x7fffffffL) return SSAM_EUNSUPPORTED;
    const int chunks = D / 8, maxc = ssam_div_up(chunks, 64);
    auto go = maxc == 1 ? quantize_rows_kernel<1> : maxc == 2 ? quantize_rows_kernel<2> : maxc == 3 ? quantize_rows_kernel<3> : maxc == 4 ? quantize_rows_kernel<4>
            : maxc <= 10 ? quantize_rows_kernel<10> : quantize_rows_kernel<0>;
    hipLaunchKernelGGL(go, dim3((unsigned)((rows + WAVES - 1) / WAVES)), dim3(64 * WAVES), 0, (hipStream_t)stream, (const uint4 *)x, (uint2 *)codes, scales, rows, chunks);
    SSAM_CHECK_LAUNCH();
    return SSAM_OK;
}

extern "C" int ssam_residual_norm(const void *x, void *x_out, const void *o, const int32_t *src, int src_batch_stride, const float *post_g, const float *post_b,
                                  const float *gate, int gate_batch_stride, float alpha, const float *pre_g, const float *pre_b, const int32_t *dst, int dst_batch_stride,
                                  float eps, void *y, int B, int N, int No, int Ny, int D, void *stream)
{
    return step(x, x_out, o, src, src_batch_stride, post_g, post_b, gate, gate_batch_stride, alpha, pre_g, pre_b, dst, dst_batch_stride, eps, y, nullptr,
                y ? STEP_BF16 : STEP_NONE, B, N, No, Ny, D, stream);
}

extern "C" int ssam_residual_norm_i8(const void *x, void *x_out, const void *o, const int32_t *src, int src_batch_stride, const float *post_g, const float *post_b,
                                     const float *gate, int gate_batch_stride, float alpha, const float *pre_g, const float *pre_b, const int32_t *dst, int dst_batch_stride,
                                     float eps, void *codes, float *scales, int B, int N, int No, int Ny, int D, void *stream)
{
    if (!pre_g || !scales) return SSAM_EINVAL;
    if (D > 0 && D % 8 == 0 && D % 16 != 0) return SSAM_EUNSUPPORTED;
    return step(x, x_out, o, src, src_batch_stride, post_g, post_b, gate, gate_batch_stride, alpha, pre_g, pre_b, dst, dst_batch_stride, eps, codes, scales, STEP_8BIT,
                B, N, No, Ny, D, stream);
}

extern "C" size_t ssam_residual_norm_backward_workspace_bytes(int B, int N, int D, int gate_images)
{
    if (B <= 0 || N <= 0 || D <= 0 || (gate_images != 1 && gate_images != B)) return 0;
    const int n = backward_workgroups(gate_images == 1 ? (long)B * N : N, gate_images);
    return (size_t)gate_images * (n + (gate_images > 1)) * 4 * D * sizeof(float);
}

extern "C" int ssam_residual_norm_backward(const void *x_out, const void *o, const int32_t *src, int src_batch_stride, const float *post_g, const float *post_b,
                                           const float *gate, int gate_batch_stride, float alpha, const float *pre_g, const int32_t *dst, int dst_batch_stride, float eps,
                                           const void *dy, const void *dx_out, void *dx, void *d_o, float *dgate, float *dpost_g, float *dpost_b, float *dpre_g, float *dpre_b,
                                           int B, int N, int No, int Ny, int D, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!x_out || !dx || (!o) != (!d_o) || (!pre_g) != (!dy) || !(eps > 0.f) || (!post_g) != (!post_b)) return SSAM_EINVAL;
    if ((dgate && !gate) || ((dpost_g || dpost_b) && !post_g) || ((dpre_g || dpre_b) && !pre_g)) return SSAM_EINVAL;
    for (const void *p : { x_out, dy, dx_out, (const void *)dx, (const void *)d_o, (const void *)dgate, (const void *)dpost_g, (const void *)dpost_b, (const void *)dpre_g, (const void *)dpre_b })
        if (!ssam_aligned16(p)) return SSAM_EINVAL;
    if (int rc = check_step(o, src, src_batch_stride, post_g, post_b, gate, gate_batch_stride, pre_g, dst, dst_batch_stride, B, N, No, Ny, D); rc != SSAM_OK) return rc;
    const bool weights = dgate || dpost_g || dpost_b || dpre_g || dpre_b;
    const int groups = gate && gate_batch_stride ? B : 1;
    if (weights) {
        if (groups > 65535) return SSAM_EUNSUPPORTED;                  // gridDim.y
        if (!workspace || !ssam_aligned16(workspace)) return SSAM_EINVAL;
        if (workspace_bytes < ssam_residual_norm_backward_workspace_bytes(B, N, D, groups)) return SSAM_EWORKSPACE;
    }
    const TokenRows rows = { src, dst, src_batch_stride, dst_batch_stride, o ? No : 0, pre_g ? Ny : 0 };
    const BackArgs a = { (const uint4 *)x_out, (const uint4 *)o, (const uint4 *)dy, (const uint4 *)dx_out, (uint4 *)dx, (uint4 *)d_o, rows, post_g, gate, pre_g,
                         gate_batch_stride, alpha, eps, (float *)workspace, weights && groups > 1 ? N : B * N, N, D / 8 };
    const WeightGrads w = { post_g, post_b, gate, gate_batch_stride, dgate, dpost_g, dpost_b, dpre_g, dpre_b, D };
    const int maxc = ssam_div_up(D / 8, 64);
    auto go = maxc == 1 ? launch_backward<1> : maxc == 2 ? launch_backward<2> : maxc == 3 ? launch_backward<3> : launch_backward<4>;
    return go(a, w, post_g != nullptr, pre_g != nullptr, weights, weights ? groups : 1, (hipStream_t)stream);
}
