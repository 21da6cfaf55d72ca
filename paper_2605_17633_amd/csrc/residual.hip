// The step between two halves of a block, forward and backward, and rows in 8 bits: the branch behind its own LayerNorm and a gate joins the scaled residual
// stream, whose LayerNorm goes to the rows that the next half reads, in bf16 or in 8 bits.  All of it is bound by HBM: one pass over the data, 16 bytes of bf16 per
// lane and request.
#include <type_traits>

#include "rows8.h"

namespace {

constexpr int WAVES = 4;                      // of a workgroup
constexpr long MOST_ROWS = 0x7fff0000L;       // row indices and what is added to them stay in 32 bits
constexpr long MOST_WORKGROUPS = 1L << 22;    // of a launch, which has less than 2^32 threads

// Past the caches: of a step over 32768 x 1280 and its gradient, one behind the other, 173 -> 146 us, of a step between two contractions 3 % or nothing.  (Loads past the caches too: 169.)
__device__ __forceinline__ void put16(uint4 *to, const uint4 &v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(to)); }
__device__ __forceinline__ void put8(uint2 *to, const uint2 &v) { __builtin_nontemporal_store(__builtin_bit_cast(unsigned long, v), reinterpret_cast<unsigned long *>(to)); }

// The 16-byte chunks of a row that a lane has: lane, lane + LANES, ...; one past the row re-reads the last one and is masked in the arithmetic.  LANES: of a row; rows of up to 256
// features take 32 of a wave's, of up to 128 16 (65536 x 144 with a wave to a row 30.8 us, bound by arithmetic, now 18.5; its gradient 63, 40).
template <int MAXC, int LANES>
struct Chunks {
    static_assert(LANES == 64 || MAXC == 1, "narrow rows");
    int at[MAXC];
    bool in[MAXC];
    float over_D;
    __device__ __forceinline__ Chunks(int chunks)
    {
        const int lane = threadIdx.x & (LANES - 1);
#pragma unroll
        for (int i = 0; i < MAXC; ++i) {
            in[i] = lane + LANES * i < chunks;
            at[i] = min(lane + LANES * i, chunks - 1);
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
            if (in[i]) put16(row + at[i], pack_bf16x8(v[i]));
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
    // v -> (v - mean) / deviation, zeros past the row; returns one over the deviation.  Two passes over the registers, fp32.
    __device__ __forceinline__ float normalise(float (&v)[MAXC][8], float eps) const
    {
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += in[i] ? v[i][e] : 0.f;
        const float mean = lanes_sum<LANES>(s) * over_D;
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) { v[i][e] = in[i] ? v[i][e] - mean : 0.f; q = fmaf(v[i][e], v[i][e], q); }
        const float rstd = rsqrtf(lanes_sum<LANES>(q) * over_D + eps);
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] *= rstd;
        return rstd;
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
    int first, tokens, N, chunks;             // tokens from `first` on
};

enum StepOut { STEP_NONE, STEP_BF16, STEP_8BIT };

// This wave, or part of one, of LANES lanes among all of the launch.
template <int LANES>
__device__ __forceinline__ int row_of_lanes()
{
    if constexpr (LANES == 64) return blockIdx.x * (blockDim.x / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    else return blockIdx.x * (blockDim.x / LANES) + threadIdx.x / LANES;
}

// One wave, or part of one, per token, its row and the branch's in registers; the norms' and the gate's vectors come from the caches.  Bound by HBM: 32768 x 1280 in the order of windows, 40 % of it
// normed (285 MB) 61 us, 4.7 TB/s; 784 x 768 4.7 us; 16384 x 1024 with 40 % of the branch, in 8 bits (97 MB) 19 us.
template <int MAXC, int LANES, bool POST, StepOut OUT>
__global__ void __launch_bounds__(256)
residual_norm_kernel(StepArgs a)
{
    const int row = a.first + row_of_lanes<LANES>();
    if (row >= a.tokens) return;
    const int b = row / a.N, t = row - b * a.N;
    const int p = a.rows.branch(b, t), q = OUT == STEP_NONE ? -1 : a.rows.out(b, t);
    const bool writes = a.x_out && (p >= 0 || a.x_out != a.x);
    if (q < 0 && !writes) return;
    const Chunks<MAXC, LANES> ch(a.chunks);
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
            if (ch.in[i]) put16(a.x_out + (long)row * a.chunks + ch.at[i], raw[i]);
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
            // magnitudes order as their bits do, infinities and NaN highest
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, ch.in[i] ? __float_as_uint(v[i][e]) & 0x7fffffffu : 0u);
            top = lanes_max<LANES>(top);
            const bool finite = top < 0x7f800000u;
            const RowScale s = row_scale(finite ? __uint_as_float(top) : 0.f);
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
                if (ch.in[i]) put8((uint2 *)a.y + to * a.chunks + ch.at[i], finite ? codes_of(v[i], s.inv) : make_uint2(0, 0));
            if ((threadIdx.x & (LANES - 1)) == 0) a.scales[to] = finite ? s.scale : __uint_as_float(0x7fc00000u);
        }
    }
}

template <int MAXC, int LANES>
int launch_step(StepArgs a, bool post, StepOut out, hipStream_t st)
{
    auto go = post ? (out == STEP_NONE ? residual_norm_kernel<MAXC, LANES, true, STEP_NONE> : out == STEP_BF16 ? residual_norm_kernel<MAXC, LANES, true, STEP_BF16> : residual_norm_kernel<MAXC, LANES, true, STEP_8BIT>)
                   : (out == STEP_NONE ? residual_norm_kernel<MAXC, LANES, false, STEP_NONE> : out == STEP_BF16 ? residual_norm_kernel<MAXC, LANES, false, STEP_BF16> : residual_norm_kernel<MAXC, LANES, false, STEP_8BIT>);
    constexpr int ROWS = WAVES * 64 / LANES;
    for (long first = 0; first < a.tokens; first += MOST_WORKGROUPS * ROWS) {
        a.first = (int)first;
        const long left = ((long)a.tokens - first + ROWS - 1) / ROWS;
        hipLaunchKernelGGL(go, dim3((unsigned)(left < MOST_WORKGROUPS ? left : MOST_WORKGROUPS)), dim3(64 * WAVES), 0, st, a);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

// The kernel for rows of so many 16-byte chunks: call(MAXC, LANES)
template <class Call>
int by_width(int chunks, Call call)
{
    using std::integral_constant;
    if (chunks <= 16) return call(integral_constant<int, 1>{}, integral_constant<int, 16>{});
    if (chunks <= 32) return call(integral_constant<int, 1>{}, integral_constant<int, 32>{});
    if (chunks <= 64) return call(integral_constant<int, 1>{}, integral_constant<int, 64>{});
    if (chunks <= 128) return call(integral_constant<int, 2>{}, integral_constant<int, 64>{});
    if (chunks <= 192) return call(integral_constant<int, 3>{}, integral_constant<int, 64>{});
    return call(integral_constant<int, 4>{}, integral_constant<int, 64>{});
}

// ---------------------------------------------------------------- backward
// A token's G = dx_out + gradient of the second LayerNorm is all that the rest needs, and stays in registers:
//   dx = alpha G (G without a branch),  dn = gate G,  do = gradient of the first LayerNorm (dn).
// The weights' gradients come from sums over tokens of at most four vectors: G h, G, dy h_x and dy (h, h_x: the normalised rows; h = o without a first LayerNorm):
//   dgate = post_g sum(G h) + post_b sum(G) or sum(G o),  dpost_g = gate sum(G h),  dpost_b = gate sum(G);  with a gate of every image the first two are summed per image.
// Waves walk the tokens and keep their share of the sums, two vectors in registers and the others in LDS (all four in registers leave one wave to a SIMD, under whose arithmetic
// nothing is requested); the eight waves of a workgroup add theirs up, a second launch adds the workgroups' up, a third the images', all in a fixed order: no atomics, the same bits every time.
// Bound by HBM: 32768 x 1280 (453 MB) 87 us, 5.2 TB/s, and 4 the sums; with sums over lanes through LDS 175, without those but all sums in registers and no token requested ahead 153.
// 784 x 768: 7.6 and 3.5 us.  Rows up to 512 are bound by the instructions of a row, which are as many whatever part of its lanes it fills (16, 32 or 64): 65536 x 144 and x 256 take 41 us both (2.8 and
// 4.9 TB/s), 65536 x 288 and x 512 66 and 74.
struct BackArgs {
    const uint4 *x_out, *o, *dy, *dx_out;
    uint4 *dx, *d_o;
    TokenRows rows;
    const float *post_g, *gate, *pre_g;
    int gate_stride;
    float alpha, eps;
    float *parts;                             // [groups][workgroups][NV][D]
    int tokens, N, chunks;                    // tokens: of a group (gridDim.y groups: images where the gate is of every image)
};

// Sums of a launch: vectors of them, and where each is; the first LDS of them are in LDS
template <bool POST, bool PRE>
struct Sums {
    static constexpr int GH = 0, G = 1, DYH = 1 + POST, DY = 2 + POST, NV = 1 + POST + 2 * PRE, IN_REGISTERS = NV < 2 ? NV : 2, IN_LDS = NV - IN_REGISTERS;
};

// Waves of a workgroup, one to a CU.  Rows above 1536 with the second LayerNorm and the weights' gradients spill 72 of the 256 registers that two waves to a SIMD have (16384 x 2048, both norms: 125 us
// with eight waves, 80 with four).  The other kernels of such rows fit 256, and four waves serve them as well: without the weights' gradients 63.9 us, with eight waves 65.0, without the second
// LayerNorm 48.1 and 47.8 (16384 x 1664 0 to 6 % faster with eight, 784 x 2048 2 to 15 % slower); so the number is the width's alone.
constexpr int back_waves(int maxc) { return maxc == 4 ? 4 : 8; }

// LDS of a workgroup: both norms' factors, and the waves' sums, or room for a vector of all of them
template <bool POST, bool PRE, bool WEIGHTS>
constexpr size_t backward_lds(int maxc)
{
    const int vectors = Sums<POST, PRE>::IN_LDS > 1 ? Sums<POST, PRE>::IN_LDS : 1;
    return sizeof(float4) * 128 * maxc * (2 + (WEIGHTS ? back_waves(maxc) * vectors : 0));
}

template <int MAXC, int LANES, bool POST, bool PRE, bool WEIGHTS>
__global__ void __launch_bounds__(64 * back_waves(MAXC))
residual_norm_backward_kernel(BackArgs a)
{
    using V = Sums<POST, PRE>;
    extern __shared__ float4 lds4[];              // [2][2 MAXC][64] factors, then [wave][IN_LDS][2 MAXC][64]: halves of a lane's chunks, lanes side by side
    constexpr int VECTOR = 2 * MAXC * 64, BACK_WAVES = back_waves(MAXC);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    constexpr int PARTS = 64 / LANES;                          // rows of a wave
    const Chunks<MAXC, LANES> ch(a.chunks);
    const float *gate = a.gate ? a.gate + (long)blockIdx.y * a.gate_stride : nullptr;
    float4 *const mine = lds4 + 2 * VECTOR + wave * (V::IN_LDS * VECTOR) + lane;
    // factors: of the second LayerNorm its gain, of the branch the gate times the first one's; zeros past the row
    for (int k = threadIdx.x; k < VECTOR; k += 64 * BACK_WAVES) {
        const int c = (k & (LANES - 1)) + 64 * (k >> 7), quad = 2 * c + ((k >> 6) & 1);
        const bool in = c < a.chunks;
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f), w = f;
        if (in && PRE) f = reinterpret_cast<const float4 *>(a.pre_g)[quad];
        if (in) {
            w = gate ? reinterpret_cast<const float4 *>(gate)[quad] : make_float4(1.f, 1.f, 1.f, 1.f);
            if constexpr (POST) {
                const float4 g = reinterpret_cast<const float4 *>(a.post_g)[quad];
                w.x *= g.x; w.y *= g.y; w.z *= g.z; w.w *= g.w;
            }
        }
        lds4[k] = f;
        lds4[VECTOR + k] = w;
    }
    float regs[WEIGHTS ? V::IN_REGISTERS : 1][MAXC][8];
    if constexpr (WEIGHTS) {
#pragma unroll
        for (int w = 0; w < V::IN_REGISTERS; ++w)
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) regs[w][i][e] = 0.f;
#pragma unroll
        for (int k = 0; k < V::IN_LDS * 2 * MAXC; ++k) mine[k * 64] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    auto factors = [&](int which, int i, float (&f)[8]) {
        const float4 lo = lds4[which * VECTOR + i * 128 + lane], hi = lds4[which * VECTOR + i * 128 + 64 + lane];
        f[0] = lo.x; f[1] = lo.y; f[2] = lo.z; f[3] = lo.w; f[4] = hi.x; f[5] = hi.y; f[6] = hi.z; f[7] = hi.w;
    };
    // sums of vector v (of lanes past the row they are never stored) += t * u
    auto add = [&](auto v_, int i, const float (&t)[8], const float (&u)[8]) {
        constexpr int v = decltype(v_)::value;
        if constexpr (v >= V::IN_LDS) {
#pragma unroll
            for (int e = 0; e < 8; ++e) regs[v - V::IN_LDS][i][e] = fmaf(t[e], u[e], regs[v - V::IN_LDS][i][e]);
        } else {
            float4 *p = mine + v * VECTOR + i * 128;
            float4 lo = p[0], hi = p[64];
            lo.x = fmaf(t[0], u[0], lo.x); lo.y = fmaf(t[1], u[1], lo.y); lo.z = fmaf(t[2], u[2], lo.z); lo.w = fmaf(t[3], u[3], lo.w);
            hi.x = fmaf(t[4], u[4], hi.x); hi.y = fmaf(t[5], u[5], hi.y); hi.z = fmaf(t[6], u[6], hi.z); hi.w = fmaf(t[7], u[7], hi.w);
            p[0] = lo;
            p[64] = hi;
        }
    };
    using std::integral_constant;
    constexpr float ONES[8] = { 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f };

    const int stride = gridDim.x * BACK_WAVES * PARTS;
    struct Token { int row, p, q; long branch, out; };         // p, q < 0: no branch, no row of y
    auto token = [&](int r) {
        Token t = { -1, -1, -1, 0, 0 };
        if (r >= a.tokens) return t;
        t.row = blockIdx.y * a.tokens + r;
        const int b = t.row / a.N, at = t.row - b * a.N;
        t.p = a.rows.branch(b, at);
        t.q = PRE ? a.rows.out(b, at) : -1;
        t.branch = ((long)b * a.rows.No + t.p) * a.chunks;
        t.out = ((long)b * a.rows.Ny + t.q) * a.chunks;
        return t;
    };
    uint4 rg[MAXC], ro[MAXC], rx[MAXC], ry[MAXC];
    auto request = [&](const Token &t) {
        if (t.row < 0) return;
        const long at = (long)t.row * a.chunks;
        if (PRE && t.q >= 0) {
            ch.load(a.x_out + at, rx);
            ch.load(a.dy + t.out, ry);
        }
        if (a.dx_out) ch.load(a.dx_out + at, rg);
        if (t.p >= 0) ch.load(a.o + t.branch, ro);
    };
    int r = row_of_lanes<LANES>();
    Token now = token(r), next = token(r + stride);            // (tokens + 2 strides stay below 2^31)
    request(now);
    for (; r < a.tokens; r += stride) {
        float g[MAXC][8], h[MAXC][8], d[MAXC][8], o[MAXC][8];
        ch.unpack(rg, g);
        ch.unpack(rx, h);
        ch.unpack(ry, d);
        ch.unpack(ro, o);
        // the next token's rows, and the token behind it: their round trips are under this one's arithmetic
        const Token t = now;
        request(next);
        now = next;
        next = token(r + 2 * stride);
        if (!a.dx_out) {
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[i][e] = 0.f;
        }
        if (PRE && t.q >= 0) {
            const float rstd = ch.normalise(h, a.eps);
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < MAXC; ++i) {
                float f[8];
                factors(0, i, f);
                if constexpr (WEIGHTS && PRE) {
                    add(integral_constant<int, V::DYH>{}, i, d[i], h[i]);
                    add(integral_constant<int, V::DY>{}, i, d[i], ONES);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[i][e] *= f[e];
                    s1 += d[i][e];
                    s2 = fmaf(d[i][e], h[i][e], s2);
                }
            }
            s1 = lanes_sum<LANES>(s1) * ch.over_D;
            s2 = lanes_sum<LANES>(s2) * ch.over_D;
#pragma unroll
            for (int i = 0; i < MAXC; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) g[i][e] = fmaf(rstd, fmaf(-h[i][e], s2, d[i][e] - s1), g[i][e]);
        }
        if (t.p >= 0) {
            float rstd = 1.f, s1 = 0.f, s2 = 0.f;
            if constexpr (POST) rstd = ch.normalise(o, a.eps);
#pragma unroll
            for (int i = 0; i < MAXC; ++i) {
                float f[8];
                factors(1, i, f);
                if constexpr (WEIGHTS) {
                    add(integral_constant<int, V::GH>{}, i, g[i], o[i]);
                    if constexpr (POST) add(integral_constant<int, V::G>{}, i, g[i], ONES);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[i][e] = g[i][e] * f[e];
                    g[i][e] *= a.alpha;
                    if constexpr (POST) {
                        s1 += d[i][e];
                        s2 = fmaf(d[i][e], o[i][e], s2);
                    }
                }
            }
            if constexpr (POST) {
                s1 = lanes_sum<LANES>(s1) * ch.over_D;
                s2 = lanes_sum<LANES>(s2) * ch.over_D;
#pragma unroll
                for (int i = 0; i < MAXC; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[i][e] = rstd * fmaf(-o[i][e], s2, d[i][e] - s1);
            }
            ch.store(a.d_o + t.branch, d);
        }
        ch.store(a.dx + (long)t.row * a.chunks, g);
    }
    if constexpr (WEIGHTS) {
        // the waves' sums, a vector at a time: those in LDS, then those of the registers in their place
        float4 *const all = lds4 + 2 * VECTOR;
        float4 *const out = reinterpret_cast<float4 *>(a.parts) + ((long)blockIdx.y * gridDim.x + blockIdx.x) * V::NV * (2 * a.chunks);
        auto reduce = [&](int vector, int at, int pitch) {
            for (int k = threadIdx.x; k < VECTOR; k += 64 * BACK_WAVES) {
                const int c = (k & 63) + 64 * (k >> 7);
                if (c >= a.chunks || (k & 63) >= LANES) continue;
                float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < BACK_WAVES; ++w)
#pragma unroll
                    for (int g = 0; g < PARTS; ++g) {
                        const float4 t = all[w * pitch + at + k + g * LANES];
                        s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
                    }
                out[(long)vector * 2 * a.chunks + 2 * c + ((k >> 6) & 1)] = s;
            }
        };
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V::IN_LDS; ++v) reduce(v, v * VECTOR, V::IN_LDS * VECTOR);
#pragma unroll
        for (int v = 0; v < V::IN_REGISTERS; ++v) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < MAXC; ++i) {
                const float *f = regs[v][i];
                all[wave * VECTOR + i * 128 + lane] = make_float4(f[0], f[1], f[2], f[3]);
                all[wave * VECTOR + i * 128 + 64 + lane] = make_float4(f[4], f[5], f[6], f[7]);
            }
            __syncthreads();
            reduce(V::IN_LDS + v, 0, VECTOR);
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

// Sums over rows of parts, of the two vectors from `first` on and four columns: eight lanes with 16 bytes each, 32 slices of the rows, eight of them in a wave.  What slice 0 of wave 0 gets is whole.
template <int NV, int VECTORS>
__device__ __forceinline__ void sum_of_rows(const float4 *parts, int rows, int first, int quads, int quad, float4 (&s)[VECTORS])
{
    __shared__ float4 lds[3][VECTORS][8];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, c = lane & 7;
#pragma unroll
    for (int k = 0; k < VECTORS; ++k) s[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int r = threadIdx.x >> 3; r < rows; r += 32)
#pragma unroll
        for (int k = 0; k < VECTORS; ++k) s[k] = add4(s[k], parts[((long)r * NV + first + k) * quads + quad]);
    auto slices = [](float v) { v += rotate16<8>(v); return gemm_quad_sum(v); };
#pragma unroll
    for (int k = 0; k < VECTORS; ++k) {
        s[k] = make_float4(slices(s[k].x), slices(s[k].y), slices(s[k].z), slices(s[k].w));
        if (wave > 0 && lane < 8) lds[wave - 1][k][c] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < VECTORS; ++k)
#pragma unroll
        for (int w = 0; w < 3; ++w) s[k] = add4(s[k], lds[w][k][c]);
}

__device__ __forceinline__ void put4(float *to, int quad, const float4 &v) { if (to) reinterpret_cast<float4 *>(to)[quad] = v; }

// parts [groups][n][NV][D] -> the gradients, 32 columns a workgroup.  blockIdx.z 0: of the branch (vectors G h and G) in group blockIdx.y; of many groups the LayerNorm's, gate in them, go to
// `images` [groups][2][D] instead.  1: of the second LayerNorm, over all groups.
template <bool POST, bool PRE>
__global__ void __launch_bounds__(256)
residual_weight_sums_kernel(const float4 *__restrict__ parts, int n, WeightGrads w, float4 *images)
{
    using V = Sums<POST, PRE>;
    const int quads = w.D / 4, quad = blockIdx.x * 8 + (threadIdx.x & 7), at = min(quad, quads - 1), group = blockIdx.y;
    const bool whole = threadIdx.x < 8 && quad < quads;
    if constexpr (PRE) if (blockIdx.z == 1) {
        if (group != 0) return;
        float4 s[2];
        sum_of_rows<V::NV>(parts, n * gridDim.y, V::DYH, quads, at, s);
        if (whole) { put4(w.dpre_g, quad, s[0]); put4(w.dpre_b, quad, s[1]); }
        return;
    }
    float4 s[1 + POST];
    sum_of_rows<V::NV>(parts + (long)group * n * V::NV * quads, n, V::GH, quads, at, s);
    if (!whole) return;
    float4 d = s[0];
    if constexpr (POST) d = add4(mul4(reinterpret_cast<const float4 *>(w.post_g)[quad], s[0]), mul4(reinterpret_cast<const float4 *>(w.post_b)[quad], s[1]));
    put4(w.dgate ? w.dgate + (long)group * w.D : nullptr, quad, d);
    if constexpr (POST) {
        if (w.gate) {
            const float4 g = reinterpret_cast<const float4 *>(w.gate + (long)group * w.gate_stride)[quad];
            s[0] = mul4(s[0], g);
            s[1] = mul4(s[1], g);
        }
        if (gridDim.y == 1) { put4(w.dpost_g, quad, s[0]); put4(w.dpost_b, quad, s[1]); }
        else { images[(long)group * 2 * quads + quad] = s[0]; images[((long)group * 2 + 1) * quads + quad] = s[1]; }
    }
}

// images [groups][2][D] -> the sums over groups, as above
__global__ void __launch_bounds__(256)
residual_image_sums_kernel(const float4 *__restrict__ images, int groups, WeightGrads w)
{
    const int quads = w.D / 4, quad = blockIdx.x * 8 + (threadIdx.x & 7);
    float4 s[2];
    sum_of_rows<2>(images, groups, 0, quads, min(quad, quads - 1), s);
    if (threadIdx.x < 8 && quad < quads) { put4(w.dpost_g, quad, s[0]); put4(w.dpost_b, quad, s[1]); }
}

// Workgroups that a group of tokens is dealt to: no more than 256 over all groups, one to a CU, which holds one of rows above 512.  (Rounded up, 3, 5, 6 or 7 groups were 258 to 260, whose last few
// ran alone for as long as the others: 7 x 4096 x 2048, a gate of every image, 236 us and now 150, 7 x 4096 x 1280 124 and 84, 3 x 4096 x 1280 60 and 45.)  Of rows up to 512 a CU holds two: above
// 128 groups each has two workgroups (129 x 400 x 144 46 us, with one 55; 129 x 400 x 1024 168 with one, with two 201).
inline int backward_workgroups(long tokens, int groups, int maxc, int lanes)
{
    const int rows = back_waves(maxc) * (64 / lanes);
    const long most = groups >= 256 ? 1 : maxc == 1 && groups > 128 ? 2 : 256 / groups, need = (tokens + rows - 1) / rows;
    return (int)(need < most ? need : most);
}

template <int MAXC, int LANES, bool POST, bool PRE>
int launch_backward(const BackArgs &a, const WeightGrads &w, bool weights, int groups, hipStream_t st)
{
    const int n = backward_workgroups(a.tokens, groups, MAXC, LANES);
    const dim3 grid(n, groups);
    auto kern = weights ? residual_norm_backward_kernel<MAXC, LANES, POST, PRE, true> : residual_norm_backward_kernel<MAXC, LANES, POST, PRE, false>;
    const size_t lds = weights ? backward_lds<POST, PRE, true>(MAXC) : backward_lds<POST, PRE, false>(MAXC);
    // more than 64 KiB of LDS per workgroup needs the per-kernel opt-in (idempotent, host-side only)
    if (lds > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return SSAM_EHIP;
    hipLaunchKernelGGL(kern, grid, dim3(64 * back_waves(MAXC)), lds, st, a);
    SSAM_CHECK_LAUNCH();
    if (!weights) return SSAM_OK;
    float4 *images = reinterpret_cast<float4 *>(a.parts + (size_t)groups * n * Sums<POST, PRE>::NV * w.D);
    hipLaunchKernelGGL((residual_weight_sums_kernel<POST, PRE>), dim3(ssam_div_up(w.D, 32), groups, 1 + PRE), dim3(256), 0, st, (const float4 *)a.parts, n, w, images);
    SSAM_CHECK_LAUNCH();
    if (POST && groups > 1) {
        hipLaunchKernelGGL(residual_image_sums_kernel, dim3(ssam_div_up(w.D, 32)), dim3(256), 0, st, (const float4 *)images, groups, w);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int MAXC, int LANES>
int launch_backward(const BackArgs &a, const WeightGrads &w, bool post, bool pre, bool weights, int groups, hipStream_t st)
{
    auto go = post ? (pre ? launch_backward<MAXC, LANES, true, true> : launch_backward<MAXC, LANES, true, false>) : (pre ? launch_backward<MAXC, LANES, false, true> : launch_backward<MAXC, LANES, false, false>);
    return go(a, w, weights, groups, st);
}

// ---------------------------------------------------------------- rows in 8 bits
// One wave, or part of one, per row: its largest magnitude, then its codes.  Bound by HBM: 32768 x 1280 20 us (6.3 TB/s), 13104 x 5120 35 (5.7).  Rows of up to 64 * 8 * MAXC features stay in registers in between; MAXC = 0: longer ones are read twice.
template <int MAXC, int LANES>
__global__ void __launch_bounds__(256)
quantize_rows_kernel(const uint4 *__restrict__ x, uint2 *__restrict__ codes, float *__restrict__ scales, long rows, int chunks)
{
    const long row = (long)blockIdx.x * (WAVES * 64 / LANES) + threadIdx.x / LANES;
    const int lane = threadIdx.x & (LANES - 1);
    if (row >= rows) return;
    x += row * chunks;
    codes += row * chunks;
    uint4 v[MAXC ? MAXC : 1];
    uint32_t top = 0;
    if constexpr (MAXC != 0) {
#pragma unroll
        for (int i = 0; i < MAXC; ++i) v[i] = x[min(lane + LANES * i, chunks - 1)];
#pragma unroll
        for (int i = 0; i < MAXC; ++i) top = max_u16x2(top, top_of_bf16x8(v[i]));
    } else {
        for (int c = lane; c < chunks; c += LANES) top = max_u16x2(top, top_of_bf16x8(x[c]));
    }
    top = lanes_max<LANES>(max(top >> 16, top & 0xffffu));
    const bool finite = top < 0x7f80u;
    const RowScale s = row_scale(finite ? bf16_bits_to_float(top) : 0.f);
    auto put = [&](int c, const uint4 &r) {
        float f[8];
        unpack_bf16x8(r, f);
        put8(codes + c, finite ? codes_of(f, s.inv) : make_uint2(0, 0));
    };
    if constexpr (MAXC != 0) {
#pragma unroll
        for (int i = 0; i < MAXC; ++i)
            if (lane + LANES * i < chunks) put(lane + LANES * i, v[i]);
    } else {
        for (int c = lane; c < chunks; c += LANES) put(c, x[c]);
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
    const StepArgs a = { (const uint4 *)x, (uint4 *)x_out, (const uint4 *)o, rows, post_g, post_b, gate, pre_g, pre_b, gate_stride, alpha, eps, y, scales, 0, B * N, N, D / 8 };
    return by_width(D / 8, [&](auto maxc, auto lanes) { return launch_step<decltype(maxc)::value, decltype(lanes)::value>(a, post_g != nullptr, out, (hipStream_t)stream); });
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
    if (D % 16 != 0 || D >= 131072 || rows >= 1L << 40) return SSAM_EUNSUPPORTED;
    const int chunks = D / 8;
    auto go = [&](auto maxc, auto lanes) -> int {
        constexpr int MAXC = decltype(maxc)::value, LANES = decltype(lanes)::value, ROWS = WAVES * 64 / LANES;
        for (long first = 0; first < rows; first += MOST_WORKGROUPS * ROWS) {
            const long left = (rows - first + ROWS - 1) / ROWS;
            hipLaunchKernelGGL((quantize_rows_kernel<MAXC, LANES>), dim3((unsigned)(left < MOST_WORKGROUPS ? left : MOST_WORKGROUPS)), dim3(64 * WAVES), 0, (hipStream_t)stream,
                               (const uint4 *)x + first * chunks, (uint2 *)codes + first * chunks, scales + first, rows - first, chunks);
            SSAM_CHECK_LAUNCH();
        }
        return SSAM_OK;
    };
    if (chunks <= 256) return by_width(chunks, go);
    if (chunks <= 640) return go(std::integral_constant<int, 10>{}, std::integral_constant<int, 64>{});
    return go(std::integral_constant<int, 0>{}, std::integral_constant<int, 64>{});
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
    if (B <= 0 || N <= 0 || D <= 0 || D > 2048 || (gate_images != 1 && gate_images != B)) return 0;
    const int n = by_width(ssam_div_up(D, 8), [&](auto maxc, auto lanes) { return backward_workgroups(gate_images == 1 ? (long)B * N : N, gate_images, maxc, lanes); });
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
    if (groups > 65535) return SSAM_EUNSUPPORTED;                      // gridDim.y
    if (weights) {
        if (!workspace || !ssam_aligned16(workspace)) return SSAM_EINVAL;
        if (workspace_bytes < ssam_residual_norm_backward_workspace_bytes(B, N, D, groups)) return SSAM_EWORKSPACE;
    }
    const TokenRows rows = { src, dst, src_batch_stride, dst_batch_stride, o ? No : 0, pre_g ? Ny : 0 };
    const BackArgs a = { (const uint4 *)x_out, (const uint4 *)o, (const uint4 *)dy, (const uint4 *)dx_out, (uint4 *)dx, (uint4 *)d_o, rows, post_g, gate, pre_g,
                         gate_batch_stride, alpha, eps, (float *)workspace, groups > 1 ? N : B * N, N, D / 8 };
    const WeightGrads w = { post_g, post_b, gate, gate_batch_stride, dgate, dpost_g, dpost_b, dpre_g, dpre_b, D };
    return by_width(D / 8, [&](auto maxc, auto lanes) {
        return launch_backward<decltype(maxc)::value, decltype(lanes)::value>(a, w, post_g != nullptr, pre_g != nullptr, weights, groups, (hipStream_t)stream);
    });
}
