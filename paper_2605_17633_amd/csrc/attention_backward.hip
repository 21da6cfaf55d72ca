// Gradients of Stripe-Sort attention (App. A.1, Alg. 1) for gfx950, of q, k, v and of both relative-position tables.
//
// With L_ij = scale q_i.k_j + BH[i][row_j] + BW[i][col_j] over the active tiles of the A-shape mask, P = softmax(L), O = P V and
// BH[i][y] = q_i . rel_h[row_i - y + w - 1] (BW likewise):
//   delta_i = dO_i . O_i,   dS = P * (dO V^T - delta),   dV = P^T dO,   dK = scale dS^T Q,
//   GH[i][y] = sum of dS_ij over the keys j of row y (GW likewise, of column x),
//   dQ_i = scale sum_j dS_ij k_j + sum_y GH[i][y] rel_h[row_i - y + w - 1] + ...,   drel_h[t] = sum_i GH[i][row_i + w - 1 - t] q_i.
// The probabilities are formed again; nothing but the forward's result is needed of it.
//
// No atomics, so results are the same every time; that takes two walks over the active tiles and a third launch:
//   rows     a wave owns 32 queries and walks their keys as the forward does (scores transposed, a query a lane, running maximum); leaves
//            dQ, -log sum exp and delta of its queries, their bias entries and GH, GW (fp16)
//   columns  a wave owns 32 keys and walks their queries: P from the statistics, dK and dV stay in registers
//   tables   drel = (G at relative positions)^T Q, a product over all queries of all groups and heads, in slices that are added up in order
//
// Groups of at most 224 tokens have a kernel of their own (attention_backward_window.h).
//
// 64 x 64, density 0.4 in position order: 16 heads of 64, one image 208 us, 16 heads of 80, four images 876: 0.34 and 0.41 PFLOP/s of the five products that a gradient cannot do
// without, of 1.16 that a large product reaches.  28 x 28, 12 heads of 64: 78 us; 50 x 50, content order, two images, 12 heads of 64: 191; 128 x 128, density 0.1, 16 heads of 64: 1665, in
// content order 2014 (one wave to a SIMD).  Under the tracer, where launches take longer (239 and 937 us together), rows are 116 and 492, columns 90 and 368, tables with their sums 22 and 73, the
// join 6.  Of a walk's time the matrix pipe is busy a quarter (rows) to two fifths (columns), the vector unit and LDS over a third each, one after the other: two waves to a SIMD,
// of which one could fill the other's gaps, wait 36 % of the time.
//
// The bias and its gradient are products with the 0/1 matrix E that has a one at every key's row and one at its column: scores
// take E T (T the entries of a query, fp16, over the scale), G is E^T dS.  E sits behind the keys' features in LDS, [key][K | E], so that one set
// of transposing reads gives K^T and E^T.  Its ones are 0x3c00: 1 in fp16, 2^-7 in bf16, which G is multiplied by at the end (in windows 2^n and 2^(8 n - 7)).
// Operand layouts of v_mfma_f32_32x32x16 and of the transposing read are those of the forward kernels.
#include "common.h"

namespace {

constexpr float LOG2E = 1.4426950408889634f;
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

struct BwdParams {
    const bf16 *q, *k, *v;
    long row_stride;
    const bf16 *rel_h, *rel_w;
    const int32_t *sigma;
    long sigma_stride;
    const bf16 *out, *dout;
    const int32_t *out_rows;
    bf16 *dq, *dk, *dv;
    long grad_stride;
    int S, w, h, n_gh;
    uint32_t per_w;              // 2^22 / w rounded up: a cell below 2^14 times it, over 2^22, is its row (the error, a cell / 2^22, is below 1 / w)
    int mask_block, n_pre;       // tile of the mask (grids: 128), tiles of the dense prefix
    float scale, scale_log2e, inv_scale, inv_scale_log2e;        // inv_scale: what turns a bias into an entry, 1 / (scale * 2^n); n = 0 on grids
    uint32_t one;                // windows: 2^n in fp16, the ones of E
    float over_one;              // and 1 over what that is as bf16, 2^(8 n - 7)
    _Float16 *tab;               // [gh][SP][EW]: bias entries of a query, over the scale
    _Float16 *gsum;              // [gh][S][EW]: GH | GW over gunit; NULL: not wanted
    // of every order (one, or one a group; see backward_prepare_kernel)
    uint4 *e;                    // [order][SP][bytes of E]
    uint32_t *blocks;            // [order][SP / 32]: the two slices of a block of keys, 0 if there are more
    int32_t *inverse;            // [order][S]: position of a cell
    float *gunit;                // [gh][S]: a power of two
    float *lse, *delta;          // [gh][SP]: -log sum exp over the scale, -delta
    const uint4 *zeros;          // 1 KB of them
    int SP;                      // S in whole 32s: rows of tab, lse and delta
};

// NT: 32 entries of E each; half of them rows, half columns
template <int D, int NT>
struct BwdCfg {
    static constexpr int EW = 32 * NT, WK = EW / 2;
    static constexpr int KS = D / 16;                        // k-steps of a product over features
    static constexpr int ES = EW / 16;                       // and over entries
    static constexpr int DT = (D + 31) / 32;                 // 32-row tiles of dK^T, dV^T
    static constexpr int VP = D + 8;                         // LDS pitches (elements): odd in 16-byte units
    static constexpr int RP = 2 * WK + 8;                    // of G at relative positions, one table
    static constexpr int UP = 4 * WK + 8;                    // of products with a table at the entries' places
};

// row | column << 16 of a position's cell (positions past the end: the last one's; cells are held to the grid)
__device__ __forceinline__ int row_col(const int32_t *sigma, int at, const BwdParams &P)
{
    const int cell = min(max(sigma[min(at, P.S - 1)], 0), P.S - 1);
    const int row = (int)((uint32_t)cell * P.per_w >> 22);
    return row | (cell - row * P.w) << 16;
}

// MFMA passes done before results are read under predicates (see the forward kernels)
__device__ __forceinline__ void mfma_settle()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ f32x16 zero16()
{
    return f32x16{ 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
}

// Operand a of step t over 16 rows of an LDS block: lane <-> column 32 * tile + (lane & 31) of rows 16 t + 8 (e / 4) + 4 half + (e & 3), the order in
// which a 32x32 result holds them.  Columns past `last` re-read that quad; what they give is not used.
__device__ __forceinline__ bf16x8 transposed(const bf16 *block, int pitch, int t, int tile, int last, int lane = threadIdx.x & 63)
{
    const int li = lane & 15;
    int col = tile * 32 + 16 * ((lane >> 4) & 1) + 4 * (li & 3);
    if (tile * 32 + 28 > last) col = min(col, last);         // (known at compile time: the others' addresses differ by constants)
    const bf16 *p = block + (16 * t + 4 * (lane >> 5) + (li >> 2)) * pitch + col;
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(p));
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(p + 8 * pitch));
    return bf16x8{ a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
}

__device__ __forceinline__ bf16x8 half_of(const f32x16 &s, int t)
{
    bf16x8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (bf16)s[8 * t + e];
    return p;
}

// The lane, not known from before: what follows from it is worked out where it is used instead of kept in registers through a walk.
__device__ __forceinline__ int lane_now()
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
}
// the other half-wave's value
__device__ __forceinline__ float other_half(float x)
{
    return __int_as_float(__builtin_amdgcn_ds_bpermute((lane_now() ^ 32) * 4, __float_as_int(x)));
}

// 32 rows held as [column tiles]^T results -> bf16 rows in memory, through the wave's LDS: whole rows of 16-byte stores.  row < 0: not stored.
// (`row` is the row of lane & 31; scratch: 32 x (D + 8) elements)
template <int D>
__device__ __forceinline__ void store_rows(const f32x16 *acc, bf16 *scratch, bf16 *base, long stride, int row)
{
    const int lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    wave_lds_fence();
#pragma unroll
    for (int dt = 0; dt < (D + 31) / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (dt * 32 + 8 * g >= D) continue;
            bf16x4 v = { (bf16)acc[dt][4 * g], (bf16)acc[dt][4 * g + 1], (bf16)acc[dt][4 * g + 2], (bf16)acc[dt][4 * g + 3] };
            *reinterpret_cast<bf16x4 *>(scratch + l32 * (D + 8) + dt * 32 + 8 * g + 4 * half) = v;
        }
    wave_lds_fence();
    constexpr int CH = D / 8;
#pragma unroll
    for (int i = lane; i < 32 * CH; i += 64) {
        const int r = i / CH, c = i - r * CH, at = __shfl(row, r, 64);
        if (at >= 0) *reinterpret_cast<uint4 *>(base + (long)at * stride + c * 8) = *reinterpret_cast<const uint4 *>(scratch + r * (D + 8) + c * 8);
    }
}

// Rows that go from memory straight into LDS lie there without padding; chunk c (16 bytes) of row r sits at place c ^ swizzle(r), so that 16 rows read at
// one chunk touch all banks, and so do the 64 bytes each of 8 rows that a transposing read takes.
template <int CHUNKS>
__device__ __forceinline__ int swizzle(int row)
{
    if (CHUNKS >= 16) return (row & 1) << 3 | (row & 2) << 1 | (row & 4) >> 1 | (row & 8) >> 3;
    if (CHUNKS == 8) return (row & 2) << 1 | (row & 4) >> 1 | (row & 8) >> 3;
    if (CHUNKS == 4) return (row & 4) >> 1 | (row & 8) >> 3;
    return (row >> 3) & 1;
}

// 16 bytes a lane from memory to LDS at lds + 16 * lane.  The compiler does not see the request: the caller waits for it (vmcnt).
__device__ __forceinline__ void request(uint32_t lds, uint32_t off, const void *from)
{
    // (uniform, and kept in scalar registers: the compiler does not always do so for an operand of assembly)
    const uint64_t f = reinterpret_cast<uint64_t>(from), base = (uint64_t)__builtin_amdgcn_readfirstlane((uint32_t)(f >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)f);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void request(uint32_t lds, const void *src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src) : "m0", "memory");
}

// Transposed operand of rows that lie so: columns 32 * tile + .. of 16 rows at `t`, in the order in which a 32x32 result holds them (operand a of step t).
template <int CHUNKS>
struct Transposed {
    static constexpr int PITCH = CHUNKS * 16;
    static constexpr int KINDS = CHUNKS == 8 ? 2 : 1;         // (rows of 16 chunks and more: the place of another tile is the first one's with bits changed)
    int at[KINDS][2], again;
    __device__ __forceinline__ Transposed(int lane = threadIdx.x & 63)
    {
        again = ((lane >> 4) & 1) * 32;
        const int li = lane & 15;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = 8 * u + 4 * (lane >> 5) + (li >> 2), f0 = (CHUNKS == 2 ? 0 : 16 * ((lane >> 4) & 1)) + 4 * (li & 3);
#pragma unroll
            for (int k = 0; k < KINDS; ++k) at[k][u] = r * PITCH + ((4 * k + (f0 >> 3)) ^ swizzle<CHUNKS>(r)) * 16 + (f0 & 7) * 2;
        }
    }
    // place of quad u of a tile that is known only when the kernel runs
    __device__ __forceinline__ int place(int u, int tile) const
    {
        if (CHUNKS == 10) return at[0][u] + tile * 64 - (tile == 2 ? again : 0);
        if (CHUNKS == 8) return at[0][u] ^ ((at[0][u] ^ at[KINDS - 1][u]) & -(tile & 1));
        return at[0][u];
    }
    // base: byte offset of the block in LDS.  (Of a last tile that the rows fill by half, 10 chunks, the other half is the same columns again.)
    __device__ __forceinline__ bf16x8 operator()(const unsigned char *smem, int base, int t, int tile) const
    {
        bf16x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            int a = CHUNKS >= 16 ? (at[0][u] ^ (tile & 3) * 64) + base + 16 * t * PITCH + tile / 4 * 256
                                 : at[tile % KINDS][u] + base + 16 * t * PITCH + tile / KINDS * KINDS * 64;
            if (CHUNKS == 10 && tile == 2) a -= again;
            v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(smem + a));
        }
        return bf16x8{ v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3] };
    }
};

// Operand a or b of step ks over features: 16 bytes of row l32 of a block.
template <int CHUNKS>
struct Straight {
    static constexpr bool LINE = CHUNKS == 2 || CHUNKS == 10;   // the swizzle changes places by twos: those of a step are 32 bytes from the last one's
    int at[LINE ? 1 : CHUNKS / 2];
    __device__ __forceinline__ Straight(int lane = threadIdx.x & 63)
    {
        const int l32 = lane & 31;
#pragma unroll
        for (int ks = 0; ks < (LINE ? 1 : CHUNKS / 2); ++ks) at[ks] = l32 * CHUNKS * 16 + ((2 * ks + (lane >> 5)) ^ swizzle<CHUNKS>(l32)) * 16;
    }
    __device__ __forceinline__ bf16x8 operator()(const unsigned char *smem, int base, int ks) const
    {
        return *reinterpret_cast<const bf16x8 *>(smem + base + (LINE ? at[0] + 32 * ks : at[LINE ? 0 : ks]));
    }
};

// Bias entries past the range of fp16 (infinities by the conversion) are bounded to it: with an infinity the zeros of E would make NaNs of a query's whole row.  NaN stays NaN.  (The mode
// bit that clamps conversions, which the forward's kernels set, is no choice here: with it the matrix instructions take NaN for 0 and infinities for the largest number, so that a
// gradient that is not finite would come back as an ordinary one.)
__device__ __forceinline__ f16x8 bounded(f16x8 v)
{
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(v, (f16x8)(_Float16)-65504.f), (f16x8)(_Float16)65504.f);
}

// entries of a slice of 16, the eight of a half-wave: a one (of fp16) at place i, if that is one of them
__device__ __forceinline__ f16x8 ones(int i, uint32_t one = 0x3c00u)
{
    u32x4 e;
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = i >> 1 == j ? (i & 1 ? one << 16 : one) : 0u;
    return __builtin_bit_cast(f16x8, e);
}

// ---------------------------------------------------------------- what the order alone decides
// E of every key as the row kernel's stages take it, the slices of a block of 32 keys (row | column << 8 | 1 << 16, or 0), the inverse of the order.  A wave a block.
template <int NT, bool LOCAL>
__global__ void __launch_bounds__(256)
backward_prepare_kernel(BwdParams P, int blocks, int total)
{
    constexpr int WK = 16 * NT, EC = LOCAL ? 4 : 4 * NT;
    const int unit = (int)blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    if (blockIdx.x == 0 && threadIdx.x < 64) const_cast<uint4 *>(P.zeros)[threadIdx.x] = make_uint4(0, 0, 0, 0);
    if (unit >= total) return;
    const int order = unit / blocks, at = (unit - order * blocks) * 32 + l32;
    const int rc = row_col(P.sigma + (long)order * P.sigma_stride, at, P), row = rc & 0xffff, col = rc >> 16;
    uint4 *to = P.e + ((long)order * P.SP + at) * EC;
    if constexpr (LOCAL) {
#pragma unroll
        for (int c = 0; c < 2; ++c) to[2 * half + c] = __builtin_bit_cast(uint4, ones(((half ? col : row) & 15) - 8 * c));
    } else {
#pragma unroll
        for (int c = 0; c < EC / 2; ++c) to[half * EC / 2 + c] = __builtin_bit_cast(uint4, ones((half ? col : row) - 8 * c));
    }
    static_assert(LOCAL || EC / 2 * 8 == WK, "");
    const int rs = __builtin_amdgcn_readfirstlane(row >> 4), cs = __builtin_amdgcn_readfirstlane(col >> 4);
    const bool two = __builtin_amdgcn_ballot_w64(row >> 4 != rs || col >> 4 != cs) == 0;
    if (lane == 0) P.blocks[unit] = two ? (uint32_t)rs | (uint32_t)cs << 8 | 1u << 16 : 0u;
    if (half == 0 && at < P.S) P.inverse[(long)order * P.S + row * P.w + col] = at;
}

// ---------------------------------------------------------------- rows
// Stages of a row walk, two buffers of them in LDS: K, V and E, straight from memory.
// LOCAL: of a key E holds the one of its row's slice of 16 entries and that of its column's, 64 keys a stage.  A block of 32 keys whose cells lie in one slice each
// (every one of the position-only order on a grid of a power of two) takes two bias products and one G product; in others every slice that occurs takes one, the other keys
// masked.  Otherwise E is whole, 32 keys a stage, and all entries are multiplied: for orders that scatter a block's cells over the grid.
template <int D, int NT, bool LOCAL>
struct RowStage {
    using C = BwdCfg<D, NT>;
    static constexpr bool FULL = D == 80 && (NT == 2 || NT == 4);         // registers and LDS are short: dO in LDS, for which the stages are halved
    static constexpr int KEYS = LOCAL && !FULL ? 64 : 32;
    static constexpr int KP = D * 2, EP = LOCAL ? 64 : C::EW * 2, TP = C::EW * 2;   // rows, in bytes
    static constexpr int K = 0, V = K + KEYS * KP, E = V + KEYS * KP, BYTES = E + KEYS * EP;
    static constexpr int T = 2 * BYTES, O = T + 4 * 32 * TP;
    static constexpr bool KEEP = NT < 8 && !(LOCAL && FULL);  // a wave's dO stays in registers, else in LDS
    static constexpr int TOTAL = O + (KEEP ? 0 : 4 * 32 * C::VP * 2);
    static_assert(2 * BYTES <= 64 * 1024, "requests reach the first 64 KB");
};

template <int D, int NT, bool LOCAL>
__host__ __device__ constexpr size_t rows_lds_bytes(int nrel)
{
    using C = BwdCfg<D, NT>;
    const size_t stage = RowStage<D, NT, LOCAL>::TOTAL, products = (size_t)4 * 32 * C::UP * 2;
    const size_t end = (size_t)C::WK * 2 + (size_t)4 * 32 * C::RP * 2 + (size_t)(nrel + 15) / 16 * 16 * C::VP * 2;
    const size_t rows = (size_t)4 * 32 * C::VP * 2;
    size_t m = end > stage ? end : stage;
    m = products > m ? products : m;
    return rows > m ? rows : m;
}

template <int D, int NT, bool LOCAL>
__global__ void __launch_bounds__(256, NT < 8 ? 2 : 1)
backward_rows_kernel(BwdParams P, int tiles)
{
    using C = BwdCfg<D, NT>;
    using St = RowStage<D, NT, LOCAL>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // the tiles of one (group, head) run on one XCD (workgroup b sits on XCD b & 7), whose L2 then serves the re-reads of its K and V
    const int tile = (blockIdx.x >> 3) % tiles, gh = ((blockIdx.x >> 3) / tiles) * 8 + (blockIdx.x & 7);
    if (gh >= P.n_gh) return;
    const int grp = gh / P.h, head = gh - grp * P.h;
    const int S = P.S, w = P.w, nrel = 2 * w - 1;
    const int q0 = tile * 128, qpos = q0 + wave * 32 + l32;
    const int order = P.sigma_stride ? grp : 0;
    const int32_t *sigma = P.sigma + (long)grp * P.sigma_stride;

    // this lane's query: its features, dO and delta
    bf16x8 qf[C::KS], of[C::KS];
    float delta = 0.f;
    int qrc = 0;                                             // row | column << 16 of the query's cell
    {
        int orow = -1;
        if (qpos < S) {
            const long slot = (long)grp * S + qpos;
            qrc = row_col(sigma, qpos, P);
            orow = P.out_rows ? P.out_rows[slot] : 0;
            const long at = (P.out_rows ? (long)orow : slot) * ((long)P.h * D) + (long)head * D + half * 8;
            if (orow >= 0) {
                const bf16 *qp = P.q + slot * P.row_stride + (long)head * D + half * 8;
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    qf[ks] = *reinterpret_cast<const bf16x8 *>(qp + ks * 16);
                    of[ks] = *reinterpret_cast<const bf16x8 *>(P.dout + at + ks * 16);
                    const bf16x8 o = *reinterpret_cast<const bf16x8 *>(P.out + at + ks * 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) delta = fmaf((float)of[ks][e], (float)o[e], delta);
                }
            }
        }
        if (orow < 0) {                                      // past the end, or its output is dropped: no gradient comes from it
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[ks][e] = of[ks][e] = (bf16)0.f;
        }
    }
    delta += __shfl_xor(delta, 32, 64);

    // Bias entries over the scale: rel Q^T, relative position t of the lane's query is its entry at_q + w - 1 - t.  All of a product's are stored, those below 0 and from w on
    // at places of their own in a row that is long enough (no predicates: a store behind one costs ten instructions), and the entries read back from where they lie for every query.
    f16x8 bt[C::ES];
    {
        _Float16 *u_row = reinterpret_cast<_Float16 *>(smem) + (wave * 32 + l32) * C::UP;
        constexpr int FIRST = 2 * C::WK;                     // the place of entry 0
        bf16x8 ahead[C::KS];                                 // rows of the next product: asked for a product earlier
        auto rows = [&](int tab, int m0) __attribute__((always_inline)) {
            const bf16 *rp = (tab ? P.rel_w : P.rel_h) + (long)min(m0 + l32, nrel - 1) * D + half * 8;
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) ahead[ks] = *reinterpret_cast<const bf16x8 *>(rp + ks * 16);
        };
        rows(0, 0);
#pragma unroll
        for (int tab = 0; tab < 2; ++tab) {
            wave_lds_fence();
            _Float16 *to = u_row + (FIRST + w - 1 + (tab ? qrc >> 16 : qrc & 0xffff) - 4 * half);
            for (int m0 = 0; m0 < nrel; m0 += 32, to -= 32) {
                f32x16 u = zero16();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ahead[ks], qf[ks], u, 0, 0, 0);
                const bool more = m0 + 32 < nrel;
                rows(more ? tab : 1, more ? m0 + 32 : 0);
                mfma_settle();
#pragma unroll
                for (int r = 0; r < 16; ++r) to[-8 * (r >> 2) - (r & 3)] = (_Float16)(u[r] * P.inv_scale);
            }
            wave_lds_fence();
#pragma unroll
            for (int c = 0; c < C::ES / 2; ++c) {            // entries 16 c + 8 half .. + 7; those from w on are zeros
                f16x8 v = *reinterpret_cast<const f16x8 *>(u_row + FIRST + 16 * c + 8 * half);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 16 * c + 8 * half + e < w ? v[e] : (_Float16)0.f;
                bt[tab * C::ES / 2 + c] = bounded(v);
            }
        }
    }
    if (qpos < P.SP) {
        _Float16 *to = P.tab + ((long)gh * P.SP + qpos) * C::EW + 8 * half;
#pragma unroll
        for (int c = 0; c < C::ES; ++c) *reinterpret_cast<f16x8 *>(to + 16 * c) = bt[c];
    }
    __syncthreads();
    const int tsw = swizzle<C::EW / 8>(l32);
    unsigned char *tl = smem + St::T + (wave * 32 + l32) * St::TP;
#pragma unroll
    for (int c = 0; c < C::ES; ++c) *reinterpret_cast<f16x8 *>(tl + ((2 * c + half) ^ tsw) * 16) = bt[c];

    bf16 *os = reinterpret_cast<bf16 *>(smem + St::O) + (wave * 32 + l32) * C::VP + half * 8;
    if constexpr (!St::KEEP)
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) *reinterpret_cast<bf16x8 *>(os + ks * 16) = of[ks];
    auto upstream = [&](int ks) { return St::KEEP ? of[ks] : *reinterpret_cast<const bf16x8 *>(os + ks * 16); };

    // stages of keys: the dense prefix, then (where a wave has a diagonal tile behind it) the workgroup's own 128
    // (A mask tile is 128 here.  Written as the constant, so that the division goes, 64 features on 32 x 32 and 80 on grids up to 64 x 64 in scattering orders spill two registers and one.)
    const int pre = min(P.n_pre * P.mask_block, S), pre_stages = (pre + St::KEYS - 1) / St::KEYS;
    const int own = (q0 + wave * 32) / P.mask_block;                                  // mask tile of the wave's queries
    const bool any_diagonal = min(q0 + 127, S - 1) / P.mask_block >= P.n_pre;
    const int stages = pre_stages + (any_diagonal ? (min(128, S - q0) + St::KEYS - 1) / St::KEYS : 0);
    const bool alive = q0 + wave * 32 < S;
    auto stage_key = [&](int s) { return s < pre_stages ? s * St::KEYS : q0 + (s - pre_stages) * St::KEYS; };

    constexpr int CH = D / 8, NI = St::KEYS * CH / 64, NQ = (NI + 3) / 4, EC = St::EP / 16, EI = St::KEYS * EC / 64, NE = (EI + 3) / 4;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)smem);
    const bf16 *kbase = P.k + (long)grp * S * P.row_stride + (long)head * D, *vbase = P.v + (long)grp * S * P.row_stride + (long)head * D;
    const uint4 *ebase = P.e + (long)order * P.SP * EC;
    auto load = [&](int s) {
        int ln = lane;
        if (D == 80) asm volatile("" : "+v"(ln));            // places are worked out again at every stage: kept, they would take registers that are short
        const int key0 = stage_key(s);
        const uint32_t to = lds0 + (s & 1) * St::BYTES;
        const unsigned char *ks = reinterpret_cast<const unsigned char *>(kbase) + (long)key0 * P.row_stride * 2, *vs = reinterpret_cast<const unsigned char *>(vbase) + (long)key0 * P.row_stride * 2;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int j = wave + 4 * i;
            if (j >= NI) continue;
            const int at = j * 64 + ln, r = at / CH, c = at % CH ^ swizzle<CH>(r);
            const uint32_t off = r * (uint32_t)P.row_stride * 2 + c * 16;
            if (key0 + St::KEYS <= S) {
                request(to + St::K + j * 1024, off, ks);
                request(to + St::V + j * 1024, off, vs);
            } else {                                         // keys past the end are zeros
                const bool in = key0 + r < S;
                request(to + St::K + j * 1024, in ? ks + off : (const void *)P.zeros);
                request(to + St::V + j * 1024, in ? vs + off : (const void *)P.zeros);
            }
        }
        // (rows of E from SP on are another order's, or what follows them: blocks past the end are left out)
#pragma unroll
        for (int i = 0; i < NE; ++i) {
            const int j = wave + 4 * i;
            if (j >= EI) continue;
            const int at = j * 64 + ln, r = at / EC, c = at % EC ^ swizzle<EC>(r);
            request(to + St::E + j * 1024, (uint32_t)(r * EC + c) * 16, ebase + (long)key0 * EC);
        }
    };
    const uint32_t *blocks = P.blocks + (long)order * (P.SP / 32);

    const Transposed<CH> kt;
    const Transposed<EC> et;
    const Straight<CH> ka;
    const int esw = swizzle<EC>(l32);

    f32x16 acc[C::DT], gt[LOCAL ? 1 : NT];
    float g[LOCAL ? C::ES : 1][8];
#pragma unroll
    for (int t = 0; t < C::DT; ++t) acc[t] = zero16();
#pragma unroll
    for (int t = 0; t < (LOCAL ? 1 : NT); ++t) gt[t] = zero16();
#pragma unroll
    for (int s = 0; s < (LOCAL ? C::ES : 1); ++s)
#pragma unroll
        for (int r = 0; r < 8; ++r) g[s][r] = 0.f;
    float m = -INFINITY, l = 0.f;
    // a block's slices are asked for a stage ahead: read where they are used they cost a trip to the cache a block
    uint32_t ahead[St::KEYS / 32];
    auto look = [&](int s) __attribute__((always_inline)) {
        if constexpr (LOCAL && C::ES > 2)
#pragma unroll
            for (int b = 0; b < St::KEYS / 32; ++b) ahead[b] = blocks[min(stage_key(s) / 32 + b, P.SP / 32 - 1)];
    };
    __syncthreads();
    load(0);
    look(0);
    for (int s = 0; s < stages; ++s) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        uint32_t now[St::KEYS / 32] = {};
        if constexpr (LOCAL && C::ES > 2)
#pragma unroll
            for (int b = 0; b < St::KEYS / 32; ++b) now[b] = __builtin_amdgcn_readfirstlane(ahead[b]);
        LDS_BARRIER();                                       // this stage has landed, and nobody reads the other buffers any more
        if (s + 1 < stages) {
            load(s + 1);
            look(s + 1);
        }
        const int key0 = stage_key(s);
#pragma unroll 1
        for (int b = 0; b < St::KEYS / 32; ++b) {
            const int kb = key0 + 32 * b;
            const bool active = alive && kb < S && (s < pre_stages ? kb < pre : own >= P.n_pre && kb / P.mask_block == own);
            if (!active) continue;                           // the same for the whole wave
            const int at = (s & 1) * St::BYTES + 32 * b * St::KP, eat = (s & 1) * St::BYTES + St::E + 32 * b * St::EP;
            const unsigned char *el = smem + eat + l32 * St::EP;
            f32x16 sc = zero16();
            int rs = 0, cs = 0, rc = 0;
            bool two = true;
            if constexpr (LOCAL && C::ES > 2) {
                const uint32_t slices = b == 0 ? now[0] : now[St::KEYS / 32 - 1];
                two = slices != 0;
                rs = slices & 0xff;
                cs = slices >> 8 & 0xff;
                if (!two) rc = row_col(sigma, kb + l32, P);
            }
            if constexpr (LOCAL) {
                const f16x8 er = *reinterpret_cast<const f16x8 *>(el + (half ^ esw) * 16), ec = *reinterpret_cast<const f16x8 *>(el + ((2 + half) ^ esw) * 16);
                if (two) {
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(er, *reinterpret_cast<const f16x8 *>(tl + ((2 * rs + half) ^ tsw) * 16), sc, 0, 0, 0);
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ec, *reinterpret_cast<const f16x8 *>(tl + ((2 * cs + C::WK / 8 + half) ^ tsw) * 16), sc, 0, 0, 0);
                } else {
                    const f16x8 none = { 0, 0, 0, 0, 0, 0, 0, 0 };
#pragma unroll 1
                    for (int i = 0; i < C::ES; ++i) {
                        const bool is_row = i < C::ES / 2, mine = (is_row ? rc >> 4 & 15 : (rc >> 20) + C::ES / 2) == i;
                        if (__builtin_amdgcn_ballot_w64(mine) == 0) continue;
                        sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(mine ? (is_row ? er : ec) : none, *reinterpret_cast<const f16x8 *>(tl + ((2 * i + half) ^ tsw) * 16), sc, 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < C::ES; ++c)
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(el + ((2 * c + half) ^ esw) * 16), *reinterpret_cast<const f16x8 *>(tl + ((2 * c + half) ^ tsw) * 16), sc, 0, 0, 0);
            }
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka(smem, at + St::K, ks), qf[ks], sc, 0, 0, 0);
            f32x16 dp = zero16();
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka(smem, at + St::V, ks), upstream(ks), dp, 0, 0, 0);
            float mx = -INFINITY;
            if (kb + 32 > S)
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[r] = kb + 8 * (r >> 2) + 4 * half + (r & 3) < S ? sc[r] : -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * P.scale_log2e;
            // the reference moves only when it is exceeded by a factor of 2^8: what the sums are in units of cancels at the end
            const bool move = mx > m + 8.f;
            if (__builtin_amdgcn_ballot_w64(move) != 0) {
                const float to = move ? mx : m, alpha = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= alpha;
#pragma unroll
                for (int t = 0; t < C::DT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
                if constexpr (LOCAL && C::ES > 2) {
#pragma unroll
                    for (int i = 0; i < C::ES; ++i)
#pragma unroll
                        for (int r = 0; r < 8; ++r) g[i][r] *= alpha;
                } else {
#pragma unroll
                    for (int t = 0; t < (LOCAL ? 1 : NT); ++t)
#pragma unroll
                        for (int r = 0; r < 16; ++r) gt[t][r] *= alpha;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[r], P.scale_log2e, -m));
                l += p;
                dp[r] = p * (dp[r] - delta);
            }
            const bf16x8 ds[2] = { half_of(dp, 0), half_of(dp, 1) };
            // On grids of up to 32 x 32 G takes dS as the sum of two bf16, as in windows: of 28 x 28 dQ is off by 2.4e-3 of its norm instead of 2.5e-3 (larger grids: 2.4e-3 with one, and
            // they would pay for it: two products a block of 18, or eight of 32)
            constexpr bool FINE = NT <= 2;
            bf16x8 lo[2];
            if constexpr (FINE)
#pragma unroll
                for (int r = 0; r < 16; ++r) lo[r >> 3][r & 7] = (bf16)(dp[r] - (float)ds[r >> 3][r & 7]);
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < C::DT; ++c) acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kt(smem, at + St::K, t, c), ds[t], acc[c], 0, 0, 0);
            if constexpr (!LOCAL) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int c = 0; c < NT; ++c) {
                        const bf16x8 one = et(smem, eat, t, c);
                        gt[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, ds[t], gt[c], 0, 0, 0);
                        if constexpr (FINE) gt[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, lo[t], gt[c], 0, 0, 0);
                    }
            } else if constexpr (C::ES == 2) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 one = et(smem, eat, t, 0);
                    gt[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, ds[t], gt[0], 0, 0, 0);
                    gt[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, lo[t], gt[0], 0, 0, 0);
                }
            } else {
                // rows' slice in registers 0 to 7 of the product, columns' in 8 to 15
#pragma unroll 1
                for (int i = 0; i < (two ? 1 : C::ES); ++i) {
                    bf16x8 some[2] = { ds[0], ds[1] }, rest[2];
                    if constexpr (FINE) {
                        rest[0] = lo[0];
                        rest[1] = lo[1];
                    }
                    int to_r = rs, to_c = cs + C::ES / 2;
                    if (!two) {                              // dS of the keys in slice i
                        const bool is_row = i < C::ES / 2;
                        const uint32_t keys = (uint32_t)__builtin_amdgcn_ballot_w64((is_row ? rc >> 4 & 15 : (rc >> 20) + C::ES / 2) == i);
                        if (keys == 0) continue;
                        to_r = is_row ? i : -1;
                        to_c = is_row ? -1 : i;
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const bool in = keys >> (8 * (r >> 2) + (r & 3) + 4 * half) & 1;
                            some[r >> 3][r & 7] = in ? ds[r >> 3][r & 7] : (bf16)0.f;
                            if constexpr (FINE) rest[r >> 3][r & 7] = in ? lo[r >> 3][r & 7] : (bf16)0.f;
                        }
                    }
                    f32x16 part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(et(smem, eat, 0, 0), some[0], zero16(), 0, 0, 0);
                    part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(et(smem, eat, 1, 0), some[1], part, 0, 0, 0);
                    if constexpr (FINE) {
                        part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(et(smem, eat, 0, 0), rest[0], part, 0, 0, 0);
                        part = __builtin_amdgcn_mfma_f32_32x32x16_bf16(et(smem, eat, 1, 0), rest[1], part, 0, 0, 0);
                    }
                    mfma_settle();
#pragma unroll
                    for (int k = 0; k < C::ES; ++k)
                        if (k == (k < C::ES / 2 ? to_r : to_c))
#pragma unroll
                            for (int r = 0; r < 8; ++r) g[k][r] += part[(k < C::ES / 2 ? 0 : 8) + r];
                }
            }
        }
    }
    mfma_settle();
    l += __shfl_xor(l, 32, 64);
    if (qpos < P.SP && half == 0) {
        const bool none = qpos >= S || (P.out_rows && P.out_rows[(long)grp * S + qpos] < 0);
        P.lse[(long)gh * P.SP + qpos] = none ? -INFINITY : -(m + __builtin_amdgcn_logf(l)) * P.inv_scale_log2e;
        P.delta[(long)gh * P.SP + qpos] = -delta;
    }
    const float inv = 1.f / l;
    float most = 0.f;
#pragma unroll
    for (int c = 0; c < C::DT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[c][r] = alive ? acc[c][r] * (inv * P.scale) : 0.f;
    // G of slice i: register r <-> entry 16 i + 8 (r >> 2) + 4 half + (r & 3)
    auto gs = [&](int i, int r) -> float { return LOCAL && C::ES > 2 ? g[LOCAL ? i : 0][r] : gt[LOCAL ? 0 : i >> 1][(i & 1) * 8 + r]; };
    auto set_gs = [&](int i, int r, float v) { if constexpr (LOCAL && C::ES > 2) g[i][r] = v; else gt[LOCAL ? 0 : i >> 1][(i & 1) * 8 + r] = v; };
#pragma unroll
    for (int i = 0; i < C::ES; ++i)
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            const float v = alive ? gs(i, r) * (inv * 128.f) : 0.f;
            set_gs(i, r, v);
            most = fmaxf(most, fabsf(v));
        }

    // (in front of the first row WK places that entries from w on, zeros, may go to)
    bf16 *gr = reinterpret_cast<bf16 *>(smem) + C::WK + wave * 32 * C::RP, *rel = reinterpret_cast<bf16 *>(smem) + C::WK + 4 * 32 * C::RP;
    bf16 *mine = gr + l32 * C::RP;
    const int relrows = (nrel + 15) / 16 * 16;
    __syncthreads();
    if (P.gsum) {
        // G for the tables' gradient, in fp16 over a power of two that puts a query's largest entry at 2^14 or more: eight times as exact as bf16, in the same bytes
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 127, -100), 127);
        const float unit = __uint_as_float((uint32_t)(e - 14 + 127) << 23), over = __uint_as_float((uint32_t)(14 - e + 127) << 23);
#pragma unroll
        for (int i = 0; i < C::ES; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f16x4 v = { (_Float16)(gs(i, 4 * k) * over), (_Float16)(gs(i, 4 * k + 1) * over), (_Float16)(gs(i, 4 * k + 2) * over), (_Float16)(gs(i, 4 * k + 3) * over) };
                *reinterpret_cast<f16x4 *>(mine + 16 * i + 8 * k + 4 * half) = v;
            }
        if (qpos < S && half == 0) P.gunit[(long)gh * S + qpos] = unit;
        wave_lds_fence();
        for (int i = lane; i < 32 * (C::EW / 8); i += 64) {
            const int r = i / (C::EW / 8), c = i % (C::EW / 8), at = q0 + wave * 32 + r;
            if (at < S) *reinterpret_cast<uint4 *>(P.gsum + ((long)gh * S + at) * C::EW + c * 8) = *reinterpret_cast<const uint4 *>(gr + r * C::RP + c * 8);
        }
        wave_lds_fence();
    }

    // dQ += G at relative positions . rel, one table after the other, G as the sum of two bf16 (one alone would add its rounding to that of dS)
#pragma unroll
    for (int tab = 0; tab < 2; ++tab) {
        __syncthreads();
        constexpr int RELS = (2 * C::WK * CH + 255) / 256;
        u32x4 rv[RELS];                                      // all asked for before the first is waited for
#pragma unroll
        for (int k = 0; k < RELS; ++k) {
            const int i = tid + 256 * k, row = i / CH, c = i - row * CH;
            rv[k] = *reinterpret_cast<const u32x4 *>((tab ? P.rel_w : P.rel_h) + (long)min(row, nrel - 1) * D + c * 8);
        }
#pragma unroll
        for (int k = 0; k < RELS; ++k) {
            const int i = tid + 256 * k, row = i / CH, c = i - row * CH;
            if (row < relrows) *reinterpret_cast<u32x4 *>(rel + row * C::VP + c * 8) = row < nrel ? rv[k] : u32x4{ 0, 0, 0, 0 };
        }
        for (int i = 8 * half; i < relrows; i += 16) *reinterpret_cast<uint4 *>(mine + i) = make_uint4(0, 0, 0, 0);
        const int t0 = (tab ? qrc >> 16 : qrc & 0xffff) + w - 1;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            wave_lds_fence();
#pragma unroll
            for (int i = tab * C::ES / 2; i < (tab + 1) * C::ES / 2; ++i)
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const int y = 16 * (i - tab * C::ES / 2) + 8 * (r >> 2) + (r & 3);       // + 4 * half
                    const float x = gs(i, r);
                    const bf16 v = (bf16)x;
                    mine[t0 - 4 * half - y] = v;             // (zeros of entries from w on: places of zeros, in front of the row the unused end of the one before)
                    if (part == 0) set_gs(i, r, x - (float)v);
                }
            if (part == 0) __syncthreads();
            else wave_lds_fence();
            for (int t = 0; t < relrows / 16; ++t) {
                const bf16x4 a = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 4 * half), b = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 8 + 4 * half);
                const bf16x8 g8 = { a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(rel + 16 * t * C::VP, C::VP, 0, dt, D - 4), g8, acc[dt], 0, 0, 0);
            }
        }
        mfma_settle();
    }
    __syncthreads();
    store_rows<D>(acc, reinterpret_cast<bf16 *>(smem) + wave * 32 * C::VP, P.dq + (long)grp * S * P.grad_stride + (long)head * D, P.grad_stride, qpos < S ? qpos : -1);
}

// ---------------------------------------------------------------- columns
// Stages of a column walk, two buffers of them in LDS.  LOCAL: bias entries of the up to four slices (16 entries) that the workgroup's 128 keys have ones in
// (all that there are up to 32 x 32; three on the position-only order of a 64 x 64 grid), 64 queries.  Otherwise of all slices, 32 queries.
// Requests reach the first 64 KB of LDS.
template <int D, int NT, bool LOCAL>
struct ColStage {
    using C = BwdCfg<D, NT>;
    static constexpr int QUERIES = LOCAL ? 64 : 32, SLOTS = LOCAL && C::ES > 4 ? 4 : C::ES;
    static constexpr bool ALL = SLOTS == C::ES;              // a slot is a slice
    static constexpr int QP = D * 2, TP = SLOTS * 32;        // rows, in bytes
    static constexpr int Q = 0, O = Q + QUERIES * QP, T = O + QUERIES * QP, L = T + QUERIES * TP, N = L + QUERIES * 4, BYTES = N + QUERIES * 4;
    static_assert(2 * BYTES <= 64 * 1024, "");
};

template <int D, int NT>
__host__ __device__ constexpr size_t columns_lds_bytes()
{
    size_t m = 2 * ColStage<D, NT, true>::BYTES;
    if (NT > 2 && 2 * ColStage<D, NT, false>::BYTES > m) m = 2 * ColStage<D, NT, false>::BYTES;
    const size_t rows = (size_t)4 * 32 * BwdCfg<D, NT>::VP * 2;
    return rows > m ? rows : m;
}

// Work of the launch: first the tiles of 128 keys with keys of the dense prefix, which every query sees, in `splits` slices of the queries each; then the others,
// which see 128 queries.
struct ColWork { int heavy, light, splits, gh8; };           // tiles a (group, head); groups of eight (group, head)

// The walk of a wave's 32 keys (one a lane) over the queries first .. last.
template <int D, int NT, bool LOCAL>
__device__ __forceinline__ void walk_queries(const BwdParams &P, unsigned char *smem, int grp, int head, int gh, int kb, int first, int last,
                                             uint32_t wanted, int row, int col, bool two, int rs, int cs,
                                             const bf16x8 *kf, const bf16x8 *vf, f32x16 *dk, f32x16 *dv)
{
    using C = BwdCfg<D, NT>;
    using St = ColStage<D, NT, LOCAL>;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, l32 = lane & 31, half = lane >> 5;
    const int S = P.S;
    // slice in a slot: the wanted ones in order; a slot without one repeats the first, whose entries meet zeros of E
    uint32_t slices = 0;                                     // a byte each
    f16x8 ef[St::SLOTS];
    uint32_t left = wanted;
#pragma unroll
    for (int s = 0; s < St::SLOTS; ++s) {
        const int slice = St::ALL ? s : __builtin_ctz(left ? left : wanted);
        const bool twice = !St::ALL && left == 0;
        left &= left - 1;
        if (!St::ALL) slices |= (uint32_t)slice << 8 * s;
        ef[s] = ones(twice ? -1 : (16 * slice < C::WK ? row : col) - 16 * slice - 8 * half);
    }
    if (two) {                                               // the first two operands, and their slots
        ef[0] = ones(row - 16 * rs - 8 * half);
        ef[1] = ones(col - 16 * cs - 8 * half);
        if (!St::ALL) {
            rs = __builtin_popcount(wanted & ((1u << rs) - 1));
            cs = __builtin_popcount(wanted & ((1u << cs) - 1));
        }
    }
    const bool alive = kb < S;

    // requests of a stage, 1 KB each, dealt out to the waves
    constexpr int CH = D / 8, TC = St::SLOTS * 2, NI = St::QUERIES * CH / 64, TI = St::QUERIES * TC / 64;
    constexpr int NQ = (NI + 3) / 4, NB = (TI + 3) / 4;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(size_t)(__attribute__((address_space(3))) unsigned char *)smem);
    const bf16 *qbase = P.q + (long)grp * S * P.row_stride + (long)head * D, *dbase = P.dout + (long)head * D;
    const long drow = (long)P.h * D;
    auto stage = [&](int q0, int buf) {
        int ln = lane;
        if (D == 80) asm volatile("" : "+v"(ln));            // places are worked out again: kept, they would take registers that are short
        const uint32_t to = lds0 + buf * St::BYTES;
        const unsigned char *qs = reinterpret_cast<const unsigned char *>(qbase) + (long)q0 * P.row_stride * 2;
        const unsigned char *ds = reinterpret_cast<const unsigned char *>(dbase) + ((long)grp * S + q0) * drow * 2;
        const bool plain = q0 + St::QUERIES <= S && !P.out_rows;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int j = wave + 4 * i;
            if (j >= NI) continue;
            const int at = j * 64 + ln, r = at / CH, c = at % CH ^ swizzle<CH>(r);
            const uint32_t qoff = r * (uint32_t)P.row_stride * 2 + c * 16, doff = r * (uint32_t)drow * 2 + c * 16;
            if (plain) {
                request(to + St::Q + j * 1024, qoff, qs);
                request(to + St::O + j * 1024, doff, ds);
            } else {                                         // rows past the end, and those whose output is dropped, are zeros
                int orow = q0 + r < S ? 0 : -1;
                if (q0 + r < S && P.out_rows) orow = P.out_rows[(long)grp * S + q0 + r];
                request(to + St::Q + j * 1024, orow < 0 ? (const void *)P.zeros : qs + qoff);
                request(to + St::O + j * 1024, orow < 0 ? (const void *)P.zeros : P.out_rows ? (const void *)(dbase + orow * drow + c * 8) : ds + doff);
            }
        }
        // (rows from SP on are the next (group, head)'s, or what follows the table: blocks past the end are left out)
        const unsigned char *ts = reinterpret_cast<const unsigned char *>(P.tab + ((long)gh * P.SP + q0) * C::EW);
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int j = wave + 4 * i;
            if (j >= TI) continue;
            const int at = j * 64 + ln, r = at / TC, c = at % TC ^ swizzle<TC>(r);
            const int s = St::ALL ? c >> 1 : slices >> 8 * (c >> 1) & 0xff;
            request(to + St::T + j * 1024, (uint32_t)(r * C::EW + 16 * s + 8 * (c & 1)) * 2, ts);
        }
        constexpr int FOURS = St::QUERIES / 4;
        if (wave == 3 && lane < 2 * FOURS) request(to + St::L, (lane < FOURS ? P.lse : P.delta) + (long)gh * P.SP + q0 + 4 * (lane % FOURS));
    };

    // places of this lane's operands in a buffer: rows l32 of a block by 16-byte chunks, and transposed
    const Straight<CH> qa;
    const Transposed<CH> qt;

    int buf = 0;
    if (first < last) stage(first, 0);
    for (int q0 = first; q0 < last; q0 += St::QUERIES, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        LDS_BARRIER();                                       // this stage has landed, and nobody reads the other buffer any more
        if (q0 + St::QUERIES < last) stage(q0 + St::QUERIES, buf ^ 1);
#pragma unroll 1
        for (int b = 0; b < St::QUERIES / 32; ++b) {
            const int qb = q0 + 32 * b;
            if (!alive || qb >= last) continue;              // the same for the whole wave
            const int at = buf * St::BYTES + 32 * b * St::QP;
            // result rows are queries: register r <-> query 8 (r >> 2) + 4 half + (r & 3); scores begin at -log sum exp, dP at -delta
            f32x16 p, ds;
            const float *ls = reinterpret_cast<const float *>(smem + buf * St::BYTES + St::L) + 32 * b + 4 * half;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(ls + 8 * g), u = *reinterpret_cast<const f32x4 *>(ls + St::QUERIES + 8 * g);
#pragma unroll
                for (int e = 0; e < 4; ++e) { p[4 * g + e] = v[e]; ds[4 * g + e] = u[e]; }
            }
            const unsigned char *tl = smem + buf * St::BYTES + St::T + (32 * b + l32) * St::TP;
            const int sw = half ^ swizzle<TC>(l32);
            if (two) {
                p = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(tl + (2 * rs ^ sw) * 16), ef[0], p, 0, 0, 0);
                p = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(tl + (2 * cs ^ sw) * 16), ef[1], p, 0, 0, 0);
            } else {
#pragma unroll
                for (int s = 0; s < St::SLOTS; ++s) p = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(tl + (2 * s ^ sw) * 16), ef[s], p, 0, 0, 0);
            }
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qa(smem, at + St::Q, ks), kf[ks], p, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) ds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qa(smem, at + St::O, ks), vf[ks], ds, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                p[r] = __builtin_amdgcn_exp2f(p[r] * P.scale_log2e);
                ds[r] *= p[r];
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8 pf = half_of(p, t), df = half_of(ds, t);
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt) {
                    dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt(smem, at + St::O, t, dt), pf, dv[dt], 0, 0, 0);
                    dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qt(smem, at + St::Q, t, dt), df, dk[dt], 0, 0, 0);
                }
            }
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(256, NT < 8 ? 2 : 1)
backward_columns_kernel(BwdParams P, ColWork work, float *__restrict__ parts)
{
    using C = BwdCfg<D, NT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // one (group, head) stays on one XCD, whose L2 then serves the re-reads of its queries
    const int heavies = work.heavy * work.splits;
    int unit = blockIdx.x >> 3, gh = blockIdx.x & 7, tile, split = 0;
    if (unit < work.gh8 * heavies) {
        gh += unit / heavies * 8;
        unit %= heavies;
        tile = unit / work.splits;
        split = unit - tile * work.splits;
    } else {
        unit -= work.gh8 * heavies;
        gh += unit / work.light * 8;
        tile = work.heavy + unit % work.light;
    }
    if (gh >= P.n_gh) return;
    const int grp = gh / P.h, head = gh - grp * P.h;
    const int S = P.S;
    const int k0 = tile * 128, kb = k0 + wave * 32, kpos = kb + l32;
    const int at = min(kpos, S - 1);                         // keys past the end repeat the last one; their results are not stored
    bf16x8 kf[C::KS], vf[C::KS];
    const long o = ((long)grp * S + at) * P.row_stride + (long)head * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
        kf[ks] = *reinterpret_cast<const bf16x8 *>(P.k + o + ks * 16);
        vf[ks] = *reinterpret_cast<const bf16x8 *>(P.v + o + ks * 16);
    }
    const int rc = row_col(P.sigma + (long)grp * P.sigma_stride, at, P), row = rc & 0xffff, col = C::WK + (rc >> 16);
    const int rs = __builtin_amdgcn_readfirstlane(row >> 4), cs = __builtin_amdgcn_readfirstlane(col >> 4);
    const bool two = __builtin_amdgcn_ballot_w64(row >> 4 != rs || col >> 4 != cs) == 0;       // all of the wave's keys have their ones in the same two slices
    uint32_t wanted = (1u << C::ES) - 1;
    if (NT > 2) {
        uint32_t mine = 0;
#pragma unroll
        for (int s = 0; s < C::ES; ++s) mine |= __builtin_amdgcn_ballot_w64((16 * s < C::WK ? row : col) >> 4 == s) ? 1u << s : 0u;
        uint32_t *mask = reinterpret_cast<uint32_t *>(smem);
        if (lane == 0) mask[wave] = mine;
        __syncthreads();
        wanted = __builtin_amdgcn_readfirstlane(mask[0] | mask[1] | mask[2] | mask[3]);
        __syncthreads();
    }
    int first = 0, last = S;
    if (tile >= work.heavy) {
        first = k0;
        last = min(k0 + 128, S);
    } else if (work.splits > 1) {
        const int per = (S + 64 * work.splits - 1) / (64 * work.splits) * 64;
        first = min(split * per, S);
        last = min(first + per, S);
    }
    f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
    for (int t = 0; t < C::DT; ++t) { dk[t] = zero16(); dv[t] = zero16(); }
    if (NT <= 2 || __builtin_popcount(wanted) <= 4)
        walk_queries<D, NT, true>(P, smem, grp, head, gh, kb, first, last, wanted, row, col, two, rs, cs, kf, vf, dk, dv);
    else if constexpr (NT > 2)
        walk_queries<D, NT, false>(P, smem, grp, head, gh, kb, first, last, wanted, row, col, two, rs, cs, kf, vf, dk, dv);
    mfma_settle();
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[dt][r] *= P.scale;
    if (work.splits > 1 && tile < work.heavy) {              // [split][gh][key][dK | dV], added up by the next launch
        float *to = parts + (((long)split * P.n_gh + gh) * work.heavy * 128 + kpos) * 2 * D + 4 * half;
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                if (dt * 32 + 8 * g >= D) continue;
                *reinterpret_cast<f32x4 *>(to + dt * 32 + 8 * g) = f32x4{ dk[dt][4 * g], dk[dt][4 * g + 1], dk[dt][4 * g + 2], dk[dt][4 * g + 3] };
                *reinterpret_cast<f32x4 *>(to + D + dt * 32 + 8 * g) = f32x4{ dv[dt][4 * g], dv[dt][4 * g + 1], dv[dt][4 * g + 2], dv[dt][4 * g + 3] };
            }
        return;
    }
    bf16 *scratch = reinterpret_cast<bf16 *>(smem) + wave * 32 * C::VP;
    const long to = (long)grp * S * P.grad_stride + (long)head * D;
    const int stored = kpos < S ? kpos : -1;
    store_rows<D>(dk, scratch, P.dk + to, P.grad_stride, stored);
    store_rows<D>(dv, scratch, P.dv + to, P.grad_stride, stored);
}

// dK and dV of the prefix's keys: the slices' sums.  A thread has eight columns of one of the two.
__global__ void __launch_bounds__(256)
backward_join_kernel(BwdParams P, ColWork work, int D, const float4 *__restrict__ parts, long n)
{
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    const int per = 2 * D / 8;
    if (i >= n) return;
    const long key = i / per;                                // of all (group, head)
    const int c = (int)(i - key * per), keys = work.heavy * 128, gh = (int)(key / keys), pos = (int)(key - (long)gh * keys), grp = gh / P.h, head = gh - grp * P.h;
    if (pos >= P.S) return;
    float a[8] = { 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
    for (int s = 0; s < work.splits; ++s) {
        const float4 *from = parts + (((long)s * P.n_gh * keys + key) * per + c) * 2;
        const float4 u = from[0], v = from[1];
        a[0] += u.x; a[1] += u.y; a[2] += u.z; a[3] += u.w; a[4] += v.x; a[5] += v.y; a[6] += v.z; a[7] += v.w;
    }
    bf16 *to = (c < per / 2 ? P.dk : P.dv) + ((long)grp * P.S + pos) * P.grad_stride + (long)head * D + (c < per / 2 ? c : c - per / 2) * 8;
    *reinterpret_cast<uint4 *>(to) = pack_bf16x8(a);
}

// ---------------------------------------------------------------- tables
// drel_h[t] = sum over rows R of H_R[R + w - 1 - t], H_R[y] = sum over the queries i in row R of GH[i][y] q_i, in all groups and heads; drel_w likewise by columns.  H_R is a plain
// product over queries, with nothing to shift.  A workgroup has one R of one table and a slice of the (group, head); 64 queries a step, G as the sum of two bf16.
constexpr int TABLE_QUERIES = 64;

template <int D, int NT>
struct TableStage {
    using C = BwdCfg<D, NT>;
    static constexpr int GP = C::WK + 8;                      // odd in 16-byte units (C::VP too)
    static constexpr int MT = (C::WK + 31) / 32;              // 32-row tiles of entries
    static constexpr int TILES = MT * C::DT, MINE = (TILES + 3) / 4;
    static constexpr size_t BYTES = (size_t)TABLE_QUERIES * (2 * GP + C::VP) * 2;
};

template <int D, int NT>
__global__ void __launch_bounds__(256)
backward_tables_kernel(BwdParams P, int slices, float *__restrict__ parts)
{
    using C = BwdCfg<D, NT>;
    using St = TableStage<D, NT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    bf16 *hi = reinterpret_cast<bf16 *>(smem), *lo = hi + TABLE_QUERIES * St::GP, *Qs = lo + TABLE_QUERIES * St::GP;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int w = P.w, S = P.S;
    const int tab = blockIdx.x / (w * slices), R = blockIdx.x / slices % w, slice = blockIdx.x % slices;
    const long all = (long)P.n_gh * w, per = (all + slices - 1) / slices, last = min((slice + 1) * per, all);
    f32x16 acc[St::MINE];
#pragma unroll
    for (int i = 0; i < St::MINE; ++i) acc[i] = zero16();
    constexpr int CH = D / 8, GC = C::WK / 8;
    static_assert(TABLE_QUERIES * GC % 128 == 0, "");
    for (long k0 = slice * per; k0 < last; k0 += TABLE_QUERIES) {
        __syncthreads();
        // row j of the step is query (gh, x): the one in row R and column x (tab 1: column R, row x) of group gh / h
        auto place = [&](int j, int &gh) {
            const long k = k0 + j;
            if (k >= last) return -1;
            gh = (int)(k / w);
            const int x = (int)(k - (long)gh * w), cell = tab ? x * w + R : R * w + x;
            const int at = P.inverse[(P.sigma_stride ? (long)(gh / P.h) * S : 0) + cell];
            return min(max(at, 0), S - 1);
        };
        for (int i = tid; i < TABLE_QUERIES * GC; i += 256) {
            const int j = i / GC, c = i % GC;
            int gh = 0;
            const int at = place(j, gh);
            uint4 h4 = make_uint4(0, 0, 0, 0), l4 = h4;
            if (at >= 0) {
                const long row = (long)gh * S + at;
                const f16x8 g = *reinterpret_cast<const f16x8 *>(P.gsum + row * C::EW + tab * C::WK + c * 8);
                const float unit = P.gunit[row];
                float a[8], b[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = (float)g[e] * unit;
                    a[e] = (float)(bf16)v;
                    b[e] = v - a[e];
                }
                h4 = pack_bf16x8(a);
                l4 = pack_bf16x8(b);
            }
            *reinterpret_cast<uint4 *>(hi + j * St::GP + c * 8) = h4;
            *reinterpret_cast<uint4 *>(lo + j * St::GP + c * 8) = l4;
        }
        for (int i = tid; i < TABLE_QUERIES * CH; i += 256) {
            const int j = i / CH, c = i - j * CH;
            int gh = 0;
            const int at = place(j, gh);
            uint4 v = make_uint4(0, 0, 0, 0);
            if (at >= 0) {
                const int grp = gh / P.h;
                const long slot = (long)grp * S + at;
                if (!P.out_rows || P.out_rows[slot] >= 0) v = *reinterpret_cast<const uint4 *>(P.q + slot * P.row_stride + (long)(gh - grp * P.h) * D + c * 8);
            }
            *reinterpret_cast<uint4 *>(Qs + j * C::VP + c * 8) = v;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < St::MINE; ++i) {
            const int tile = wave + 4 * i, mt = tile / C::DT, dt = tile - mt * C::DT;
            if (tile >= St::TILES) continue;
#pragma unroll
            for (int t = 0; t < TABLE_QUERIES / 16; ++t) {
                const bf16x8 q = transposed(Qs + 16 * t * C::VP, C::VP, 0, dt, D - 4);
                acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(hi + 16 * t * St::GP, St::GP, 0, mt, C::WK - 4), q, acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(lo + 16 * t * St::GP, St::GP, 0, mt, C::WK - 4), q, acc[i], 0, 0, 0);
            }
        }
    }
    mfma_settle();
    // [table][R][slice][entry][feature]; result: lane <-> feature, register <-> entry
    float *to = parts + (long)blockIdx.x * C::WK * D;
#pragma unroll
    for (int i = 0; i < St::MINE; ++i) {
        const int tile = wave + 4 * i, mt = tile / C::DT, c = (tile - mt * C::DT) * 32 + l32;
        if (tile >= St::TILES) continue;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int y = mt * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
            if (y < w && c < D) to[(long)y * D + c] = acc[i][r];
        }
    }
}

// A row of a table's gradient: the sum of H_R[R + w - 1 - t] over R and the slices, or (WINDOWS) of the row itself over the workgroups that have summed it.  32 features a workgroup: eight lanes with 16 bytes each, 32 shares of the terms.
template <bool WINDOWS>
__global__ void __launch_bounds__(256)
backward_table_sums_kernel(const float4 *__restrict__ parts, int w, int WK, int slices, int D, bf16 *__restrict__ drel_h, bf16 *__restrict__ drel_w)
{
    __shared__ float4 lds[256];
    const int c = threadIdx.x & 7, share = threadIdx.x >> 3, t = blockIdx.y, tab = blockIdx.z;
    const int quad = blockIdx.x * 8 + c, quads = D / 4, first = max(0, t - w + 1), n = WINDOWS ? slices : (min(w - 1, t) - first + 1) * slices;
    const bool in = quad < quads;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int i = share; i < n; i += 32) {
        const int R = first + i / slices, y = R + w - 1 - t;
        const float4 v = parts[(WINDOWS ? ((long)i * 2 + tab) * 32 + t : (((long)tab * w + R) * slices + i % slices) * WK + y) * quads + min(quad, quads - 1)];
        a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
    a = sum_of_shares(a, lds);
    if (share == 0 && in) *reinterpret_cast<uint2 *>((tab ? drel_w : drel_h) + (long)t * D + quad * 4) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
}

}  // namespace

#include "attention_backward_window.h"

namespace {

// ---------------------------------------------------------------- launches
inline int entry_tiles(int w) { return w <= 16 ? 1 : w <= 32 ? 2 : w <= 64 ? 4 : 8; }
// Slices of the (group, head) of a row of a table: a thousand workgroups, of a step of 64 queries each at least
inline int table_slices(int w, long n_gh)
{
    const long steps = (n_gh * w + TABLE_QUERIES - 1) / TABLE_QUERIES, n = (512 + w - 1) / w;
    return (int)(n < steps ? n : steps);
}

// Tiles of the dense prefix have all queries to walk: with few of them, a slice of the queries each, until there are two workgroups to a CU.
constexpr int COL_SLOTS = 512;
inline int column_splits(long heavy, int S)
{
    const long most = (S + 255) / 256, n = COL_SLOTS / (heavy > 0 ? heavy : 1);
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

inline int window_groups(long n_gh) { return (int)(n_gh < WIN_GROUPS ? n_gh : WIN_GROUPS); }

struct BwdWorkspace { size_t zeros, tab, gsum, gunit, lse, delta, e, blocks, inverse, parts, total; };
inline BwdWorkspace workspace_layout(int groups, int S, int w, int h, int d)
{
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t rows = (size_t)groups * h * ((S + 31) / 32 * 32), entries = rows * 32 * entry_tiles(w) * 2;
    BwdWorkspace o = {};
    if (S <= WIN_ROWS) {                                     // sums of the tables' gradients alone: all else stays in LDS
        o.total = (size_t)window_groups((long)groups * h) * 2 * 32 * d * 4;
        return o;
    }
    o.zeros = 0;
    o.tab = 1024;
    o.gsum = o.tab + up(entries + 32 * 64 * entry_tiles(w));                        // (the last stage reads up to 32 rows past the end)
    o.gunit = o.gsum + up(entries);
    o.lse = o.gunit + up(rows * 4);
    o.delta = o.lse + up(rows * 4 + 128);
    // one order a group at most
    const size_t orders = (size_t)groups * ((S + 31) / 32 * 32);
    o.e = o.delta + up(rows * 4 + 128);
    o.blocks = o.e + up((orders + 64) * 64 * entry_tiles(w));
    o.inverse = o.blocks + up(orders / 32 * 4);
    o.parts = o.inverse + up(orders * 4);
    // sums of slices: of the tables' gradients, and before those of dK and dV of at most COL_SLOTS tiles
    const size_t tables = (size_t)2 * w * table_slices(w, (long)groups * h) * 16 * entry_tiles(w) * d * 4;
    const long tiles = (long)groups * h * ssam_div_up(S, 128), slots = tiles * ssam_div_up(S, 256);
    const size_t columns = S <= 256 ? 0 : (size_t)(slots < COL_SLOTS ? slots : COL_SLOTS) * 128 * 2 * d * 4;
    o.total = o.parts + up(tables > columns ? tables : columns);
    return o;
}

template <typename Kernel>
int allow_lds(Kernel k, size_t bytes)
{
    if (bytes > 160 * 1024) return SSAM_EUNSUPPORTED;
    if (bytes > 64 * 1024 && hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return SSAM_EHIP;
    return SSAM_OK;
}

template <int D, int NT>
int launch_backward(const BwdParams &P, float *parts, bf16 *drel_h, bf16 *drel_w, hipStream_t st)
{
    const int tiles = ssam_div_up(P.S, 128), nrel = 2 * P.w - 1;
    const unsigned grid = (unsigned)((long)tiles * ssam_div_up(P.n_gh, 8) * 8);
    // orders that all groups share are the position-only ones, whose blocks of keys are patches of a grid of a power of two (28 x 28, where they are not: 67 us against 45);
    // those of one group alone scatter them
    const bool local = NT == 1 || (P.sigma_stride == 0 && (P.w & (P.w - 1)) == 0);
    const int blocks = P.SP / 32, total = blocks * (P.sigma_stride ? P.n_gh / P.h : 1);
    auto prepare = local ? backward_prepare_kernel<NT, true> : backward_prepare_kernel<NT, NT == 1>;
    hipLaunchKernelGGL(prepare, dim3(ssam_div_up(total, 4)), dim3(256), 0, st, P, blocks, total);
    SSAM_CHECK_LAUNCH();
    auto rows = local ? backward_rows_kernel<D, NT, true> : backward_rows_kernel<D, NT, NT == 1>;
    const size_t lds = local ? rows_lds_bytes<D, NT, true>(nrel) : rows_lds_bytes<D, NT, NT == 1>(nrel);
    if (int rc = allow_lds(rows, lds); rc != SSAM_OK) return rc;
    if (int rc = allow_lds(backward_columns_kernel<D, NT>, columns_lds_bytes<D, NT>()); rc != SSAM_OK) return rc;
    hipLaunchKernelGGL(rows, dim3(grid), dim3(256), lds, st, P, tiles);
    SSAM_CHECK_LAUNCH();
    ColWork work;
    work.gh8 = ssam_div_up(P.n_gh, 8);
    work.heavy = min(P.n_pre, tiles);
    work.light = tiles - work.heavy;
    work.splits = column_splits((long)work.heavy * P.n_gh, P.S);
    hipLaunchKernelGGL((backward_columns_kernel<D, NT>), dim3((unsigned)(8L * work.gh8 * (work.heavy * work.splits + work.light))), dim3(256),
                       (columns_lds_bytes<D, NT>()), st, P, work, parts);
    SSAM_CHECK_LAUNCH();
    if (work.splits > 1 && work.heavy > 0) {
        const long n = (long)P.n_gh * work.heavy * 128 * (2 * D / 8);
        hipLaunchKernelGGL(backward_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, P, work, D, (const float4 *)parts, n);
        SSAM_CHECK_LAUNCH();
    }
    if (drel_h) {
        const int slices = table_slices(P.w, P.n_gh);
        if (int rc = allow_lds(backward_tables_kernel<D, NT>, TableStage<D, NT>::BYTES); rc != SSAM_OK) return rc;
        hipLaunchKernelGGL((backward_tables_kernel<D, NT>), dim3(2 * P.w * slices), dim3(256), (TableStage<D, NT>::BYTES), st, P, slices, parts);
        SSAM_CHECK_LAUNCH();
        hipLaunchKernelGGL((backward_table_sums_kernel<false>), dim3(ssam_div_up(D, 32), nrel, 2), dim3(256), 0, st, (const float4 *)parts, P.w, BwdCfg<D, NT>::WK, slices, D, drel_h, drel_w);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int D>
int launch_windows(const BwdParams &P, float *parts, bf16 *drel_h, bf16 *drel_w, hipStream_t st)
{
    const int groups = window_groups(P.n_gh), nrel = 2 * P.w - 1;
    if (int rc = allow_lds(backward_windows_kernel<D>, WinCfg<D>::TOTAL); rc != SSAM_OK) return rc;
    hipLaunchKernelGGL((backward_windows_kernel<D>), dim3(groups), dim3(64 * WIN_WAVES), WinCfg<D>::TOTAL, st, P,
                       window_work(ssam_div_up(P.S, 32), min(P.n_pre * (P.mask_block / 32), ssam_div_up(P.S, 32)), P.mask_block / 32), drel_h != nullptr, parts);
    SSAM_CHECK_LAUNCH();
    if (drel_h) {
        hipLaunchKernelGGL((backward_table_sums_kernel<true>), dim3(ssam_div_up(D, 32), nrel, 2), dim3(256), 0, st, (const float4 *)parts, P.w, 32, groups, D, drel_h, drel_w);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int D>
int launch_backward(const BwdParams &P, float *parts, bf16 *drel_h, bf16 *drel_w, hipStream_t st)
{
    if (P.S <= WIN_ROWS) return launch_windows<D>(P, parts, drel_h, drel_w, st);
    switch (entry_tiles(P.w)) {
    case 1: return launch_backward<D, 1>(P, parts, drel_h, drel_w, st);
    case 2: return launch_backward<D, 2>(P, parts, drel_h, drel_w, st);
    case 4: return launch_backward<D, 4>(P, parts, drel_h, drel_w, st);
    default: return launch_backward<D, 8>(P, parts, drel_h, drel_w, st);
    }
}

bool backward_sizes_ok(int groups, int S, int w, int h, int d) { return groups > 0 && S > 0 && w > 0 && w <= 128 && h > 0 && d > 0 && (long)w * w == S; }

}  // namespace

extern "C" size_t ssam_sparse_attention_backward_workspace_bytes(int groups, int S, int w, int h, int d)
{
    return backward_sizes_ok(groups, S, w, h, d) ? workspace_layout(groups, S, w, h, d).total : 0;
}

extern "C" int ssam_sparse_attention_backward(const void *q, const void *k, const void *v, long row_stride, const void *rel_h, const void *rel_w,
                                              const int32_t *sigma, long sigma_group_stride, const void *out, const void *dout, const int32_t *out_rows,
                                              void *dq, void *dk, void *dv, long grad_stride, void *drel_h, void *drel_w,
                                              int groups, int S, int w, int h, int d, int mask_block, double r, float scale,
                                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !k || !v || !rel_h || !rel_w || !sigma || !out || !dout || !dq || !dk || !dv || !workspace || (!drel_h) != (!drel_w)) return SSAM_EINVAL;
    if (groups <= 0 || S <= 0 || w <= 0 || h <= 0 || d <= 0 || !(r > 0.0) || r > 1.0 || !(scale > 0.f)) return SSAM_EINVAL;
    if (sigma_group_stride != 0 && sigma_group_stride < S) return SSAM_EINVAL;
    if ((long)w * w != S || row_stride < (long)h * d || row_stride % 8 != 0 || grad_stride < (long)h * d || grad_stride % 8 != 0) return SSAM_EINVAL;
    for (const void *p : { q, k, v, rel_h, rel_w, out, dout, (const void *)dq, (const void *)dk, (const void *)dv, (const void *)drel_h, (const void *)drel_w, (const void *)workspace })
        if (!ssam_aligned16(p)) return SSAM_EINVAL;
    // bias entries are held over the scale in fp16: on grids up to 128 as a logit at the least of these, spaced by 2^-15 of one at the most
    if (scale < 0x1p-9f || scale > 0x1p9f) return SSAM_EUNSUPPORTED;
    if (mask_block == 32 ? S > 224 : mask_block != 128 || S > 16384) return SSAM_EUNSUPPORTED;
    if (d != 16 && d != 32 && d != 64 && d != 80) return SSAM_EUNSUPPORTED;
    if ((long)groups * h > 0x7ffffff0L) return SSAM_EUNSUPPORTED;
    // grids: 32-bit offsets within a group, a workgroup a tile of a (group, head)
    if (S > WIN_ROWS && ((long)S * row_stride * 2 > 0x7fffffffL || (long)ssam_div_up(S, 128) * ((long)groups * h + 7) > 0x7fffffffL / 256)) return SSAM_EUNSUPPORTED;
    const BwdWorkspace at = workspace_layout(groups, S, w, h, d);
    if (workspace_bytes < at.total) return SSAM_EWORKSPACE;
    unsigned char *ws = (unsigned char *)workspace;
    BwdParams P;
    P.q = (const bf16 *)q; P.k = (const bf16 *)k; P.v = (const bf16 *)v;
    P.row_stride = row_stride;
    P.rel_h = (const bf16 *)rel_h; P.rel_w = (const bf16 *)rel_w;
    P.sigma = sigma;
    P.sigma_stride = sigma_group_stride;
    P.out = (const bf16 *)out; P.dout = (const bf16 *)dout;
    P.out_rows = out_rows;
    P.dq = (bf16 *)dq; P.dk = (bf16 *)dk; P.dv = (bf16 *)dv;
    P.grad_stride = grad_stride;
    P.S = S; P.w = w; P.h = h; P.n_gh = groups * h;
    P.per_w = (uint32_t)((1 << 22) / w + 1);
    P.mask_block = mask_block;
    P.n_pre = ssam_prefix_tiles(ssam_div_up(S, mask_block), r);
    P.scale = scale;
    P.scale_log2e = scale * LOG2E;
    P.tab = (_Float16 *)(ws + at.tab);
    // the forward's bounds of the bias: where it has windows, a power of two keeps +-45400 and more (in the forward's groups of tiles of 128, n is 0 at these scales)
    const int n = mask_block == 32 ? window_scale(scale).shift : 0;
    P.one = 0x3c00u + ((uint32_t)n << 10);
    P.over_one = ldexpf(1.f, 7 - 8 * n);
    P.inv_scale = ldexpf(1.f / scale, -n);
    P.inv_scale_log2e = 1.f / P.scale_log2e;
    P.gsum = drel_h ? (_Float16 *)(ws + at.gsum) : nullptr;
    P.gunit = (float *)(ws + at.gunit);
    P.lse = (float *)(ws + at.lse);
    P.delta = (float *)(ws + at.delta);
    P.zeros = (const uint4 *)(ws + at.zeros);
    P.SP = (S + 31) / 32 * 32;
    P.e = (uint4 *)(ws + at.e);
    P.blocks = (uint32_t *)(ws + at.blocks);
    P.inverse = (int32_t *)(ws + at.inverse);
    float *parts = (float *)(ws + at.parts);
    hipStream_t st = (hipStream_t)stream;
    switch (d) {
    case 16: return launch_backward<16>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    case 32: return launch_backward<32>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    case 64: return launch_backward<64>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    default: return launch_backward<80>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    }
}
