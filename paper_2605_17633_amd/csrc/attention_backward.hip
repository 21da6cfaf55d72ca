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
//            dQ, -log2 sum exp and delta of its queries, their bias entries (fp16) and GH, GW (bf16)
//   columns  a wave owns 32 keys and walks their queries: P from the statistics, dK and dV stay in registers
//   tables   drel = (G at relative positions)^T Q, a product over all queries of all groups and heads, in slices that are added up in order
//
// The bias and its gradient are products with the 0/1 matrix E that has a one at every key's row and one at its column: scores
// take E T (T the entries of a query, fp16, in log2 units), G is E^T dS.  E sits behind the keys' features in LDS, [key][K | E], so that one set
// of transposing reads gives K^T and E^T.  Its ones are 0x3c00: 1 in fp16, 2^-7 in bf16, which G is multiplied by at the end.
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
    int mask_block, n_pre;       // tile of the mask, tiles of the dense prefix
    float scale, scale_log2e;
    _Float16 *tab;               // [gh][S][EW]: bias entries of a query, times log2 e
    bf16 *gsum;                  // [gh][S][EW]: GH | GW; NULL: not wanted
    float2 *stat;                // [gh][S]: -log2 sum exp2, delta
};

// NT: 32 entries of E each; half of them rows, half columns
template <int D, int NT>
struct BwdCfg {
    static constexpr int EW = 32 * NT, WK = EW / 2;
    static constexpr int KS = D / 16;                        // k-steps of a product over features
    static constexpr int ES = EW / 16;                       // and over entries
    static constexpr int DT = (D + 31) / 32;                 // 32-row tiles of dK^T, dV^T
    static constexpr int CT = (D + EW + 31) / 32;            // and of [dQ | G]^T
    static constexpr int KP = D + EW + 8, VP = D + 8;        // LDS pitches (elements): odd in 16-byte units
    static constexpr int TP = EW + 8;                        // of bias entries
    static constexpr int RP = 2 * WK + 8;                    // of G at relative positions, one table
};
constexpr int ROW_KEYS = 64;     // keys of a stage of the row kernel
constexpr int COL_QUERIES = 32;  // queries of a stage of the column kernel

// MFMA passes done before results are read under predicates (see the forward kernels)
__device__ __forceinline__ void mfma_settle()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ void wave_lds_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__device__ __forceinline__ f32x16 zero16()
{
    return f32x16{ 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f };
}

// Operand a of step t over 16 rows of an LDS block: lane <-> column 32 * tile + (lane & 31) of rows 16 t + 8 (e / 4) + 4 half + (e & 3), the order in
// which a 32x32 result holds them.  Columns past `last` re-read that quad; what they give is not used.
__device__ __forceinline__ bf16x8 transposed(const bf16 *block, int pitch, int t, int tile, int last)
{
    const int lane = threadIdx.x & 63, li = lane & 15;
    const int col = min(tile * 32 + 16 * ((lane >> 4) & 1) + 4 * (li & 3), last);
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

// ---------------------------------------------------------------- rows
template <int D, int NT>
__host__ __device__ constexpr size_t rows_lds_bytes(int nrel)
{
    using C = BwdCfg<D, NT>;
    const size_t stage = (size_t)ROW_KEYS * (C::KP + C::VP) * 2;
    const size_t tables = (size_t)4 * 32 * C::TP * 2;
    const size_t end = (size_t)4 * 32 * C::RP * 2 + (size_t)(nrel + 31) / 16 * 16 * C::VP * 2;
    const size_t rows = (size_t)4 * 32 * C::VP * 2;
    size_t m = stage > tables ? stage : tables;
    m = end > m ? end : m;
    return rows > m ? rows : m;
}

template <int D, int NT>
__global__ void __launch_bounds__(256, 1)
attn_backward_rows_kernel(BwdParams P, int tiles)
{
    using C = BwdCfg<D, NT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // the tiles of one (group, head) run on one XCD (workgroup b sits on XCD b & 7), whose L2 then serves the re-reads of its K and V
    const int tile = (blockIdx.x >> 3) % tiles, gh = ((blockIdx.x >> 3) / tiles) * 8 + (blockIdx.x & 7);
    if (gh >= P.n_gh) return;
    const int grp = gh / P.h, head = gh - grp * P.h;
    const int S = P.S, w = P.w, nrel = 2 * w - 1;
    const int q0 = tile * 128, qpos = q0 + wave * 32 + l32;
    const int32_t *sigma = P.sigma + (long)grp * P.sigma_stride;

    // this lane's query: its features, dO and delta
    bf16x8 qf[C::KS], of[C::KS];
    float delta = 0.f;
    int orow = -1, qrow = 0, qcol = 0;
    if (qpos < S) {
        const long slot = (long)grp * S + qpos;
        const int cell = sigma[qpos];
        qrow = cell / w;
        qcol = cell - qrow * w;
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
    if (orow < 0) {                                          // past the end, or its output is dropped: no gradient comes from it
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
            for (int e = 0; e < 8; ++e) qf[ks][e] = of[ks][e] = (bf16)0.f;
    }
    delta += __shfl_xor(delta, 32, 64);

    // bias entries: rel Q^T, relative position t of the lane's query is its entry at_q + w - 1 - t
    _Float16 *tq = reinterpret_cast<_Float16 *>(smem) + (wave * 32 + l32) * C::TP;
    for (int p = w + half; p < C::WK; p += 2) tq[p] = tq[C::WK + p] = (_Float16)0.f;
    for (int m0 = 0; m0 < nrel; m0 += 32)
#pragma unroll
        for (int tab = 0; tab < 2; ++tab) {
            const bf16 *rp = (tab ? P.rel_w : P.rel_h) + (long)min(m0 + l32, nrel - 1) * D + half * 8;
            f32x16 u = zero16();
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(rp + ks * 16), qf[ks], u, 0, 0, 0);
            mfma_settle();
            const int p0 = (tab ? qcol : qrow) + w - 1 - m0 - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int p = p0 - 8 * (r >> 2) - (r & 3);
                // a bias past the range of fp16 (45000 as a logit) is cut: an infinity would make NaNs of the zeros of E
                if ((unsigned)p < (unsigned)w) tq[tab * C::WK + p] = (_Float16)__builtin_amdgcn_fmed3f(u[r] * LOG2E, -65504.f, 65504.f);
            }
        }
    wave_lds_fence();
    f16x8 bt[C::ES];
#pragma unroll
    for (int c = 0; c < C::ES; ++c) bt[c] = *reinterpret_cast<const f16x8 *>(tq + 16 * c + 8 * half);
    if (qpos < S) {
        _Float16 *to = P.tab + ((long)gh * S + qpos) * C::EW + 8 * half;
#pragma unroll
        for (int c = 0; c < C::ES; ++c) *reinterpret_cast<f16x8 *>(to + 16 * c) = bt[c];
    }
    __syncthreads();

    // stages of 64 keys: the dense prefix, then (where a wave has a diagonal tile behind it) the workgroup's own 128
    bf16 *Ks = reinterpret_cast<bf16 *>(smem), *Vs = Ks + ROW_KEYS * C::KP;
    const int pre = min(P.n_pre * P.mask_block, S), pre_stages = ssam_div_up(pre, ROW_KEYS);
    const int own = (q0 + wave * 32) / P.mask_block;                                  // mask tile of the wave's queries
    const bool any_diagonal = min(q0 + 127, S - 1) / P.mask_block >= P.n_pre;
    const int stages = pre_stages + (any_diagonal ? ssam_div_up(min(128, S - q0), ROW_KEYS) : 0);
    const bool alive = q0 + wave * 32 < S;

    for (int i = tid; i < ROW_KEYS * (C::EW / 8); i += 256)                          // E starts empty
        *reinterpret_cast<uint4 *>(Ks + (i / (C::EW / 8)) * C::KP + D + (i % (C::EW / 8)) * 8) = make_uint4(0, 0, 0, 0);

    constexpr int CH = D / 8, NLOAD = (ROW_KEYS * CH + 255) / 256;
    u32x4 kr[NLOAD], vr[NLOAD];
    int cell_next = -1;
    const bf16 *kbase = P.k + (long)grp * S * P.row_stride + (long)head * D, *vbase = P.v + (long)grp * S * P.row_stride + (long)head * D;
    auto stage_key = [&](int s) { return s < pre_stages ? s * ROW_KEYS : q0 + (s - pre_stages) * ROW_KEYS; };
    auto load = [&](int s) {
        const int key0 = stage_key(s);
#pragma unroll
        for (int i = 0; i < NLOAD; ++i) {
            const int id = tid + 256 * i, row = id / CH, c = id - row * CH;
            kr[i] = vr[i] = u32x4{ 0, 0, 0, 0 };
            if (id < ROW_KEYS * CH && key0 + row < S) {
                const long at = (long)(key0 + row) * P.row_stride + c * 8;
                kr[i] = *reinterpret_cast<const u32x4 *>(kbase + at);
                vr[i] = *reinterpret_cast<const u32x4 *>(vbase + at);
            }
        }
        if (tid < ROW_KEYS) cell_next = key0 + tid < S ? sigma[key0 + tid] : -1;
    };
    int one_row = -1, one_col = -1;                                                   // where this thread's key has its ones
    auto store = [&]() {
#pragma unroll
        for (int i = 0; i < NLOAD; ++i) {
            const int id = tid + 256 * i, row = id / CH, c = id - row * CH;
            if (id < ROW_KEYS * CH) {
                *reinterpret_cast<u32x4 *>(Ks + row * C::KP + c * 8) = kr[i];
                *reinterpret_cast<u32x4 *>(Vs + row * C::VP + c * 8) = vr[i];
            }
        }
        if (tid < ROW_KEYS) {
            uint16_t *e = reinterpret_cast<uint16_t *>(Ks + tid * C::KP + D);
            if (one_row >= 0) e[one_row] = e[one_col] = 0;
            one_row = -1;
            if (cell_next >= 0) {
                one_row = cell_next / w;
                one_col = C::WK + cell_next - one_row * w;
                e[one_row] = e[one_col] = 0x3c00;
            }
        }
    };

    f32x16 acc[C::CT];
#pragma unroll
    for (int t = 0; t < C::CT; ++t) acc[t] = zero16();
    float m = -INFINITY, l = 0.f;
    if (stages > 0) load(0);
    for (int s = 0; s < stages; ++s) {
        LDS_BARRIER();                                       // every wave is done with the previous stage
        store();
        LDS_BARRIER();
        const int key0 = stage_key(s);
        if (s + 1 < stages) load(s + 1);
#pragma unroll
        for (int b = 0; b < ROW_KEYS / 32; ++b) {
            const int kb = key0 + 32 * b;
            const bool active = alive && kb < S && (s < pre_stages ? kb < pre : own >= P.n_pre && kb / P.mask_block == own);
            if (!active) continue;                           // wave-uniform
            const bf16 *kblk = Ks + 32 * b * C::KP, *vblk = Vs + 32 * b * C::VP;
            f32x16 sc = zero16(), bias = zero16(), dp = zero16();
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks)
                sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(kblk + l32 * C::KP + ks * 16 + half * 8), qf[ks], sc, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < C::ES; ++c)
                bias = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(kblk + l32 * C::KP + D + c * 16 + half * 8), bt[c], bias, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks)
                dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(vblk + l32 * C::VP + ks * 16 + half * 8), of[ks], dp, 0, 0, 0);
            mfma_settle();
            float mx = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                sc[r] = fmaf(sc[r], P.scale_log2e, bias[r]);
                if (kb + 32 > S) sc[r] = kb + 8 * (r >> 2) + 4 * half + (r & 3) < S ? sc[r] : -INFINITY;
                mx = fmaxf(mx, sc[r]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            // the reference moves only when it is exceeded by a factor of 2^8: what the sums are in units of cancels at the end
            const bool move = mx > m + 8.f;
            if (__builtin_amdgcn_ballot_w64(move) != 0) {
                const float to = move ? mx : m, alpha = __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= alpha;
#pragma unroll
                for (int t = 0; t < C::CT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(sc[r] - m);
                l += p;
                dp[r] = p * (dp[r] - delta);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8 ds = half_of(dp, t);
#pragma unroll
                for (int c = 0; c < C::CT; ++c) acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(kblk, C::KP, t, c, D + C::EW - 4), ds, acc[c], 0, 0, 0);
            }
        }
    }
    mfma_settle();
    l += __shfl_xor(l, 32, 64);
    if (qpos < S && half == 0)
        P.stat[(long)gh * S + qpos] = orow < 0 ? make_float2(-INFINITY, 0.f) : make_float2(-m - __builtin_amdgcn_logf(l), delta);
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < C::CT; ++c)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const float f = c * 32 + 8 * g < D ? inv * P.scale : inv * 128.f;       // (a group of eight columns is on one side)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[c][4 * g + e] = alive ? acc[c][4 * g + e] * f : 0.f;
        }

    // dQ += G at relative positions . rel, one table after the other
    bf16 *gr = reinterpret_cast<bf16 *>(smem) + wave * 32 * C::RP, *rel = reinterpret_cast<bf16 *>(smem) + 4 * 32 * C::RP;
    bf16 *mine = gr + l32 * C::RP;
    const int relrows = (nrel + 15) / 16 * 16;
#pragma unroll
    for (int tab = 0; tab < 2; ++tab) {
        __syncthreads();
        for (int i = tid; i < relrows * CH; i += 256) {
            const int row = i / CH, c = i - row * CH;
            u32x4 v = { 0, 0, 0, 0 };
            if (row < nrel) v = *reinterpret_cast<const u32x4 *>((tab ? P.rel_w : P.rel_h) + (long)row * D + c * 8);
            *reinterpret_cast<u32x4 *>(rel + row * C::VP + c * 8) = v;
        }
        for (int i = 8 * half; i < relrows; i += 16) *reinterpret_cast<uint4 *>(mine + i) = make_uint4(0, 0, 0, 0);
        wave_lds_fence();
        const int t0 = (tab ? qcol : qrow) + w - 1;
#pragma unroll
        for (int c = 0; c < C::CT; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int col0 = c * 32 + 8 * (r >> 2) + (r & 3);                    // + 4 * half
                if (c * 32 + 8 * (r >> 2) < D + tab * C::WK || c * 32 + 8 * (r >> 2) >= D + (tab + 1) * C::WK) continue;
                const int y = col0 + 4 * half - D - tab * C::WK;
                if (y < w) mine[t0 - y] = (bf16)acc[c][r];
            }
        __syncthreads();
        for (int t = 0; t < relrows / 16; ++t) {
            const bf16x4 a = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 4 * half), b = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 8 + 4 * half);
            const bf16x8 g8 = { a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(rel + 16 * t * C::VP, C::VP, 0, dt, D - 4), g8, acc[dt], 0, 0, 0);
            // (of a last tile that D fills by half the rest are entries of G, which the operand's repeated columns change: GW's is taken
            // before, see below)
        }
        mfma_settle();
    }
    store_rows<D>(acc, reinterpret_cast<bf16 *>(smem) + wave * 32 * C::VP, P.dq + (long)grp * S * P.grad_stride + (long)head * D, P.grad_stride, qpos < S ? qpos : -1);
}
}  // namespace
