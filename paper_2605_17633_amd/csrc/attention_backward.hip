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
// The bias and its gradient are products with the 0/1 matrix E that has a one at every key's row and one at its column: scores
// take E T (T the entries of a query, fp16, over the scale), G is E^T dS.  E sits behind the keys' features in LDS, [key][K | E], so that one set
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
    float scale, scale_log2e, inv_scale, inv_scale_log2e;
    _Float16 *tab;               // [gh][SP][EW]: bias entries of a query, over the scale
    _Float16 *gsum;              // [gh][S][EW]: GH | GW over gunit; NULL: not wanted
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
    static constexpr int CT = (D + EW + 31) / 32;            // and of [dQ | G]^T
    static constexpr int KP = D + EW + 8, VP = D + 8;        // LDS pitches (elements): odd in 16-byte units
    static constexpr int TP = EW + 8;                        // of bias entries
    static constexpr int RP = 2 * WK + 8;                    // of G at relative positions, one table
    static constexpr int ROW_KEYS = NT < 8 ? 64 : 32;        // keys of a stage of the row kernel
    static constexpr bool KEEP = NT < 8;                     // a wave's queries, dO and bias entries stay in registers, else in LDS
};

// bit 23 of the mode register: fp16 results past the range are clamped instead of rounded to infinity (which would make NaNs of the zeros of E)
__device__ __forceinline__ void clamp_fp16() { __builtin_amdgcn_s_setreg(1 | 23 << 6 | (1 - 1) << 11, 1); }

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
    const size_t tables = (size_t)4 * 32 * C::TP * 2;
    const size_t stage = (size_t)C::ROW_KEYS * (C::KP + C::VP) * 2 + tables + 16 + (C::KEEP ? 0 : (size_t)4 * 32 * 2 * C::VP * 2);
    const size_t end = (size_t)4 * 32 * C::RP * 2 + (size_t)(nrel + 15) / 16 * 16 * C::VP * 2;
    const size_t rows = (size_t)4 * 32 * C::VP * 2;
    const size_t m = end > stage ? end : stage;
    return rows > m ? rows : m;
}

template <int D, int NT>
__global__ void __launch_bounds__(256, NT < 8 ? 2 : 1)
attn_backward_rows_kernel(BwdParams P, int tiles)
{
    using C = BwdCfg<D, NT>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    // the tiles of one (group, head) run on one XCD (workgroup b sits on XCD b & 7), whose L2 then serves the re-reads of its K and V
    const int tile = (blockIdx.x >> 3) % tiles, gh = ((blockIdx.x >> 3) / tiles) * 8 + (blockIdx.x & 7);
    if (gh >= P.n_gh) return;
    clamp_fp16();
    if (blockIdx.x == 0 && tid < 64) const_cast<uint4 *>(P.zeros)[tid] = make_uint4(0, 0, 0, 0);
    const int grp = gh / P.h, head = gh - grp * P.h;
    const int S = P.S, w = P.w, nrel = 2 * w - 1;
    const int q0 = tile * 128, qpos = q0 + wave * 32 + l32;
    const int32_t *sigma = P.sigma + (long)grp * P.sigma_stride;

    // this lane's query: its features, dO and delta
    bf16x8 qf[C::KS], of[C::KS];
    float delta = 0.f;
    int orow = -1, qrc = 0;                                  // row | column << 16 of the query's cell
    if (qpos < S) {
        const long slot = (long)grp * S + qpos;
        const int cell = sigma[qpos];
        qrc = cell / w;
        qrc |= (cell - qrc * w) << 16;
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

    // bias entries over the scale: rel Q^T, relative position t of the lane's query is its entry at_q + w - 1 - t
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
            const int p0 = (tab ? qrc >> 16 : qrc & 0xffff) + w - 1 - m0 - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int p = p0 - 8 * (r >> 2) - (r & 3);
                if ((unsigned)p < (unsigned)w) tq[tab * C::WK + p] = (_Float16)(u[r] * P.inv_scale);
            }
        }
    wave_lds_fence();
    if (qpos < P.SP) {
        _Float16 *to = P.tab + ((long)gh * P.SP + qpos) * C::EW + 8 * half;
#pragma unroll
        for (int c = 0; c < C::ES; ++c) *reinterpret_cast<f16x8 *>(to + 16 * c) = *reinterpret_cast<const f16x8 *>(tq + 16 * c + 8 * half);
    }
    const _Float16 *tl = tq + 8 * half;

    // stages of keys: the dense prefix, then (where a wave has a diagonal tile behind it) the workgroup's own 128
    bf16 *Ks = reinterpret_cast<bf16 *>(smem) + 4 * 32 * (C::TP + (C::KEEP ? 0 : 2 * C::VP)), *Vs = Ks + C::ROW_KEYS * C::KP;
    uint32_t *slices = reinterpret_cast<uint32_t *>(Vs + C::ROW_KEYS * C::VP);
    // where registers are short, the wave's queries and dO lie behind the bias entries
    bf16 *qs = reinterpret_cast<bf16 *>(smem) + 4 * 32 * C::TP + (wave * 32 + l32) * 2 * C::VP + half * 8, *os = qs + C::VP;
    if constexpr (!C::KEEP)
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
            *reinterpret_cast<bf16x8 *>(qs + ks * 16) = qf[ks];
            *reinterpret_cast<bf16x8 *>(os + ks * 16) = of[ks];
        }
    auto query = [&](int ks) { return C::KEEP ? qf[ks] : *reinterpret_cast<const bf16x8 *>(qs + ks * 16); };
    auto upstream = [&](int ks) { return C::KEEP ? of[ks] : *reinterpret_cast<const bf16x8 *>(os + ks * 16); };
    const int pre = min(P.n_pre * P.mask_block, S), pre_stages = (pre + C::ROW_KEYS - 1) / C::ROW_KEYS;
    const int own = (q0 + wave * 32) / P.mask_block;                                  // mask tile of the wave's queries
    const bool any_diagonal = min(q0 + 127, S - 1) / P.mask_block >= P.n_pre;
    const int stages = pre_stages + (any_diagonal ? (min(128, S - q0) + C::ROW_KEYS - 1) / C::ROW_KEYS : 0);
    const bool alive = q0 + wave * 32 < S;

    for (int i = tid; i < C::ROW_KEYS * (C::EW / 8); i += 256)                       // E starts empty
        *reinterpret_cast<uint4 *>(Ks + (i / (C::EW / 8)) * C::KP + D + (i % (C::EW / 8)) * 8) = make_uint4(0, 0, 0, 0);

    // Places of a thread's chunks are worked out again at every stage (`fresh`): kept, they would take registers from the accumulators.
    auto fresh = [&]() { int t = tid; asm volatile("" : "+v"(t)); return t; };
    constexpr int CH = D / 8, SIDE = C::ROW_KEYS * CH, NLOAD = (SIDE + 255) / 256;
    u32x4 kr[NLOAD], vr[NLOAD];
    int cell_next = -1;
    const bf16 *kbase = P.k + (long)grp * S * P.row_stride + (long)head * D, *vbase = P.v + (long)grp * S * P.row_stride + (long)head * D;
    auto stage_key = [&](int s) { return s < pre_stages ? s * C::ROW_KEYS : q0 + (s - pre_stages) * C::ROW_KEYS; };
    auto load = [&](int s) {
        const int key0 = stage_key(s), t = fresh();
#pragma unroll
        for (int i = 0; i < NLOAD; ++i) {
            const int id = t + 256 * i, row = id / CH, c = id - row * CH;
            kr[i] = vr[i] = u32x4{ 0, 0, 0, 0 };
            if (id < SIDE && key0 + row < S) {               // (a group's rows lie within 2^31 bytes)
                const uint32_t at = (uint32_t)(key0 + row) * (uint32_t)P.row_stride + c * 8;
                kr[i] = *reinterpret_cast<const u32x4 *>(kbase + at);
                vr[i] = *reinterpret_cast<const u32x4 *>(vbase + at);
            }
        }
        if (tid < C::ROW_KEYS) cell_next = key0 + tid < S ? sigma[key0 + tid] : -1;
    };
    int ones = -1;                                           // where this thread's key has its ones: row | column << 8
    auto store = [&]() {
        const int t = fresh();
#pragma unroll
        for (int i = 0; i < NLOAD; ++i) {
            const int id = t + 256 * i, row = id / CH, c = id - row * CH;
            if (id < SIDE) {
                *reinterpret_cast<u32x4 *>(Ks + row * C::KP + c * 8) = kr[i];
                *reinterpret_cast<u32x4 *>(Vs + row * C::VP + c * 8) = vr[i];
            }
        }
        if (wave == 0 && tid < C::ROW_KEYS) {
            uint16_t *e = reinterpret_cast<uint16_t *>(Ks + tid * C::KP + D);
            if (ones >= 0) e[ones & 0xff] = e[ones >> 8] = 0;
            ones = -1;
            if (cell_next >= 0) {
                const int row = cell_next / w, col = C::WK + cell_next - row * w;
                ones = row | col << 8;
                e[row] = e[col] = 0x3c00;
            }
            // slices of 16 entries: where all keys of a block have their ones in the same two (rows and columns), the others are left out
            const int s2 = ones >> 4 & 0xf0f, first = __shfl(s2, lane & 32, 64);
            const uint64_t differ = __builtin_amdgcn_ballot_w64(ones >= 0 && s2 != first);
            if ((lane & 31) == 0) slices[lane >> 5] = (uint32_t)(differ >> (lane & 32)) == 0 ? (uint32_t)s2 | 0x10000u : 0u;
        }
    };

    f32x16 acc[C::CT];
#pragma unroll
    for (int t = 0; t < C::CT; ++t) acc[t] = zero16();
    asm volatile("" : "+v"(qrc));
    float m = -INFINITY, l = 0.f;
    __syncthreads();
    if (stages > 0) load(0);
    for (int s = 0; s < stages; ++s) {
        LDS_BARRIER();                                       // every wave is done with the previous stage
        store();
        LDS_BARRIER();
        const int key0 = stage_key(s);
        if (s + 1 < stages) load(s + 1);
#pragma unroll 1
        for (int b = 0; b < C::ROW_KEYS / 32; ++b) {
            const int kb = key0 + 32 * b;
            const bool active = alive && kb < S && (s < pre_stages ? kb < pre : own >= P.n_pre && kb / P.mask_block == own);
            if (!active) continue;                           // the same for the whole wave
            const bf16 *kblk = Ks + 32 * b * C::KP, *vblk = Vs + 32 * b * C::VP;
            const bf16 *kl = kblk + l32 * C::KP + half * 8, *vl = vblk + l32 * C::VP + half * 8;
            const uint32_t two = NT > 1 ? __builtin_amdgcn_readfirstlane(slices[b]) : 0;
            const int rs = two & 0xff, cs = (two >> 8) & 0xff;
            f32x16 sc = zero16();
            if (NT > 1 && two != 0) {
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(kl + D + rs * 16), *reinterpret_cast<const f16x8 *>(tl + 16 * rs), sc, 0, 0, 0);
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(kl + D + cs * 16), *reinterpret_cast<const f16x8 *>(tl + 16 * cs), sc, 0, 0, 0);
            } else {
#pragma unroll
                for (int c = 0; c < C::ES; ++c) {
                    if (!C::KEEP && c % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(kl + D + c * 16), *reinterpret_cast<const f16x8 *>(tl + 16 * c), sc, 0, 0, 0);
                }
            }
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(kl + ks * 16), query(ks), sc, 0, 0, 0);
            f32x16 dp = zero16();
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(vl + ks * 16), upstream(ks), dp, 0, 0, 0);
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
                for (int t = 0; t < C::CT; ++t) {
                    if (!C::KEEP) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[t][r] *= alpha;
                }
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[r], P.scale_log2e, -m));
                l += p;
                dp[r] = p * (dp[r] - delta);
            }
            const bf16x8 ds[2] = { half_of(dp, 0), half_of(dp, 1) };
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int c = 0; c < C::CT; ++c) {
                    // eleven tiles of accumulators leave no registers for operands read further ahead
                    if (!C::KEEP && c % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(kblk, C::KP, t, c, D + C::EW - 4), ds[t], acc[c], 0, 0, 0);
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
    for (int c = 0; c < C::CT; ++c) {
        if (!C::KEEP) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const bool is_g = c * 32 + 8 * g >= D;                                    // (a group of eight columns is on one side)
            const float f = is_g ? inv * 128.f : inv * P.scale;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = alive ? acc[c][4 * g + e] * f : 0.f;
                acc[c][4 * g + e] = v;
                if (is_g && c * 32 + 8 * g < D + C::EW) most = fmaxf(most, fabsf(v));
            }
        }
    }

    bf16 *gr = reinterpret_cast<bf16 *>(smem) + wave * 32 * C::RP, *rel = reinterpret_cast<bf16 *>(smem) + 4 * 32 * C::RP;
    bf16 *mine = gr + l32 * C::RP;
    const int relrows = (nrel + 15) / 16 * 16;
    __syncthreads();
    if (P.gsum) {
        // G for the tables' gradient, in fp16 over a power of two that puts a query's largest entry at 2^14 or more: eight times as exact as bf16, in the same bytes
        most = fmaxf(most, __shfl_xor(most, 32, 64));
        const int e = min(max((int)(__float_as_uint(most) >> 23) - 127, -100), 127);
        const float unit = __uint_as_float((uint32_t)(e - 14 + 127) << 23), over = __uint_as_float((uint32_t)(14 - e + 127) << 23);
#pragma unroll
        for (int c = 0; c < C::CT; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = c * 32 + 8 * g - D;
                if (col < 0 || col >= C::EW) continue;
                f16x4 v = { (_Float16)(acc[c][4 * g] * over), (_Float16)(acc[c][4 * g + 1] * over), (_Float16)(acc[c][4 * g + 2] * over), (_Float16)(acc[c][4 * g + 3] * over) };
                *reinterpret_cast<f16x4 *>(mine + col + 4 * half) = v;
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
        for (int i = tid; i < relrows * CH; i += 256) {
            const int row = i / CH, c = i - row * CH;
            u32x4 v = { 0, 0, 0, 0 };
            if (row < nrel) v = *reinterpret_cast<const u32x4 *>((tab ? P.rel_w : P.rel_h) + (long)row * D + c * 8);
            *reinterpret_cast<u32x4 *>(rel + row * C::VP + c * 8) = v;
        }
        for (int i = 8 * half; i < relrows; i += 16) *reinterpret_cast<uint4 *>(mine + i) = make_uint4(0, 0, 0, 0);
        const int t0 = (tab ? qrc >> 16 : qrc & 0xffff) + w - 1;
        f32x16 add[C::DT];
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt) add[dt] = zero16();
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            wave_lds_fence();
#pragma unroll
            for (int c = 0; c < C::CT; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (c * 32 + 8 * (r >> 2) < D + tab * C::WK || c * 32 + 8 * (r >> 2) >= D + (tab + 1) * C::WK) continue;
                    const int y = c * 32 + 8 * (r >> 2) + (r & 3) + 4 * half - D - tab * C::WK;
                    const bf16 v = (bf16)acc[c][r];
                    if (y < w) mine[t0 - y] = v;
                    if (part == 0) acc[c][r] -= (float)v;
                }
            if (part == 0) __syncthreads();
            else wave_lds_fence();
            for (int t = 0; t < relrows / 16; ++t) {
                const bf16x4 a = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 4 * half), b = *reinterpret_cast<const bf16x4 *>(mine + 16 * t + 8 + 4 * half);
                const bf16x8 g8 = { a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt) add[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transposed(rel + 16 * t * C::VP, C::VP, 0, dt, D - 4), g8, add[dt], 0, 0, 0);
            }
        }
        mfma_settle();
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (dt * 32 + 8 * (r >> 2) < D) acc[dt][r] += add[dt][r];             // (the rest of a last tile that D fills by half is GH)
    }
    __syncthreads();
    store_rows<D>(acc, reinterpret_cast<bf16 *>(smem) + wave * 32 * C::VP, P.dq + (long)grp * S * P.grad_stride + (long)head * D, P.grad_stride, qpos < S ? qpos : -1);
}

// ---------------------------------------------------------------- columns
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
__device__ __forceinline__ void request(uint32_t lds, uint32_t off, const void *base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void request(uint32_t lds, const void *src)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(src) : "m0", "memory");
}

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
    auto ones = [&](int i) {                                 // entries of a slice: a one at place i, if that is one of its eight
        u32x4 e;
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = i >> 1 == j ? (i & 1 ? 0x3c000000u : 0x3c00u) : 0u;
        return __builtin_bit_cast(f16x8, e);
    };
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
    const bool prefix = kb / P.mask_block < P.n_pre, alive = kb < S;

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

    // places of this lane's operands in a buffer: rows l32 of a block by 16-byte chunks, and transposed (rows +0 and +8)
    int ka[C::KS], tr[CH == 8 ? 2 : 1][2];
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) ka[ks] = l32 * St::QP + ((2 * ks + half) ^ swizzle<CH>(l32)) * 16;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int li = lane & 15, r = 8 * u + 4 * half + (li >> 2);
#pragma unroll
        for (int dt = 0; dt < (CH == 8 ? 2 : 1); ++dt) {
            const int f0 = (D == 16 ? 0 : 16 * ((lane >> 4) & 1)) + 4 * (li & 3);
            tr[dt][u] = r * St::QP + ((4 * dt + (f0 >> 3)) ^ swizzle<CH>(r)) * 16 + (f0 & 7) * 2;
        }
    }
    auto transpose = [&](int base, int t, int dt) {
        bf16x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            int at = tr[CH == 8 ? dt : 0][u] + base + 16 * t * St::QP + (CH == 8 ? 0 : dt * 64);
            if (D == 80 && dt == 2) at -= ((lane >> 4) & 1) * 32;       // the other half of a last tile that D fills by half: the same columns, not used
            v[u] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(smem + at));
        }
        return bf16x8{ v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3] };
    };

    int buf = 0;
    if (first < last) stage(first, 0);
    for (int q0 = first; q0 < last; q0 += St::QUERIES, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        LDS_BARRIER();                                       // this stage has landed, and nobody reads the other buffer any more
        if (q0 + St::QUERIES < last) stage(q0 + St::QUERIES, buf ^ 1);
#pragma unroll 1
        for (int b = 0; b < St::QUERIES / 32; ++b) {
            const int qb = q0 + 32 * b;
            if (!alive || qb >= last || !(prefix || qb / P.mask_block == kb / P.mask_block)) continue;     // the same for the whole wave
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
            for (int ks = 0; ks < C::KS; ++ks) p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(smem + at + St::Q + ka[ks]), kf[ks], p, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) ds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(smem + at + St::O + ka[ks]), vf[ks], ds, 0, 0, 0);
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
                    dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transpose(at + St::O, t, dt), pf, dv[dt], 0, 0, 0);
                    dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(transpose(at + St::Q, t, dt), df, dk[dt], 0, 0, 0);
                }
            }
        }
    }
}

template <int D, int NT>
__global__ void __launch_bounds__(256, NT < 8 ? 2 : 1)
attn_backward_columns_kernel(BwdParams P, ColWork work, float *__restrict__ parts)
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
    const int S = P.S, w = P.w;
    const int k0 = tile * 128, kb = k0 + wave * 32, kpos = kb + l32;
    const int at = min(kpos, S - 1);                         // keys past the end repeat the last one; their results are not stored
    bf16x8 kf[C::KS], vf[C::KS];
    const long o = ((long)grp * S + at) * P.row_stride + (long)head * D + half * 8;
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks) {
        kf[ks] = *reinterpret_cast<const bf16x8 *>(P.k + o + ks * 16);
        vf[ks] = *reinterpret_cast<const bf16x8 *>(P.v + o + ks * 16);
    }
    const int cell = P.sigma[(long)grp * P.sigma_stride + at], row = cell / w, col = C::WK + cell - row * w;
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
attn_backward_join_kernel(BwdParams P, ColWork work, int D, const float4 *__restrict__ parts, long n)
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
// A unit is 32 queries of one (group, head).  A workgroup adds up those of a slice in registers: result [relative position of both tables][feature].
template <int D, int NT>
__host__ __device__ constexpr size_t tables_lds_bytes()
{
    using C = BwdCfg<D, NT>;
    return (size_t)32 * (2 * (4 * C::WK + 8) + C::VP) * 2;
}

template <int D, int NT>
__global__ void __launch_bounds__(256, NT >= 8 ? 1 : 2)
attn_backward_tables_kernel(BwdParams P, int units_per_gh, long units, float *__restrict__ parts)
{
    using C = BwdCfg<D, NT>;
    constexpr int TT = 4 * C::WK / 32;                       // 32-row tiles of relative positions
    constexpr int MINE = (TT + 3) / 4, GP = 4 * C::WK + 8;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    bf16 *Gs = reinterpret_cast<bf16 *>(smem), *Qs = Gs + 2 * 32 * GP;       // G is the sum of two bf16, one [32][GP] behind the other
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l32 = lane & 31, half = lane >> 5;
    const int S = P.S, w = P.w;
    f32x16 acc[MINE][C::DT];
#pragma unroll
    for (int i = 0; i < MINE; ++i)
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt) acc[i][dt] = zero16();
    const long per = (units + gridDim.x - 1) / gridDim.x, u1 = min((long)(blockIdx.x + 1) * per, units);
    for (long u = blockIdx.x * per; u < u1; ++u) {
        const int gh = (int)(u / units_per_gh), q0 = (int)(u - (long)gh * units_per_gh) * 32, grp = gh / P.h, head = gh - grp * P.h;
        __syncthreads();
        for (int i = tid; i < 2 * 32 * (GP / 8); i += 256) *reinterpret_cast<uint4 *>(Gs + i * 8) = make_uint4(0, 0, 0, 0);
        constexpr int CH = D / 8;
        for (int i = tid; i < 32 * CH; i += 256) {
            const int row = i / CH, c = i - row * CH;
            uint4 v = make_uint4(0, 0, 0, 0);
            if (q0 + row < S) {
                const long slot = (long)grp * S + q0 + row;
                if (!P.out_rows || P.out_rows[slot] >= 0) v = *reinterpret_cast<const uint4 *>(P.q + slot * P.row_stride + (long)head * D + c * 8);
            }
            *reinterpret_cast<uint4 *>(Qs + row * C::VP + c * 8) = v;
        }
        __syncthreads();
        for (int i = tid; i < 32 * (C::EW / 8); i += 256) {
            const int row = i / (C::EW / 8), c = i % (C::EW / 8), tab = c * 8 >= C::WK, y0 = c * 8 - tab * C::WK;
            if (q0 + row >= S || y0 >= w) continue;
            const int cell = P.sigma[(long)grp * P.sigma_stride + q0 + row], r = cell / w, t0 = (tab ? cell - r * w : r) + w - 1 - y0;
            const f16x8 g = *reinterpret_cast<const f16x8 *>(P.gsum + ((long)gh * S + q0 + row) * C::EW + c * 8);
            const float unit = P.gunit[(long)gh * S + q0 + row];
            bf16 *to = Gs + row * GP + tab * 2 * C::WK + t0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (y0 + e >= w) continue;
                const float v = (float)g[e] * unit;
                const bf16 hi = (bf16)v;
                to[-e] = hi;
                to[32 * GP - e] = (bf16)(v - (float)hi);
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            bf16x8 qt[C::DT];
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt) qt[dt] = transposed(Qs, C::VP, t, dt, D - 4);
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                if (wave * MINE + i >= TT) continue;
                const bf16x8 hi = transposed(Gs, GP, t, wave * MINE + i, GP - 4), lo = transposed(Gs + 32 * GP, GP, t, wave * MINE + i, GP - 4);
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt) {
                    acc[i][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, qt[dt], acc[i][dt], 0, 0, 0);
                    acc[i][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, qt[dt], acc[i][dt], 0, 0, 0);
                }
            }
        }
    }
    mfma_settle();
    // result: lane <-> feature, register <-> relative position
    float *to = parts + (long)blockIdx.x * 4 * C::WK * D;
#pragma unroll
    for (int i = 0; i < MINE; ++i)
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int t = (wave * MINE + i) * 32 + 8 * (r >> 2) + 4 * half + (r & 3), c = dt * 32 + l32;
                if (wave * MINE + i < TT && c < D) to[(long)t * D + c] = acc[i][dt][r];
            }
}

// [n][2][2 WK][D] sums of slices -> bf16 tables of nrel rows.  A workgroup adds up 32 columns: eight lanes with 16 bytes each, 32 slices of the n.
__global__ void __launch_bounds__(256)
attn_backward_table_sums_kernel(const float4 *__restrict__ parts, int n, int table, int used, bf16 *__restrict__ drel_h, bf16 *__restrict__ drel_w)
{
    __shared__ float4 lds[256];
    const int c = threadIdx.x & 7, slice = threadIdx.x >> 3;
    const int col = (blockIdx.x * 8 + c) * 4;                // element of the table
    const bool in = col < used;
    const long at = ((long)blockIdx.y * table + min(col, used - 4)) / 4;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int r = slice; r < n; r += 32) {
        const float4 t = parts[(long)r * 2 * table / 4 + at];
        a.x += t.x; a.y += t.y; a.z += t.z; a.w += t.w;
    }
    lds[threadIdx.x] = a;
    __syncthreads();
#pragma unroll
    for (int half = 16; half > 0; half >>= 1) {
        if (slice < half) {
            const float4 t = lds[threadIdx.x + half * 8];
            a.x += t.x; a.y += t.y; a.z += t.z; a.w += t.w;
            lds[threadIdx.x] = a;
        }
        __syncthreads();
    }
    if (slice == 0 && in) *reinterpret_cast<uint2 *>((blockIdx.y ? drel_w : drel_h) + col) = make_uint2(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w));
}

// ---------------------------------------------------------------- launches
inline int entry_tiles(int w) { return w <= 16 ? 1 : w <= 32 ? 2 : w <= 64 ? 4 : 8; }
inline long table_units(int S, long n_gh) { return n_gh * ssam_div_up(S, 32); }
inline int table_slices(long units) { return (int)(units < 256 ? units : 256); }

// Tiles of the dense prefix have all queries to walk: with few of them, a slice of the queries each, until there are two workgroups to a CU.
constexpr int COL_SLOTS = 512;
inline int column_splits(long heavy, int S)
{
    const long most = (S + 255) / 256, n = COL_SLOTS / (heavy > 0 ? heavy : 1);
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

struct BwdWorkspace { size_t zeros, tab, gsum, gunit, lse, delta, parts, total; };
inline BwdWorkspace workspace_layout(int groups, int S, int w, int h, int d)
{
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    const size_t rows = (size_t)groups * h * ((S + 31) / 32 * 32), entries = rows * 32 * entry_tiles(w) * 2;
    BwdWorkspace o;
    o.zeros = 0;
    o.tab = 1024;
    o.gsum = o.tab + up(entries + 32 * 64 * entry_tiles(w));                        // (the last stage reads up to 32 rows past the end)
    o.gunit = o.gsum + up(entries);
    o.lse = o.gunit + up(rows * 4);
    o.delta = o.lse + up(rows * 4 + 128);
    o.parts = o.delta + up(rows * 4 + 128);
    // sums of slices: of the tables' gradients, and before those of dK and dV of at most COL_SLOTS tiles
    const size_t tables = (size_t)table_slices(table_units(S, (long)groups * h)) * 64 * entry_tiles(w) * d * 4;
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
    const size_t lds = rows_lds_bytes<D, NT>(nrel);
    if (int rc = allow_lds(attn_backward_rows_kernel<D, NT>, lds); rc != SSAM_OK) return rc;
    if (int rc = allow_lds(attn_backward_columns_kernel<D, NT>, columns_lds_bytes<D, NT>()); rc != SSAM_OK) return rc;
    hipLaunchKernelGGL((attn_backward_rows_kernel<D, NT>), dim3(grid), dim3(256), lds, st, P, tiles);
    SSAM_CHECK_LAUNCH();
    ColWork work;
    work.gh8 = ssam_div_up(P.n_gh, 8);
    work.heavy = ssam_div_up(min(P.n_pre * P.mask_block, P.S), 128);                // (windows: mask tiles are 32, a wave looks at its own)
    work.light = tiles - work.heavy;
    work.splits = P.mask_block == 128 ? column_splits((long)work.heavy * P.n_gh, P.S) : 1;
    hipLaunchKernelGGL((attn_backward_columns_kernel<D, NT>), dim3((unsigned)(8L * work.gh8 * (work.heavy * work.splits + work.light))), dim3(256),
                       (columns_lds_bytes<D, NT>()), st, P, work, parts);
    SSAM_CHECK_LAUNCH();
    if (work.splits > 1 && work.heavy > 0) {
        const long n = (long)P.n_gh * work.heavy * 128 * (2 * D / 8);
        hipLaunchKernelGGL(attn_backward_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, P, work, D, (const float4 *)parts, n);
        SSAM_CHECK_LAUNCH();
    }
    if (drel_h) {
        const int per = ssam_div_up(P.S, 32), slices = table_slices(table_units(P.S, P.n_gh)), used = nrel * D;
        hipLaunchKernelGGL((attn_backward_tables_kernel<D, NT>), dim3(slices), dim3(256), (tables_lds_bytes<D, NT>()), st, P, per, table_units(P.S, P.n_gh), parts);
        SSAM_CHECK_LAUNCH();
        hipLaunchKernelGGL(attn_backward_table_sums_kernel, dim3(ssam_div_up(used, 32), 2), dim3(256), 0, st, (const float4 *)parts, slices,
                           2 * BwdCfg<D, NT>::WK * D, used, drel_h, drel_w);
        SSAM_CHECK_LAUNCH();
    }
    return SSAM_OK;
}

template <int D>
int launch_backward(const BwdParams &P, float *parts, bf16 *drel_h, bf16 *drel_w, hipStream_t st)
{
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
    // bias entries are held over the scale in fp16: up to 128 as a logit at the least of these, spaced by 2^-15 of one at the most
    if (scale < 0x1p-9f || scale > 0x1p9f) return SSAM_EUNSUPPORTED;
    if (mask_block == 32 ? S > 224 : mask_block != 128 || S > 16384) return SSAM_EUNSUPPORTED;
    if ((long)S * row_stride * 2 > 0x7fffffffL) return SSAM_EUNSUPPORTED;              // 32-bit offsets within a group
    if (d != 16 && d != 32 && d != 64 && d != 80) return SSAM_EUNSUPPORTED;
    if ((long)groups * h > 0x7ffffff0L || (long)ssam_div_up(S, 128) * ((long)groups * h + 7) > 0x7fffffffL / 256) return SSAM_EUNSUPPORTED;
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
    P.mask_block = mask_block;
    P.n_pre = ssam_prefix_tiles(ssam_div_up(S, mask_block), r);
    P.scale = scale;
    P.scale_log2e = scale * LOG2E;
    P.tab = (_Float16 *)(ws + at.tab);
    P.inv_scale = 1.f / scale;
    P.inv_scale_log2e = 1.f / P.scale_log2e;
    P.gsum = drel_h ? (_Float16 *)(ws + at.gsum) : nullptr;
    P.gunit = (float *)(ws + at.gunit);
    P.lse = (float *)(ws + at.lse);
    P.delta = (float *)(ws + at.delta);
    P.zeros = (const uint4 *)(ws + at.zeros);
    P.SP = (S + 31) / 32 * 32;
    float *parts = (float *)(ws + at.parts);
    hipStream_t st = (hipStream_t)stream;
    switch (d) {
    case 16: return launch_backward<16>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    case 32: return launch_backward<32>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    case 64: return launch_backward<64>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    default: return launch_backward<80>(P, parts, (bf16 *)drel_h, (bf16 *)drel_w, st);
    }
}
