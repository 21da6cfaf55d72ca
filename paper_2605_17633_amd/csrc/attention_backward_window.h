// Gradients of attention where a group's keys and queries fit into LDS together (S <= 224: windows): one workgroup does all of a (group, head).
//
// Q, K, V and dO are read once, and what the walks hand to each other (bias entries, statistics, G) never leaves the CU: the three launches that grids take read the features
// three times.  A workgroup stays on its CU and takes one (group, head) after the other, so that the tables' gradient, (G at relative positions)^T Q, is added up in registers.
//   rows     wave i has the queries of tile i (32): scores, P, dS over its keys; leaves dQ, G, -log sum exp
//   tables   a 32 x 32 tile of drel a wave, over all queries
//   columns  every active (query tile, key tile) once more with P from the statistics.  Keys of the dense prefix see all queries: their query tiles are dealt out to several waves,
//            whose sums are added through LDS in order; the others see one tile of the mask
// Why eight waves and all of LDS: the features of a (group, head) of 14 x 14 x 80 are 126 KB, so one workgroup has the CU, and two waves to a SIMD have 256 registers each.
// 1600 (group, head) of 14 x 14 x 80 (four images, 16 heads, density 0.5) take 223 us, 300 of 64 features 52; in rows, columns and tables as for grids they took 336 and 66.  A (group, head)
// is a chain of phases between barriers, 32 us of the former: 13 until its rows are there (250 MB read and 150 written at 1.8 TB/s over the whole), 3 bias entries, 4 to 6 rows, 3 G,
// 4 dQ and tables, 4 to 6 columns; the matrix pipe is busy 15 % of the time.
// The space of K and V holds G (as the sum of two bf16) and the relative positions' features once the rows are done; that of E then holds the bias entries T.
#pragma once

namespace {

constexpr int WIN_ROWS = 224, WIN_TILES = WIN_ROWS / 32, WIN_WAVES = 8, WIN_GROUPS = 256;

// Who has which keys on columns.  A key tile of the dense prefix sees all query tiles, `per` of them a share, and a wave has one share; the waves left over have the tiles behind
// the prefix, which see one tile of the mask, in turn (with none left over, the last waves have one each besides).  So few shares that the longest wave has least.
struct WindowWork { int shares, per; };
inline WindowWork window_work(int tiles, int heavy, int mask_tile)
{
    WindowWork best = { 1, tiles };
    int least = 1 << 30;
    for (int want = 1; want <= tiles && heavy; ++want) {
        const int per = (tiles + want - 1) / want, shares = (tiles + per - 1) / per, others = WIN_WAVES - heavy * shares, n = tiles - heavy, light = mask_tile < tiles ? mask_tile : tiles;
        if (others < 0) break;
        const int longest = n == 0 ? per : others == 0 ? per + light : per > (n + others - 1) / others * light ? per : (n + others - 1) / others * light;
        if (longest < least) {
            least = longest;
            best = { shares, per };
        }
    }
    return best;
}

template <int D>
struct WinCfg {
    using C = BwdCfg<D, 1>;
    static constexpr int RB = D * 2, EB = C::EW * 2, GB = 128;                      // rows, in bytes; of G: 2 x 32 relative positions
    static constexpr int Q = 0, O = Q + WIN_ROWS * RB, K = O + WIN_ROWS * RB, V = K + WIN_ROWS * RB;
    static constexpr int G = K, GPART = WIN_ROWS * GB, REL = G + 2 * GPART, REND = REL + 2 * 32 * C::VP * 2;
    static constexpr int VEND = V + WIN_ROWS * RB, E = VEND > REND ? VEND : REND;
    static constexpr int L = E + WIN_ROWS * EB, N = L + WIN_ROWS * 4, TOTAL = N + WIN_ROWS * 4;
    static constexpr int PART = 32 * 2 * D * 4;                                     // dK and dV of a key tile
    static_assert(TOTAL <= 160 * 1024 && (WIN_TILES - 1) * PART <= TOTAL, "");
};

// 32 result rows [column tiles]^T straight to memory: of two groups of eight features a half-wave takes one each, 16 bytes a lane
template <int D>
__device__ __forceinline__ void store_direct(const f32x16 *acc, bf16 *row, bool stored)
{
    const int half = lane_now() >> 5;
#pragma unroll
    for (int c = 0; c < D / 8; c += 2) {
        uint32_t x[2][2];
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[g][i] = pack_bf16x2(acc[(c + g) / 4][(c + g) % 4 * 4 + 2 * i], acc[(c + g) / 4][(c + g) % 4 * 4 + 2 * i + 1]);
        const auto a = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false), b = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
        if (stored) *reinterpret_cast<uint4 *>(row + (c + half) * 8) = make_uint4(a[0], b[0], a[1], b[1]);
    }
}

template <int D>
__global__ void __launch_bounds__(64 * WIN_WAVES, 2)
backward_windows_kernel(BwdParams P, WindowWork work, bool tables, float *__restrict__ parts)
{
    using C = BwdCfg<D, 1>;
    using W = WinCfg<D>;
    constexpr int CH = D / 8, EC = W::EB / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int S = P.S, w = P.w, nrel = 2 * w - 1, tiles = (S + 31) / 32, mb = P.mask_block == 128 ? 2 : 0;                        // (log of a mask tile's 32s)
    const int heavy = min(P.n_pre << mb, tiles);
    const bool alive = wave < tiles;
    // this wave's work on columns: a tile behind the prefix, and a share of a tile of the prefix
    const int shares = work.shares, per = work.per, share = wave % shares, dense = wave / shares, others = WIN_WAVES - heavy * shares;
    const int light = others == 0 ? heavy + WIN_WAVES - 1 - wave : wave >= WIN_WAVES - others ? heavy + wave - (WIN_WAVES - others) : tiles, step = others ? others : WIN_WAVES;
    // (tiles; a light one >= tiles, a dense one >= heavy: none)

    f32x16 table = zero16();                                  // drel of table wave / DT, features 32 (wave % DT) ..

#pragma unroll 1
    for (long first = 0; first < P.n_gh; first += gridDim.x) {
        // neighbours of a group share cache lines: they run on one XCD (workgroup b sits on XCD b & 7)
        const int gh = (int)first + ((gridDim.x & 7) == 0 ? (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) : (int)blockIdx.x);
        if (gh >= P.n_gh) break;                             // the same for the whole workgroup
        const int grp = gh / P.h, head = gh - grp * P.h;
        const int lane = lane_now(), tid = wave * 64 + lane, l32 = lane & 31, half = lane >> 5, pos = wave * 32 + l32;
        const int esw = swizzle<EC>(l32) ^ half;
        const bf16 *rel_h = P.rel_h, *rel_w = P.rel_w;
        asm volatile("" : "+s"(rel_h), "+s"(rel_w));           // (read again for every (group, head): kept, their rows would take 40 registers)
        const int rc = row_col(P.sigma + (long)grp * P.sigma_stride, pos, P), row = rc & 0xffff, col = rc >> 16;
        // Features of all rows, 16 bytes a thread and whole rows by neighbouring threads (a wave that reads its own operands' places asks for twice as many lines, and the requests are
        // what bounds this); parts of dO . O go where E comes to lie.  Rows past the end, and of queries whose output is dropped, are zeros.
        constexpr int LOADS = (WIN_ROWS * CH + 64 * WIN_WAVES - 1) / (64 * WIN_WAVES);
        bf16x8 rf[2][C::KS];
        {
            u32x4 x[5][LOADS];
            uint32_t live = 0;                                // bit k: the row exists, bit 16 + k: and its output is not dropped
            int outs[LOADS];
            if (P.out_rows) {
#pragma unroll
                for (int k = 0; k < LOADS; ++k) outs[k] = P.out_rows[(long)grp * S + min((tid + 64 * WIN_WAVES * k) / CH, S - 1)];
            } else {
#pragma unroll
                for (int k = 0; k < LOADS; ++k) outs[k] = 0;
            }
            // (no branch around a load: all of them are asked for before the first is waited for)
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int i = tid + 64 * WIN_WAVES * k, r = i / CH, c = i - r * CH;
                const long at = (long)grp * S + min(r, S - 1), from = at * P.row_stride + (long)head * D + c * 8;
                const long place = (P.out_rows ? (long)max(outs[k], 0) : at) * ((long)P.h * D) + (long)head * D + c * 8;
                live |= r < S ? outs[k] >= 0 ? 0x10001u << k : 1u << k : 0u;
                x[0][k] = *reinterpret_cast<const u32x4 *>(P.k + from);
                x[1][k] = *reinterpret_cast<const u32x4 *>(P.v + from);
                x[2][k] = *reinterpret_cast<const u32x4 *>(P.q + from);
                x[3][k] = *reinterpret_cast<const u32x4 *>(P.dout + place);
                x[4][k] = *reinterpret_cast<const u32x4 *>(P.out + place);
            }
#pragma unroll
            for (int tab = 0; tab < 2; ++tab)
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) rf[tab][ks] = *reinterpret_cast<const bf16x8 *>((tab ? rel_w : rel_h) + (long)min(l32, nrel - 1) * D + half * 8 + ks * 16);
            __syncthreads();                                 // nobody reads the (group, head) before any more
#pragma unroll
            for (int k = 0; k < LOADS; ++k) {
                const int i = tid + 64 * WIN_WAVES * k, r = i / CH, c = i - r * CH;
                if (r >= WIN_ROWS) continue;
                unsigned char *to = smem + r * W::RB + (c ^ swizzle<CH>(r)) * 16;
                const bf16x8 d = __builtin_bit_cast(bf16x8, x[3][k]), o = __builtin_bit_cast(bf16x8, x[4][k]);
                float dot = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) dot = fmaf((float)d[e], (float)o[e], dot);
#pragma unroll
                for (int n = 0; n < 4; ++n) x[n][k] = live >> (n < 2 ? k : 16 + k) & 1 ? x[n][k] : u32x4{ 0, 0, 0, 0 };
                *reinterpret_cast<u32x4 *>(to + W::K) = x[0][k];
                *reinterpret_cast<u32x4 *>(to + W::V) = x[1][k];
                *reinterpret_cast<u32x4 *>(to + W::Q) = x[2][k];
                *reinterpret_cast<u32x4 *>(to + W::O) = x[3][k];
                *reinterpret_cast<float *>(smem + W::E + r * W::EB + c * 4) = live >> (16 + k) & 1 ? dot : 0.f;
            }
        }
        const Straight<CH> fa(lane);
        bf16x8 qf[C::KS], of[C::KS];
        f16x8 bt[2] = { { 0, 0, 0, 0, 0, 0, 0, 0 }, { 0, 0, 0, 0, 0, 0, 0, 0 } };
        float delta = 0.f;
        __syncthreads();
        // (a wave behind the last tile reads what lies behind, so that these are not undefined on any way: the compiler would keep the last ones)
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
            qf[ks] = fa(smem, W::Q + 32 * wave * W::RB, ks);
            of[ks] = fa(smem, W::O + 32 * wave * W::RB, ks);
        }
        if (alive) {
            unsigned char *mine = smem + W::E + pos * W::EB;
#pragma unroll
            for (int c = 0; c < CH; c += 2) delta += *reinterpret_cast<const float *>(mine + (c + half) * 4);
            delta += other_half(delta);
            const int usw = l32 >> 2 & 7;                     // (rows of 64 bytes: four eight-byte places apart share banks without it)
            // bias entries over the scale: rel Q^T, whose 32 rows hold all relative positions (w <= 14) and fill the query's row of E for now; entry y is position t0 - y
#pragma unroll
            for (int tab = 0; tab < 2; ++tab) {
                f32x16 u = zero16();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(rf[tab][ks], qf[ks], u, 0, 0, 0);
                mfma_settle();
                wave_lds_fence();
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *reinterpret_cast<f16x4 *>(mine + ((2 * g + half) ^ usw) * 8) = f16x4{ (_Float16)(u[4 * g] * P.inv_scale), (_Float16)(u[4 * g + 1] * P.inv_scale), (_Float16)(u[4 * g + 2] * P.inv_scale),
                                                                                      (_Float16)(u[4 * g + 3] * P.inv_scale) };
                wave_lds_fence();
                const int t0 = (tab ? col : row) + w - 1 - 8 * half;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = max(t0 - e, 0);
                    const _Float16 x = *reinterpret_cast<const _Float16 *>(mine + ((t >> 2) ^ usw) * 8 + (t & 3) * 2);
                    bt[tab][e] = 8 * half + e < w ? x : (_Float16)0.f;
                }
                bt[tab] = bounded(bt[tab]);
            }
            wave_lds_fence();
            // E: a half-wave has the row's 16 entries, the other one the column's
#pragma unroll
            for (int c = 0; c < 2; ++c) *reinterpret_cast<f16x8 *>(mine + ((2 * half + c) ^ swizzle<EC>(l32)) * 16) = ones((half ? col : row) - 8 * c, P.one);
        }
        __syncthreads();
        const Transposed<CH> ft(lane);

        // ---- rows
        const Transposed<EC> et(lane);
        // (of 80 features Q and dO come back from LDS for every block: registers for them are short)
        f32x16 acc[C::DT], gt = zero16();
#pragma unroll
        for (int t = 0; t < C::DT; ++t) acc[t] = zero16();
        float m = -INFINITY, l = 0.f;
#pragma unroll 1
        for (int j = 0; j < tiles; ++j) {
            if (!alive || !(j < heavy || j >> mb == wave >> mb)) continue;         // the same for the whole wave
            const int at = 32 * j * W::RB;
            const unsigned char *el = smem + W::E + (32 * j + l32) * W::EB;
            f32x16 sc = zero16(), dp = zero16();
            if (D == 80) asm volatile("" : "+v"(bt[0]), "+v"(bt[1]));       // (else the compiler puts them into scratch memory)
            sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(el + esw * 16), bt[0], sc, 0, 0, 0);
            sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(el + (2 ^ esw) * 16), bt[1], sc, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa(smem, at + W::K, ks), D == 80 ? fa(smem, W::Q + 32 * wave * W::RB, ks) : qf[ks], sc, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa(smem, at + W::V, ks), D == 80 ? fa(smem, W::O + 32 * wave * W::RB, ks) : of[ks], dp, 0, 0, 0);
            const int left = S - 32 * j - 4 * half;           // keys past the end
            float mx = -INFINITY;
            if (32 * j + 32 > S)
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[r] = 8 * (r >> 2) + (r & 3) < left ? sc[r] : -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[r]);
            mx = fmaxf(mx, other_half(mx)) * P.scale_log2e;
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
#pragma unroll
                for (int r = 0; r < 16; ++r) gt[r] *= alpha;
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[r], P.scale_log2e, -m));
                l += p;
                dp[r] = p * (dp[r] - delta);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const bf16x8 ds = half_of(dp, t);
#pragma unroll
                for (int c = 0; c < C::DT; ++c) acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ft(smem, at + W::K, t, c), ds, acc[c], 0, 0, 0);
                // (G takes dS as the sum of two bf16: one alone leaves dQ and both tables' gradients off by 2.6e-3 of their
                // norm in 14 x 14 windows, this by 2.4e-3, for 4 of 224 us)
                bf16x8 lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) lo[e] = (bf16)(dp[8 * t + e] - (float)ds[e]);
                const bf16x8 one = et(smem, W::E + 32 * j * W::EB, t, 0);
                gt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, ds, gt, 0, 0, 0);
                gt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(one, lo, gt, 0, 0, 0);
            }
        }
        mfma_settle();
        constexpr int RELS = (64 * CH + 64 * WIN_WAVES - 1) / (64 * WIN_WAVES);
        u32x4 rv[RELS];                                      // 32 rows a table, zeros behind its own
#pragma unroll
        for (int k = 0; k < RELS; ++k) {
            const int i = tid + 64 * WIN_WAVES * k, r = i / CH, c = i - r * CH;
            rv[k] = u32x4{ 0, 0, 0, 0 };
            if (r < 64 && (r & 31) < nrel) rv[k] = *reinterpret_cast<const u32x4 *>((r < 32 ? rel_h : rel_w) + (long)(r & 31) * D + c * 8);
        }
        // a wave's first keys on columns
        const int tile0 = light < tiles ? light : dense < heavy ? dense : 0;
        bf16x8 kf[C::KS], vf[C::KS];
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks) {
            kf[ks] = fa(smem, W::K + 32 * tile0 * W::RB, ks);
            vf[ks] = fa(smem, W::V + 32 * tile0 * W::RB, ks);
        }
        __syncthreads();                                     // K, V and E are read
        if (alive) {
            l += other_half(l);
            const float inv = 1.f / l;
            if (half == 0) {
                const bool none = pos >= S || (P.out_rows && P.out_rows[(long)grp * S + pos] < 0);
                reinterpret_cast<float *>(smem + W::L)[pos] = none ? -INFINITY : -(m + __builtin_amdgcn_logf(l)) * P.inv_scale_log2e;
                reinterpret_cast<float *>(smem + W::N)[pos] = -delta;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c) *reinterpret_cast<f16x8 *>(smem + W::E + pos * W::EB + ((2 * c) ^ esw) * 16) = bt[c];
#pragma unroll
            for (int t = 0; t < C::DT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[t][r] *= inv * P.scale;
            // G at relative positions, hi and lo: of a table entry y sits at t0 - y; register r <-> entry 8 (r >> 2 & 1) + 4 half + (r & 3) of table r >> 3
            unsigned char *mine = smem + W::G + pos * W::GB;
            const int gsw = swizzle<8>(l32);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                *reinterpret_cast<uint4 *>(mine + ((4 * half + c) ^ gsw) * 16) = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(mine + W::GPART + ((4 * half + c) ^ gsw) * 16) = make_uint4(0, 0, 0, 0);
            }
            wave_lds_fence();
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // (entries from w on are none: as zeros they go to positions below the first one's or, from the front of the row, to its end)
                const int y = 8 * (r >> 2 & 1) + 4 * half + (r & 3), at = 32 * (r >> 3) + (((r >> 3 ? col : row) + w - 1 - y) & 31);
                const float x = y < w ? gt[r] * (inv * P.over_one) : 0.f;
                const bf16 hi = (bf16)x;
                bf16 *to = reinterpret_cast<bf16 *>(mine + ((at >> 3) ^ gsw) * 16) + (at & 7);
                *to = hi;
                to[W::GPART / 2] = (bf16)(x - (float)hi);
            }
        }
#pragma unroll
        for (int k = 0; k < RELS; ++k) {
            const int i = tid + 64 * WIN_WAVES * k, r = i / CH, c = i - r * CH;
            if (i < 64 * CH) *reinterpret_cast<u32x4 *>(smem + W::REL + (r * C::VP + c * 8) * 2) = rv[k];
        }
        __syncthreads();
        if (alive) {
            const unsigned char *mine = smem + W::G + pos * W::GB;
            const int gsw = swizzle<8>(l32);
            const bf16 *rel = reinterpret_cast<const bf16 *>(smem + W::REL);
#pragma unroll
            for (int t = 0; t < 4; ++t) {                     // 16 relative positions of table t / 2
                bf16x8 g8[2];
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    const unsigned char *at = mine + part * W::GPART + 8 * half;
                    const bf16x4 a = *reinterpret_cast<const bf16x4 *>(at + ((2 * t) ^ gsw) * 16), b = *reinterpret_cast<const bf16x4 *>(at + ((2 * t + 1) ^ gsw) * 16);
                    g8[part] = bf16x8{ a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
                }
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt) {
                    const bf16x8 f = transposed(rel + 16 * t * C::VP, C::VP, 0, dt, D - 4, lane);
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, g8[0], acc[dt], 0, 0, 0);
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f, g8[1], acc[dt], 0, 0, 0);
                }
            }
            mfma_settle();
            const int stored = wave * 32 + (lane_now() & 31);
            store_direct<D>(acc, P.dq + ((long)grp * S + stored) * P.grad_stride + (long)head * D, stored < S);
        }

        // ---- tables
        if (tables && wave < 2 * C::DT) {
            const int tab = wave / C::DT, dt = wave % C::DT;
            const Transposed<8> gtr(lane);
            int f0 = W::Q + ft.place(0, dt), f1 = W::Q + ft.place(1, dt), g0 = W::G + gtr.place(0, tab), g1 = W::G + gtr.place(1, tab);
            const auto read = [&](int at0, int at1) __attribute__((always_inline)) {
                const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(smem + at0));
                const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((__attribute__((address_space(3))) bf16x4 *)(smem + at1));
                return bf16x8{ a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3] };
            };
#pragma unroll 1
            for (int i = 0; i < tiles; ++i) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const bf16x8 f = read(f0 + 16 * t * W::RB, f1 + 16 * t * W::RB);
                    table = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read(g0 + 16 * t * W::GB, g1 + 16 * t * W::GB), f, table, 0, 0, 0);
                    table = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read(g0 + 16 * t * W::GB + W::GPART, g1 + 16 * t * W::GB + W::GPART), f, table, 0, 0, 0);
                }
                f0 += 32 * W::RB;
                f1 += 32 * W::RB;
                g0 += 32 * W::GB;
                g1 += 32 * W::GB;
            }
        }

        // ---- columns
        f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
        for (int t = 0; t < C::DT; ++t) { dk[t] = zero16(); dv[t] = zero16(); }
#pragma unroll 1
        for (int next = light;; next += step) {              // the tiles behind the prefix, then the share
            const bool behind = next < tiles;
            if (!behind && dense >= heavy) break;             // the same for the whole wave
            const int tile = behind ? next : dense, i0 = behind ? tile >> mb << mb : share * per, i1 = min(i0 + (behind ? 1 << mb : per), tiles);
            const int kpos = tile * 32 + l32;
            if (tile != tile0) {                             // (keys past the end repeat the last one; their results are not stored)
                const long from = ((long)grp * S + min(kpos, S - 1)) * P.row_stride + (long)head * D + half * 8;
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    kf[ks] = *reinterpret_cast<const bf16x8 *>(P.k + from + ks * 16);
                    vf[ks] = *reinterpret_cast<const bf16x8 *>(P.v + from + ks * 16);
                }
            }
            const int krc = row_col(P.sigma + (long)grp * P.sigma_stride, kpos, P);
            const f16x8 er = ones((krc & 0xffff) - 8 * half, P.one), ec = ones((krc >> 16) - 8 * half, P.one);
#pragma unroll
            for (int t = 0; t < C::DT; ++t) { dk[t] = zero16(); dv[t] = zero16(); }
#pragma unroll 1
            for (int i = i0; i < i1; ++i) {
                const int at = 32 * i * W::RB;
                f32x16 p, ds;                                 // rows are queries: scores begin at -log sum exp, dP at -delta
                const float *ls = reinterpret_cast<const float *>(smem + W::L) + 32 * i + 4 * half;
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 v = *reinterpret_cast<const f32x4 *>(ls + 8 * g), u = *reinterpret_cast<const f32x4 *>(ls + WIN_ROWS + 8 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { p[4 * g + e] = v[e]; ds[4 * g + e] = u[e]; }
                }
                const unsigned char *tl = smem + W::E + (32 * i + l32) * W::EB;
                p = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(tl + esw * 16), er, p, 0, 0, 0);
                p = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(tl + (2 ^ esw) * 16), ec, p, 0, 0, 0);
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) p = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa(smem, at + W::Q, ks), kf[ks], p, 0, 0, 0);
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) ds = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa(smem, at + W::O, ks), vf[ks], ds, 0, 0, 0);
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
                        dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ft(smem, at + W::O, t, dt), pf, dv[dt], 0, 0, 0);
                        dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ft(smem, at + W::Q, t, dt), df, dk[dt], 0, 0, 0);
                    }
                }
            }
            mfma_settle();
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) dk[dt][r] *= P.scale;
            if (behind || shares == 1) {
                const int stored = tile * 32 + (lane_now() & 31);
                const long to = ((long)grp * S + stored) * P.grad_stride + (long)head * D;
                store_direct<D>(dk, P.dk + to, stored < S);
                store_direct<D>(dv, P.dv + to, stored < S);
            }
            if (!behind) break;
        }
        if (shares > 1 && heavy) {                           // the shares of a tile, added up in order
            __syncthreads();
            // [tile][share - 1][quad of registers][lane]
            float *at = reinterpret_cast<float *>(smem + (long)dense * (shares - 1) * W::PART) + 4 * lane;
            if (dense < heavy && share > 0) {
                float *to = at + (share - 1) * (W::PART / 4);
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        if (dt * 32 + 8 * g >= D) continue;
                        *reinterpret_cast<f32x4 *>(to + (dt * 4 + g) * 256) = f32x4{ dk[dt][4 * g], dk[dt][4 * g + 1], dk[dt][4 * g + 2], dk[dt][4 * g + 3] };
                        *reinterpret_cast<f32x4 *>(to + (D / 8 + dt * 4 + g) * 256) = f32x4{ dv[dt][4 * g], dv[dt][4 * g + 1], dv[dt][4 * g + 2], dv[dt][4 * g + 3] };
                    }
            }
            __syncthreads();
            if (dense < heavy && share == 0) {
#pragma unroll 1
                for (int s = 0; s < shares - 1; ++s, at += W::PART / 4)
#pragma unroll
                    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            if (dt * 32 + 8 * g >= D) continue;
                            const f32x4 a = *reinterpret_cast<const f32x4 *>(at + (dt * 4 + g) * 256), b = *reinterpret_cast<const f32x4 *>(at + (D / 8 + dt * 4 + g) * 256);
#pragma unroll
                            for (int e = 0; e < 4; ++e) { dk[dt][4 * g + e] += a[e]; dv[dt][4 * g + e] += b[e]; }
                        }
                const int stored = dense * 32 + (lane_now() & 31);
                const long to = ((long)grp * S + stored) * P.grad_stride + (long)head * D;
                store_direct<D>(dk, P.dk + to, stored < S);
                store_direct<D>(dv, P.dv + to, stored < S);
            }
        }
    }
    if (tables && wave < 2 * C::DT) {                        // [workgroup][table][relative position][feature]; result: lane <-> feature, register <-> position
        mfma_settle();
        const int lane = lane_now(), half = lane >> 5, c = wave % C::DT * 32 + (lane & 31);
        float *to = parts + ((long)blockIdx.x * 2 + wave / C::DT) * 32 * D + c;
        if (c < D)
#pragma unroll
            for (int r = 0; r < 16; ++r) to[(long)(8 * (r >> 2) + 4 * half + (r & 3)) * D] = table[r];
    }
}

}  // namespace
