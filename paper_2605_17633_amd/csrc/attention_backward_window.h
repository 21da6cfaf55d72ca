// Gradients of attention where a group's keys and queries fit into LDS together (S <= 224: windows): one workgroup does all of a (group, head).
//
// Q, K, V and dO are read once, and what the walks hand to each other (bias entries, statistics, G) never leaves the CU: the three launches that grids take read the features
// three times.  A workgroup stays on its CU and takes one (group, head) after the other, so that the tables' gradient, (G at relative positions)^T Q, is added up in registers.
//   rows     wave i has the queries of tile i (32): scores, P, dS over its keys; leaves dQ, G, -log sum exp
//   tables   a 32 x 32 tile of drel a wave, over all queries
//   columns  every active (query tile, key tile) once more with P from the statistics.  Keys of the dense prefix see all queries: their query tiles are dealt out to several waves,
//            whose sums are added through LDS in order; the others see one tile of the mask, and a wave has at most one of them, in front of its share of the prefix
// The space of K and V holds G (as the sum of two bf16) and the relative positions' features once the rows are done; that of E then holds the bias entries T.
#pragma once

namespace {

constexpr int WIN_ROWS = 224, WIN_TILES = WIN_ROWS / 32, WIN_WAVES = 8, WIN_GROUPS = 256;

template <int D>
struct WinCfg {
    using C = BwdCfg<D, 1>;
    static constexpr int RB = D * 2, EB = C::EW * 2, GB = 128;                      // rows, in bytes; of G: 2 x 32 relative positions
    static constexpr int Q = 0, O = Q + WIN_ROWS * RB, UEND = WIN_TILES * 32 * C::UP * 2, OEND = O + WIN_ROWS * RB;
    static constexpr int K = OEND > UEND ? OEND : UEND, V = K + WIN_ROWS * RB;      // (up to UEND lie products with the tables before Q and dO do)
    static constexpr int G = K, GPART = WIN_ROWS * GB, REL = G + 2 * GPART, REND = REL + 2 * 32 * C::VP * 2;
    static constexpr int VEND = V + WIN_ROWS * RB, E = VEND > REND ? VEND : REND;
    static constexpr int L = E + WIN_ROWS * EB, N = L + WIN_ROWS * 4, TOTAL = N + WIN_ROWS * 4;
    static constexpr int PART = 32 * 2 * D * 4;                                     // dK and dV of a key tile
    static_assert(TOTAL <= 160 * 1024 && (WIN_TILES - 1) * PART <= TOTAL, "");
};

// 32 result rows [column tiles]^T straight to memory, eight bytes a lane: two half-waves fill 16 bytes of a row, and the cache puts rows together
template <int D>
__device__ __forceinline__ void store_direct(const f32x16 *acc, bf16 *row, bool stored)
{
    const int half = lane_now() >> 5;
    if (!stored) return;
#pragma unroll
    for (int dt = 0; dt < (D + 31) / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (dt * 32 + 8 * g >= D) continue;
            *reinterpret_cast<bf16x4 *>(row + dt * 32 + 8 * g + 4 * half) = bf16x4{ (bf16)acc[dt][4 * g], (bf16)acc[dt][4 * g + 1], (bf16)acc[dt][4 * g + 2], (bf16)acc[dt][4 * g + 3] };
        }
}

template <int D>
__global__ void __launch_bounds__(64 * WIN_WAVES, 2)
backward_windows_kernel(BwdParams P, bool tables, float *__restrict__ parts)
{
    using C = BwdCfg<D, 1>;
    using W = WinCfg<D>;
    constexpr int CH = D / 8, EC = W::EB / 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    clamp_fp16();
    const int S = P.S, w = P.w, nrel = 2 * w - 1, tiles = (S + 31) / 32, mb = P.mask_block == 128 ? 2 : 0;                        // (log of a mask tile's 32s)
    const int heavy = min(P.n_pre << mb, tiles);
    const bool alive = wave < tiles;
    // this wave's work on columns: a tile behind the prefix, and a share of a tile of the prefix
    const int want = heavy ? min(max(WIN_WAVES / heavy, 1), tiles) : 1, per = (tiles + want - 1) / want, shares = (tiles + per - 1) / per;
    const int light = heavy + WIN_WAVES - 1 - wave, share = wave % shares, dense = wave / shares;       // (tiles; a light one >= tiles, a dense one >= heavy: none)

    f32x16 table = zero16();                                  // drel of table wave / DT, features 32 (wave % DT) ..

#pragma unroll 1
    for (long first = 0; first < P.n_gh; first += gridDim.x) {
        // neighbours of a group share cache lines: they run on one XCD (workgroup b sits on XCD b & 7)
        const int gh = (int)first + ((gridDim.x & 7) == 0 ? (int)((blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3)) : (int)blockIdx.x);
        if (gh >= P.n_gh) break;                             // the same for the whole workgroup
        const int grp = gh / P.h, head = gh - grp * P.h;
        const int lane = lane_now(), tid = wave * 64 + lane, l32 = lane & 31, half = lane >> 5, pos = wave * 32 + l32;
        const int esw = swizzle<EC>(l32) ^ half, fsw = swizzle<CH>(l32) ^ half;
        const bf16 *rel_h = P.rel_h, *rel_w = P.rel_w;
        asm volatile("" : "+s"(rel_h), "+s"(rel_w));           // (read again for every (group, head): kept, their rows would take 40 registers)
        const long slot = (long)grp * S + min(pos, S - 1);
        const int rc = row_col(P.sigma + (long)grp * P.sigma_stride, pos, P), row = rc & 0xffff, col = rc >> 16;
        bf16x8 qf[C::KS], of[C::KS];
        float delta = 0.f;
        f16x8 bt[2];
        const int orow = pos < S ? P.out_rows ? P.out_rows[slot] : 0 : -1;
        {
            bf16x8 kf[C::KS], vf[C::KS];
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
                for (int e = 0; e < 8; ++e) qf[ks][e] = of[ks][e] = kf[ks][e] = vf[ks][e] = (bf16)0.f;
            if (pos < S) {
                const long from = slot * P.row_stride + (long)head * D + half * 8;
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    kf[ks] = *reinterpret_cast<const bf16x8 *>(P.k + from + ks * 16);
                    vf[ks] = *reinterpret_cast<const bf16x8 *>(P.v + from + ks * 16);
                }
                if (orow >= 0) {                              // (else its output is dropped: no gradient comes from it)
                    const long at = (P.out_rows ? (long)orow : slot) * ((long)P.h * D) + (long)head * D + half * 8;
#pragma unroll
                    for (int ks = 0; ks < C::KS; ++ks) {
                        qf[ks] = *reinterpret_cast<const bf16x8 *>(P.q + from + ks * 16);
                        of[ks] = *reinterpret_cast<const bf16x8 *>(P.dout + at + ks * 16);
                        const bf16x8 o = *reinterpret_cast<const bf16x8 *>(P.out + at + ks * 16);
#pragma unroll
                        for (int e = 0; e < 8; ++e) delta = fmaf((float)of[ks][e], (float)o[e], delta);
                    }
                }
            }
            __syncthreads();                                 // nobody reads the (group, head) before any more
            if (alive) {
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) {
                    unsigned char *to = smem + pos * W::RB + ((2 * ks) ^ fsw) * 16;
                    *reinterpret_cast<bf16x8 *>(to + W::K) = kf[ks];
                    *reinterpret_cast<bf16x8 *>(to + W::V) = vf[ks];
                }
                // E: a half-wave has the row's 16 entries, the other one the column's
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    *reinterpret_cast<f16x8 *>(smem + W::E + pos * W::EB + ((2 * half + c) ^ swizzle<EC>(l32)) * 16) = ones((half ? col : row) - 8 * c);
            }
        }
        delta += other_half(delta);
        if (alive) {
            // bias entries over the scale: rel Q^T, whose 32 rows hold all relative positions (w <= 14), and the entries back from where they lie for this query
            constexpr int FIRST = 2 * C::WK;
            _Float16 *u_row = reinterpret_cast<_Float16 *>(smem) + (wave * 32 + l32) * C::UP;
#pragma unroll
            for (int tab = 0; tab < 2; ++tab) {
                wave_lds_fence();
                _Float16 *to = u_row + (FIRST + w - 1 + (tab ? col : row) - 4 * half);
                const bf16 *rp = (tab ? rel_w : rel_h) + (long)min(l32, nrel - 1) * D + half * 8;
                f32x16 u = zero16();
#pragma unroll
                for (int ks = 0; ks < C::KS; ++ks) u = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(rp + ks * 16), qf[ks], u, 0, 0, 0);
                mfma_settle();
#pragma unroll
                for (int r = 0; r < 16; ++r) to[-8 * (r >> 2) - (r & 3)] = (_Float16)(u[r] * P.inv_scale);
                wave_lds_fence();
                f16x8 v = *reinterpret_cast<const f16x8 *>(u_row + FIRST + 8 * half);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 8 * half + e < w ? v[e] : (_Float16)0.f;
                bt[tab] = v;
            }
        }
        __syncthreads();
        if (alive)
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) {
                unsigned char *to = smem + pos * W::RB + ((2 * ks) ^ fsw) * 16;
                *reinterpret_cast<bf16x8 *>(to + W::Q) = qf[ks];
                *reinterpret_cast<bf16x8 *>(to + W::O) = of[ks];
            }
        // (Q and dO are read behind the rows' barrier; K, V and E were written in front of the one above)

        const Transposed<CH> ft(lane);
        const Straight<CH> fa(lane);

        // ---- rows
        const Transposed<EC> et(lane);
        // (of 80 features dO comes back from LDS for every block, and V is not read along with K: registers for them are short)
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
            sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(el + esw * 16), bt[0], sc, 0, 0, 0);
            sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const f16x8 *>(el + (2 ^ esw) * 16), bt[1], sc, 0, 0, 0);
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa(smem, at + W::K, ks), qf[ks], sc, 0, 0, 0);
            if (D == 80) asm volatile("" : "+v"(bt[0]), "+v"(bt[1]));
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
                gt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(et(smem, W::E + 32 * j * W::EB, t, 0), ds, gt, 0, 0, 0);
            }
        }
        mfma_settle();
        __syncthreads();                                     // K, V and E are read
        if (alive) {
            l += other_half(l);
            const float inv = 1.f / l;
            if (half == 0) {
                reinterpret_cast<float *>(smem + W::L)[pos] = orow < 0 ? -INFINITY : -(m + __builtin_amdgcn_logf(l)) * P.inv_scale_log2e;
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
                *reinterpret_cast<uint4 *>(mine + (4 * half + c) * 16) = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4 *>(mine + W::GPART + (4 * half + c) * 16) = make_uint4(0, 0, 0, 0);
            }
            wave_lds_fence();
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int y = 8 * (r >> 2 & 1) + 4 * half + (r & 3), at = 32 * (r >> 3) + (r >> 3 ? col : row) + w - 1 - y;
                const float x = gt[r] * (inv * 128.f);
                const bf16 hi = (bf16)x;
                if (y < w) {
                    bf16 *to = reinterpret_cast<bf16 *>(mine + ((at >> 3) ^ gsw) * 16) + (at & 7);
                    *to = hi;
                    to[W::GPART / 2] = (bf16)(x - (float)hi);
                }
            }
        }
        for (int i = tid; i < 64 * CH; i += 64 * WIN_WAVES) {
            const int r = i / CH, c = i - r * CH;
            u32x4 v = { 0, 0, 0, 0 };
            if ((r & 31) < nrel) v = *reinterpret_cast<const u32x4 *>((r < 32 ? rel_h : rel_w) + (long)(r & 31) * D + c * 8);
            *reinterpret_cast<u32x4 *>(smem + W::REL + (r * C::VP + c * 8) * 2) = v;
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
#pragma unroll 1
            for (int i = 0; i < tiles; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    // (the place of a tile is part of a constant where the rows' pitch asks for it: one of three features' tiles, one of two tables)
                    bf16x8 f;
                    if (dt == 0) f = ft(smem, W::Q + 32 * i * W::RB, t, 0);
                    else if (dt == 1) f = ft(smem, W::Q + 32 * i * W::RB, t, 1 % C::DT);
                    else f = ft(smem, W::Q + 32 * i * W::RB, t, 2 % C::DT);
#pragma unroll
                    for (int part = 0; part < 2; ++part) {
                        const int at = W::G + part * W::GPART + 32 * i * W::GB;
                        const bf16x8 g = tab ? gtr(smem, at, t, 1) : gtr(smem, at, t, 0);
                        table = __builtin_amdgcn_mfma_f32_32x32x16_bf16(g, f, table, 0, 0, 0);
                    }
                }
        }

        // ---- columns
        f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
        for (int t = 0; t < C::DT; ++t) { dk[t] = zero16(); dv[t] = zero16(); }
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            const int tile = pass ? dense : light, i0 = pass ? share * per : tile >> mb << mb, i1 = min(i0 + (pass ? per : 1 << mb), tiles);
            if (tile >= (pass ? heavy : tiles)) continue;     // the same for the whole wave
            const int kpos = tile * 32 + l32;
            const long kslot = (long)grp * S + min(kpos, S - 1);      // keys past the end repeat the last one; their results are not stored
            bf16x8 kf[C::KS], vf[C::KS];
#pragma unroll
            for (int ks = 0; ks < C::KS; ++ks) {
                kf[ks] = *reinterpret_cast<const bf16x8 *>(P.k + kslot * P.row_stride + (long)head * D + half * 8 + ks * 16);
                vf[ks] = *reinterpret_cast<const bf16x8 *>(P.v + kslot * P.row_stride + (long)head * D + half * 8 + ks * 16);
            }
            const int krc = row_col(P.sigma + (long)grp * P.sigma_stride, kpos, P);
            const f16x8 er = ones((krc & 0xffff) - 8 * half), ec = ones((krc >> 16) - 8 * half);
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
            if (pass == 0 || shares == 1) {
                const int stored = tile * 32 + (lane_now() & 31);
                const long to = ((long)grp * S + stored) * P.grad_stride + (long)head * D;
                store_direct<D>(dk, P.dk + to, stored < S);
                store_direct<D>(dv, P.dv + to, stored < S);
            }
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
