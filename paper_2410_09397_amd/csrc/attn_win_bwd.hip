// Windowed attention, backward, bf16 (widths of 64, 128 and 256 columns, other rows padded: see attn_win_fwd.hip), in the tiling of the backward without a window (attn_bwd.hip), whose
// layouts, phases and wave priorities these kernels share:
//   win_dq_kernel    a workgroup owns 128 rows r = t * group + head of the group and streams the 64-key tiles that they see (SPLIT = 2: 64 rows,
//                    two waves for 32 of them with a key half of every tile each)
//   win_dkdv_kernel  a workgroup owns 64 keys and streams the 64-token tiles that see them, of one head of the group after the other: the sum
//                    over the heads that share the keys is a longer stream into the same accumulators
// No atomics, so the same call gives the same bits.  A key that is a sink is seen by every token behind it: the tokens that see a tile
// with sinks are shared out over p.parts workgroups, whose fp32 sums win_keys_kernel brings together; where there are fewer key tiles than
// places on the chip, those of the other tiles over p.rest_parts.  P and dS are rounded to bf16 for the
// products that use them (2^-9 of each weight; at the padded head dimensions by choice: see attn_win_fwd.hip), sums are fp32.
#include <type_traits>

#include "attn_internal.hpp"
#include "attn_win_tiles.hpp"

namespace attn {
namespace {

constexpr int kPrioScores = 3, kPrioSoftmax = 0, kPrioProducts = 1;

// ------------------------------------------------------------------------------------------------------------- dQ
template <int D, int SPLIT, bool PAD>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) win_dq_kernel(WinParams p, int row_blocks) {
    constexpr int KS = D / 16, MT = D / 32, kTile = 64 * D * 2, BR = 128 / SPLIT;
    extern __shared__ __attribute__((aligned(1024))) char smem[];  // [stage][K, V]
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wq = SPLIT == 1 ? w : w & 1, wk = SPLIT == 1 ? 0 : w >> 1;
    int bk, blk;
    decode_block(blockIdx.x, row_blocks, p.batch * p.kv_heads, bk, blk);
    const int b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = (row_blocks - 1 - blk) * BR;
    const int w0 = min(r0 + 32 * wq, rows - 1), w1 = min(r0 + 32 * wq + 31, rows - 1);  // rows of this wave (repeated past the end)
    auto place = [&](int r, int& t, int& head) {
        t = win_token(p, r);
        head = kvh * p.group + r - t * p.group;
    };
    int t, head;
    place(min(w0 + l32, rows - 1), t, head);
    const int t_lo = win_token(p, w0), t_hi = win_token(p, w1);
    LaneBounds see;
    see.init(p, t, s.len);
    WinTiles<64> tiles;
    tiles.init(p, s.len, win_token(p, r0), win_token(p, min(r0 + BR - 1, rows - 1)));

    // Q and dO rows of a wave come through 16 KB (d = 128) of the stages that only this wave reads, then O for delta = rowsum(dO o O), which stays in
    // the workspace for the key owners.  Queries outside their sequence have delta 0.
    char* mine = smem + w * (2 * 32 * D * 2);
    auto copy_rows = [&](const void* base, char* to) {
#pragma unroll
        for (int u = 0; u < 32 / CopyLane<D>::kRows; ++u) {
            const int row = CopyLane<D>::row_of(u, lane);
            int qt, qh;
            place(min(w0 + row, rows - 1), qt, qh);
            const __bf16* from = static_cast<const __bf16*>(base) + s.q_base + (long)qh * p.q_h + (long)qt * p.q_n;
            copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(from), row, lane, p.d), lds_address(to + u * 1024));
        }
    };
    copy_rows(p.Q, mine);
    copy_rows(p.dO, mine + 32 * D * 2);
    FragOffsets<D> offsets;
    offsets.init(lane);
    const long stat = s.lse_base + (long)head * s.lse_h + t;
    const float lse = see.hi >= 0 ? p.LSE_in[stat] * kLog2e : 0.f;
    bf16x8 qf[KS], gf[KS];
    wait_direct_loads();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = offsets.frag(mine, 0, 0, ks);
        gf[ks] = offsets.frag(mine + 32 * D * 2, 0, 0, ks);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    copy_rows(p.O_in, mine);
    wait_direct_loads();
    float dl = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 of = offsets.frag(mine, 0, 0, ks);
#pragma unroll
        for (int e = 0; e < 8; ++e) dl += (float)of[e] * (float)gf[ks][e];
    }
    dl += __shfl_xor(dl, 32, 64);
    if (see.hi < 0) dl = 0.f;
    if (h == 0 && wk == 0 && r0 + 32 * wq + l32 < rows) p.delta[stat] = dl;
    settle(lse);
    settle(dl);
    __syncthreads();  // the stages are free

    TileLoader<D, 64> loader;
    loader.init(tid, p.k_n);
    const long kv = (long)b * p.k_b + (long)kvh * p.k_h;
    const __bf16 *K = static_cast<const __bf16*>(p.K) + kv, *V = static_cast<const __bf16*>(p.V) + kv;
    auto request = [&](int j0, char* stage) {
        if (!PAD && tiles.whole(p, j0)) {
            loader.load(K + (long)j0 * p.k_n, stage);
            loader.load(V + (long)j0 * p.k_n, stage + kTile);
        } else {
#pragma unroll
            for (int u = 0; u < 64 / (4 * CopyLane<D>::kRows); ++u) {
                const int inst = u * 4 + w, row = CopyLane<D>::row_of(inst, lane);
                const long at = (long)tiles.row(p, j0 + row) * p.k_n;
                copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(K + at), row, lane, p.d), lds_address(stage + inst * 1024));
                copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(V + at), row, lane, p.d), lds_address(stage + kTile + inst * 1024));
            }
        }
    };
    const int n_it = tiles.count;
    if (n_it > 0) request(tiles.start(0), smem);
    f32x16 dq[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 16; ++i) dq[mt][i] = 0.f;
    FragAddrs<D> fo;
    fo.init(offsets);
    if constexpr (SPLIT > 1) fo.shift_rows(32 * wk);
    const float c = p.scale * kLog2e;
    // the dP chains start from -delta (not at d = 256, which has no 16 registers for it)
    constexpr bool kDeltaInAcc = D == 128;
    f32x16 ndl;
#pragma unroll
    for (int i = 0; i < 16; ++i) ndl[i] = kDeltaInAcc ? -dl : 0.f;
    wait_direct_loads();
    __syncthreads();

    auto tile = [&](auto stage_off, int j0, bool masked) {
        const int off = stage_off;
#pragma unroll
        for (int T = 0; T < 2 / SPLIT; ++T) {
            __builtin_amdgcn_s_setprio(kPrioScores);
            if (D < 256 && SPLIT == 1 && T == 1 && j0 + 32 >= p.sinks && j0 + 63 < t_lo - p.window + 1) break;  // (of a tile of sinks: nothing is seen of this half)
            f32x16 st, dp = ndl;
#pragma unroll
            for (int i = 0; i < 16; ++i) st[i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const bf16x8 kf = fo.frag(smem, off, 32 * T, ks), vf = fo.frag(smem, off + kTile, 32 * T, ks);
                st = mfma32(kf, qf[ks], st);
                dp = mfma32(vf, gf[ks], dp);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(kPrioSoftmax);
#pragma unroll
            for (int i = 0; i < 16; ++i) dp[i] = __builtin_amdgcn_exp2f(fmaf(st[i], c, -lse)) * (kDeltaInAcc ? dp[i] : dp[i] - dl);
            if (masked) {
                const int j = j0 + 32 * T + 4 * h, hi = see.hi - j, lo = see.lo - j, sink = p.sinks - j;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int x = 8 * (i >> 2) + (i & 3);
                    dp[i] = x <= hi && (x >= lo || x < sink) ? dp[i] : 0.f;
                }
            }
            bf16x8 ds[2], kt[2][MT];
#pragma unroll
            for (int x = 0; x < 2; ++x) ds[x] = acc_to_operand(dp, x);
            __builtin_amdgcn_s_setprio(kPrioProducts);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) kt[0][mt] = fo.frag_t(smem, off, mt, 32 * T);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                if (x == 0) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) kt[1][mt] = fo.frag_t(smem, off, mt, 32 * T + 16);
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) dq[mt] = mfma32(kt[x][mt], ds[x], dq[mt]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto step = [&](auto stage_off, int it) {
        const int off = stage_off, j0 = tiles.start(it) + 32 * wk;  // (of the keys that this wave looks at)
        if (it + 1 < n_it) request(tiles.start(it + 1), smem + (2 * kTile - off));
        constexpr int kLast = 64 / SPLIT - 1;
        const bool none = j0 > t_hi || (j0 + kLast < t_lo - p.window + 1 && j0 >= p.sinks) || r0 + 32 * wq >= rows;
        const bool all = j0 + kLast <= t_lo && t_hi < s.len && (t_hi - j0 < p.window || j0 + kLast < p.sinks);
        if (D == 256 || !none) tile(stage_off, j0, !all);  // (see win_out_kernel)
        wait_direct_loads();
        __syncthreads();
    };
    if constexpr (D == 256) {
        for (int it = 0; it < n_it; ++it) step(it & 1 ? 2 * kTile : 0, it);
    } else
    for (int it = 0; it < n_it; it += 2) {
        step(std::integral_constant<int, 0>{}, it);
        if (it + 1 < n_it) step(std::integral_constant<int, 2 * kTile>{}, it + 1);
    }

    constexpr int kMeet = SPLIT == 2 ? 2 * 4 * MT * 1024 : 0;
    if constexpr (SPLIT == 2) {  // the two waves of a row meet in LDS (see win_out_kernel)
        auto slot = [&](int g) { return reinterpret_cast<f32x4*>(smem) + (wq * 4 * MT + g) * 64 + lane; };
        if (wk == 1) {
#pragma unroll
            for (int g = 0; g < 4 * MT; ++g) {
                const f32x16& a = dq[g / 4];
                *slot(g) = f32x4{a[4 * (g % 4)], a[4 * (g % 4) + 1], a[4 * (g % 4) + 2], a[4 * (g % 4) + 3]};
            }
        }
        __syncthreads();
        if (wk == 1) return;
#pragma unroll
        for (int g = 0; g < 4 * MT; ++g) {
            const f32x4 a = *slot(g);
#pragma unroll
            for (int e = 0; e < 4; ++e) dq[g / 4][4 * (g % 4) + e] += a[e];
        }
    }
    typedef RowStage<D> Rows;
    static_assert(kMeet + 4 / SPLIT * Rows::kBytes <= 4 * kTile, "the rows fit the stages");
    char* out = smem + kMeet + wq * Rows::kBytes;
#pragma unroll
    for (int g = 0; g < 4 * MT; ++g) {
        const f32x16& a = dq[g / 4];
        Rows::put(out, g,
                  u32x2{pack_bf16(a[4 * (g % 4)] * p.scale, a[4 * (g % 4) + 1] * p.scale),
                        pack_bf16(a[4 * (g % 4) + 2] * p.scale, a[4 * (g % 4) + 3] * p.scale)},
                  lane);
    }
    wave_exchange();
#pragma unroll
    for (int x = 0; x < 32; x += 64 / Rows::kLanes) {
        const int row = x + lane / Rows::kLanes, cc = lane % Rows::kLanes, r = r0 + 32 * wq + row;
        if (r < rows && (!PAD || 8 * cc < p.d)) {
            int qt, qh;
            place(r, qt, qh);
            *reinterpret_cast<u32x4*>(static_cast<__bf16*>(p.dQ) + s.q_base + (long)qh * p.q_h + (long)qt * p.q_n + 8 * cc) =
                *reinterpret_cast<const u32x4*>(out + row * Rows::kPitch + 16 * cc);
        }
    }
}

// --------------------------------------------------------------------------------------------------------- dK, dV
// Phase 1, wave (wk, wx): S^T and dP^T for key half wk and token half wx; P and dS to LDS as [token][key] tiles.
// Phase 2: dV^T (wx = 0) or dK^T (wx = 1) for the half wk of d, all 64 keys and tokens.
template <int D, bool PAD>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) win_dkdv_kernel(WinParams p, int key_blocks) {
    constexpr int KS = D / 16, MT = D / 32, MH = MT / 2, kTile = 64 * D * 2, kStage = 2 * kTile, kP = 64 * 64 * 2;
    extern __shared__ __attribute__((aligned(1024))) char smem[];  // [stage][Q, dO], P, dS
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wk = w & 1, wx = w >> 1;
    int bk, blk;
    decode_block(blockIdx.x, key_blocks, p.batch * p.kv_heads, bk, blk);
    const int b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    WinKeys keys;
    keys.init(p, blk, 64, s.len);
    const int j0 = keys.j0, i0 = keys.i0, i1 = keys.i1;
    const int t_tiles = (i1 - i0 + 63) / 64, jobs = t_tiles * p.group;
    const long kv = (long)b * p.k_b + (long)kvh * p.k_h;

    f32x16 acc[MH][2];
#pragma unroll
    for (int m = 0; m < MH; ++m)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][kt][i] = 0.f;
    if (jobs > 0) {
        const float c = p.scale * kLog2e;
        TileLoader<D, 64> loader;
        loader.init(tid, p.q_n);
        // what the next job's rows need: its tile, the head's base, this lane's statistics
        int g_next = 0, t_next = 0, ti_next = i0;
        const __bf16 *Qh = static_cast<const __bf16*>(p.Q) + s.q_base + (long)kvh * p.group * p.q_h;
        const __bf16 *Gh = static_cast<const __bf16*>(p.dO) + s.q_base + (long)kvh * p.group * p.q_h;
        const float* lse_g = p.LSE_in + s.lse_base + (long)kvh * p.group * s.lse_h;
        const float* delta_g = p.delta + s.lse_base + (long)kvh * p.group * s.lse_h;
        float lse_raw = 0.f, delta_raw = 0.f;
        auto fetch_rows = [&] {
            const int i = min(ti_next + 32 * wx + l32, i1 - 1);
            lse_raw = lse_g[(long)g_next * s.lse_h + i];
            delta_raw = delta_g[(long)g_next * s.lse_h + i];
        };
        // 64 rows from `row0` on; rows from `end` on repeat the last one
        auto load_rows = [&](const TileLoader<D, 64>& by, const __bf16* base, long ld, int row0, int end, char* to) {
            if constexpr (PAD) {
                int l = lane;  // (formed again for every tile: d > 128 has no registers to keep what a lane copies)
                asm volatile("" : "+v"(l));
#pragma unroll
                for (int u = 0; u < 64 / (4 * CopyLane<D>::kRows); ++u) {
                    const int inst = u * 4 + w, row = CopyLane<D>::row_of(inst, l);
                    const __bf16* from = base + (long)min(row0 + row, end - 1) * ld;
                    copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(from), row, l, p.d), lds_address(to + inst * 1024));
                }
            } else {
                by.load(base, ld, row0, end, to, tid);
            }
        };
        auto fetch = [&](char* stage) {
            load_rows(loader, Qh + (long)g_next * p.q_h, p.q_n, ti_next, i1, stage);
            load_rows(loader, Gh + (long)g_next * p.q_h, p.q_n, ti_next, i1, stage + kTile);
            fetch_rows();
        };
        auto advance = [&] {
            ti_next += 64;
            if (++t_next == t_tiles) {
                t_next = 0;
                ti_next = i0;
                ++g_next;
            }
        };
        {
            // the owned rows come through the second stage; rows past the sequence repeat its last one, which nothing sees
            TileLoader<D, 64> own;
            own.init(tid, p.k_n);
            load_rows(own, static_cast<const __bf16*>(p.K) + kv, p.k_n, j0, s.len, smem + kStage);
            load_rows(own, static_cast<const __bf16*>(p.V) + kv, p.k_n, j0, s.len, smem + kStage + kTile);
        }
        fetch(smem);
        FragOffsets<D> fo;
        FragOffsets<64> fp;
        fo.init(lane);
        fp.init(lane);
        wait_direct_loads();
        __syncthreads();
        bf16x8 kf[KS], vf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = fo.frag(smem, kStage, 32 * wk, ks);
            vf[ks] = fo.frag(smem, kStage + kTile, 32 * wk, ks);
        }
        lds_barrier();  // (the second job's copies go into that stage)
        constexpr int kPOff = 2 * kStage, kDsOff = kPOff + kP;
        const int p_wr = tile_off<64>(32 * wx + l32, 4 * wk) + 8 * (h ^ (l32 & 1));
        fp.tr0 ^= (((lane & 15) >> 2) & 1) << 3;
        int q_rm[KS], a_tr[MH][2], b_tr[2][2], p_slot[4];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q_rm[ks] = fo.rm(ks) + 32 * wx * (D * 2);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
#pragma unroll
            for (int m = 0; m < MH; ++m) a_tr[m][half] = fo.tr(MH * wk + m, half) + (wx == 0 ? kTile : 0);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) b_tr[kt][half] = fp.tr(kt, half) + (wx == 0 ? kPOff : kDsOff);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) p_slot[g] = kPOff + (p_wr ^ (g << 4));

        int ti = i0;
        auto job = [&](auto stage_off, int it) {
            const int q_off = stage_off;
            const float lse = lse_raw * kLog2e, delta = delta_raw;
            const int i = ti + 32 * wx + l32;
            const bool all = ti >= j0 + 63 && ti + 64 <= i1 && (ti + 63 - j0 < p.window || j0 + 63 < p.sinks);
            // the next tile's copies go between the products of phase 1, one per k-step, where the tile is whole
            bool spread = false;
            const __bf16 *next_q = nullptr, *next_g = nullptr;
            char* next_stage = smem + (kStage - q_off);
            if (it + 1 < jobs) {
                advance();
                spread = !PAD && ti_next + 64 <= i1;
                if (spread) {
                    next_q = Qh + (long)g_next * p.q_h + (long)ti_next * p.q_n;
                    next_g = Gh + (long)g_next * p.q_h + (long)ti_next * p.q_n;
                    loader.hold(next_q);
                    loader.hold(next_g);
                    fetch_rows();
                } else {
                    fetch(next_stage);
                }
            }
            __builtin_amdgcn_s_setprio(kPrioScores);
            f32x16 st, dp;
#pragma unroll
            for (int x = 0; x < 16; ++x) st[x] = dp[x] = 0.f;
            {
                constexpr int kAhead = 2;  // fragments are requested two k-steps in front of their products
                bf16x8 fq[KS], fg[KS];
#pragma unroll
                for (int ks = 0; ks < kAhead; ++ks) {
                    fq[ks] = FragOffsets<D>::read(smem, q_rm[ks], q_off);
                    fg[ks] = FragOffsets<D>::read(smem, q_rm[ks], q_off + kTile);
                }
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (ks + kAhead < KS) {
                        fq[ks + kAhead] = FragOffsets<D>::read(smem, q_rm[ks + kAhead], q_off);
                        fg[ks + kAhead] = FragOffsets<D>::read(smem, q_rm[ks + kAhead], q_off + kTile);
                    }
                    st = mfma32(kf[ks], fq[ks], st);
                    dp = mfma32(vf[ks], fg[ks], dp);
                    if (spread) {
                        constexpr int kPer = TileLoader<D, 64>::kInst;
                        static_assert(2 * kPer == KS, "one copy per k-step");
                        if (ks < kPer) loader.load_one(ks, next_q, next_stage);
                        else loader.load_one(ks - kPer, next_g, next_stage + kTile);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(kPrioSoftmax);
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                st[x] = __builtin_amdgcn_exp2f(fmaf(st[x], c, -lse));
                dp[x] = st[x] * (dp[x] - delta);
            }
            if (!all) {
                const int j = j0 + 32 * wk + 4 * h, hi = (i < i1 ? i : -1) - j, lo = i - p.window + 1 - j, sink = p.sinks - j;
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const int k = 8 * (x >> 2) + (x & 3);
                    const bool seen = k <= hi && (k >= lo || k < sink);
                    st[x] = seen ? st[x] : 0.f;
                    dp[x] = seen ? dp[x] : 0.f;
                }
            }
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                *reinterpret_cast<u32x2*>(smem + p_slot[g]) = u32x2{pack_bf16(st[4 * g], st[4 * g + 1]), pack_bf16(st[4 * g + 2], st[4 * g + 3])};
                *reinterpret_cast<u32x2*>(smem + p_slot[g] + kP) = u32x2{pack_bf16(dp[4 * g], dp[4 * g + 1]), pack_bf16(dp[4 * g + 2], dp[4 * g + 3])};
            }
            lds_barrier();  // P and dS visible; the copies stay in flight
            __builtin_amdgcn_s_setprio(kPrioProducts);
            {
                bf16x8 at[2][MH], bt[2][2];
                auto request = [&](int ks) {
#pragma unroll
                    for (int m = 0; m < MH; ++m) at[ks & 1][m] = FragOffsets<D>::read_t(smem, a_tr[m][0], a_tr[m][1], 16 * ks, q_off);
#pragma unroll
                    for (int kt = 0; kt < 2; ++kt) bt[ks & 1][kt] = FragOffsets<64>::read_t(smem, b_tr[kt][0], b_tr[kt][1], 16 * ks);
                };
                request(0);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) {
                    if (ks + 1 < 4) request(ks + 1);
#pragma unroll
                    for (int m = 0; m < MH; ++m)
#pragma unroll
                        for (int kk = 0; kk < 2; ++kk) {
                            const int kt = (m & 1) ? 1 - kk : kk;  // consecutive products share an operand
                            acc[m][kt] = mfma32(at[ks & 1][m], bt[ks & 1][kt], acc[m][kt]);
                        }
                }
            }
            ti = ti_next;
            wait_direct_loads();
            __syncthreads();
        };
        for (int it = 0; it < jobs; it += 2) {
            job(std::integral_constant<int, 0>{}, it);
            if (it + 1 < jobs) job(std::integral_constant<int, kStage>{}, it + 1);
        }
    }

    if (keys.slot >= 0) {  // fp32 sums of this part: [dK, dV][64 keys][d]
        const int d = PAD ? p.d : D;
        float* dst = p.part_kv + (((long)bk * p.slots + keys.slot) * 2 + (wx == 0 ? 1 : 0)) * 64 * d;
        const float f = wx == 0 ? 1.f : p.scale;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int m = 0; m < MH; ++m)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x16& a = acc[m][kt];
                    if (32 * (MH * wk + m) + 8 * g < d)
                        *reinterpret_cast<f32x4*>(dst + (32 * kt + l32) * d + 32 * (MH * wk + m) + 8 * g + 4 * h) =
                        f32x4{a[4 * g] * f, a[4 * g + 1] * f, a[4 * g + 2] * f, a[4 * g + 3] * f};
                }
        return;
    }
    const float f = wx == 0 ? 1.f : p.scale;
    typedef RowStage<D> Rows;
    constexpr int kGrad = 2 * Rows::kBytes;  // 64 rows: dV, then dK
    static_assert(2 * kGrad <= 2 * kStage + 2 * kP, "the stages are free after the last tile");
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int m = 0; m < MH; ++m)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x16& a = acc[m][kt];
                Rows::put(smem + wx * kGrad + kt * Rows::kBytes, 4 * (MH * wk + m) + g,
                          u32x2{pack_bf16(a[4 * g] * f, a[4 * g + 1] * f), pack_bf16(a[4 * g + 2] * f, a[4 * g + 3] * f)}, lane);
            }
    __syncthreads();
    const long out = kv + (long)j0 * p.k_n;
    if (PAD && 8 * (lane % Rows::kLanes) >= p.d) return;  // (the columns of a lane are the same in every row that it stores)
    Rows::template store<64, 4>(smem, static_cast<__bf16*>(p.dV) + out, p.k_n, p.n - j0, lane, w);
    Rows::template store<64, 4>(smem + kGrad, static_cast<__bf16*>(p.dK) + out, p.k_n, p.n - j0, lane, w);
}

template <int D, int SPLIT, bool PAD>
hipError_t launch(const WinParams& p, hipStream_t stream) {
    constexpr int q_lds = 4 * 64 * D * 2, k_lds = q_lds + 2 * 64 * 64 * 2, BR = 128 / SPLIT;
    hipError_t e = allow_lds(win_dq_kernel<D, SPLIT, PAD>, q_lds);
    if (e == hipSuccess) e = allow_lds(win_dkdv_kernel<D, PAD>, k_lds);
    if (e != hipSuccess) return e;
    const int rows = (int)(((long)p.n * p.group + BR - 1) / BR), keys = p.sink_tiles * p.parts + ((p.n + 63) / 64 - p.sink_tiles) * p.rest_parts;
    const long bk = (long)p.batch * p.kv_heads;
    hipLaunchKernelGGL((win_dq_kernel<D, SPLIT, PAD>), dim3((unsigned)(rows * bk)), dim3(kThreads), q_lds, stream, p, rows);
    hipLaunchKernelGGL((win_dkdv_kernel<D, PAD>), dim3((unsigned)(keys * bk)), dim3(kThreads), k_lds, stream, p, keys);
    return hipGetLastError();
}
template <int D>
hipError_t launch(int rows, const WinParams& p, hipStream_t stream) {
    if (p.d < D) return rows == 64 ? launch<D, 2, true>(p, stream) : launch<D, 1, true>(p, stream);
    return rows == 64 ? launch<D, 2, false>(p, stream) : launch<D, 1, false>(p, stream);
}

}  // namespace

hipError_t launch_win_bwd(int rows, const WinParams& p, hipStream_t stream) {
    return p.d <= 64 ? launch<64>(rows, p, stream) : p.d <= 128 ? launch<128>(rows, p, stream) : launch<256>(rows, p, stream);
}

}  // namespace attn
