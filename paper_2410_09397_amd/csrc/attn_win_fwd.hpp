// The forward kernels of windowed attention on bf16-MFMA as functions (attn_win_fwd.hip says what each is for), over tensors or pages, and (TREE) over
// pages whose last tokens are a tree of drafted ones: attn_tree_fwd.hip.  HIP device code only.
#pragma once
#include <type_traits>

#include "attn_internal.hpp"
#include "attn_win_tiles.hpp"

namespace attn {
namespace {

__device__ __forceinline__ void win_place(const WinParams& p, int kvh, int r, int& t, int& head) {
    t = win_token(p, r);
    head = kvh * p.group + r - t * p.group;
}

// Softmax state of 32 rows on a wave, and one tile's turn.  st: NT accumulators of 32 keys each, in: scores; out: weights.
template <int D>
struct WinRows {
    static constexpr int MT = D / 32;
    f32x16 o[MT];
    float m, l;  // reference of the exponentials (scaled, base 2); this lane's half of the sum
    __device__ __forceinline__ void init() {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
        m = -__builtin_inff();
        l = 0.f;
    }
    // `masked`: applies what sees() says of this lane's query and register i of accumulator T of its half.  (A branch
    // around the bounds alone: with one around the whole tile the accumulators of both sides meet behind it, and the compiler keeps two sets:
    // 228 bytes of scratch at d = 128.)
    template <int NT, typename Sees>
    __device__ __forceinline__ void weights(f32x16 (&st)[NT], float cs, bool masked, Sees sees) {
        if (masked) {
            const auto seen = sees();
#pragma unroll
            for (int T = 0; T < NT; ++T)
#pragma unroll
                for (int i = 0; i < 16; ++i) st[T][i] = seen(T, 8 * (i >> 2) + (i & 3)) ? st[T][i] : -__builtin_inff();
        }
        float mx = max3(st[0][0], st[0][1], st[0][2]), my = max3(st[NT - 1][13], st[NT - 1][14], st[NT - 1][15]);
        if constexpr (NT == 2) {
#pragma unroll
            for (int i = 3; i < 15; i += 2) mx = max3(mx, st[0][i], st[0][i + 1]);
#pragma unroll
            for (int i = 1; i < 13; i += 2) my = max3(my, st[1][i], st[1][i + 1]);
            mx = max3(mx, my, __builtin_elementwise_maximum(st[0][15], st[1][0]));
        } else {
#pragma unroll
            for (int i = 3; i < 13; i += 2) mx = max3(mx, st[0][i], st[0][i + 1]);
            mx = __builtin_elementwise_maximum(mx, my);
        }
        // the reference moves only when a maximum has grown by more than 2^8 (O / l and m + log2 l do not depend on it)
        constexpr float kSlack = 8.f;
        if (__builtin_amdgcn_ballot_w64(mx * cs > m + kSlack) != 0) {
            mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 32, 64));
            const float cand = mx * cs, m_new = cand > m + kSlack ? cand : m;
            const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -__builtin_inff() ? 0.f : m_new));
            l *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[mt][i] *= alpha;
            m = m_new;
        }
        const float m_use = m == -__builtin_inff() ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int T = 0; T < NT; ++T)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float f = __builtin_amdgcn_exp2f(fmaf(st[T][i], cs, -m_use));
                st[T][i] = f;
                sum += f;
            }
        l += sum;
    }
};

// |scale| log2 e for scores that stay raw until the exponential; a negative scale goes into Q, a zero one becomes the smallest normal
// number, so that masked scores stay -inf.
__device__ __forceinline__ float win_scale(float scale) { return fmaxf(fabsf(scale) * kLog2e, 1.17549435e-38f); }
template <int KS>
__device__ __forceinline__ void win_sign(float scale, bf16x8 (&qf)[KS]) {
    if (scale < 0.f) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 v = __builtin_bit_cast(u32x4, qf[ks]);
            v ^= 0x80008000u;
            qf[ks] = __builtin_bit_cast(bf16x8, v);
        }
    }
}

// ------------------------------------------------------------------------------------------------------- many rows
// Tiles of 64 keys for a workgroup of four waves, K and V at once.
template <int D, int SRC, bool PAD>
struct TileFeed {
    static constexpr int kBytes = 64 * D * 2, kInst = 64 / (4 * CopyLane<D>::kRows);
    static constexpr int kChunks = D / 64;  // 16-code chunks per thread and tensor
    TileLoader<D, 64> loader;               // tensors
    PageWindow pages;
    CodeChunk kc[SRC == kCodes ? kChunks : 1], vc[SRC == kCodes ? kChunks : 1];
    // Tiles of pages that start on a multiple of their size and are all there: the rows that one instruction of a wave fetches lie in one page, whose address is
    // then scalar arithmetic, and what a lane adds to it is the same for every tile.
    static constexpr int kWaveRows = SRC == kCodes ? 1024 / D : CopyLane<D>::kRows, kOffs = SRC == kPages && D == 256 ? 2 : 1;
    static constexpr bool kEven = !PAD && !(SRC == kCodes && D == 64);  // (codes at d = 64: the registers of the second form cost a workgroup of four per CU)
    unsigned off[kOffs];
    bool even;
    __device__ __forceinline__ void init(const WinParams& p, int tid) {
        if constexpr (SRC == kTensors) {
            loader.init(tid, p.k_n);
        } else {
            pages.init();
            const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
            even = kEven && (1 << p.page_shift) >= kWaveRows && p.k_n < (1l << 26);
            if constexpr (SRC == kPages) {
#pragma unroll
                for (int x = 0; x < kOffs; ++x)  // (the swizzle of a row repeats after 16)
                    off[x] = (unsigned)(lane / (D / 8)) * (unsigned)p.k_n * 2u + 16u * ((lane % (D / 8)) ^ swz<D>(CopyLane<D>::row_of(x * 4 + w, lane)));
            } else {
                off[0] = (unsigned)(lane / (D / 16)) * (unsigned)p.k_n + 16u * (lane % (D / 16));
            }
        }
    }
    // key j, the same for all lanes, among the pages that cover() has read: element offset of its row and place of its exponent
    __device__ __forceinline__ PageRow scalar_row(const WinParams& p, int kvh, int j) const {
        return win_page_row(p, __builtin_amdgcn_readlane(pages.ids, (j >> p.page_shift) - pages.first), kvh, j);
    }
    // requests a tile; bf16: straight into the LDS stage (K at `stage`, V at stage + 2 kBytes); codes: into registers
    template <typename Tiles>
    __device__ __forceinline__ void request(const WinParams& p, const Tiles& tiles, int b, int kvh, int j0, char* stage, int tid) {
        const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
        if constexpr (SRC == kTensors) {
            const long base = (long)b * p.k_b + (long)kvh * p.k_h;
            const __bf16 *K = static_cast<const __bf16*>(p.K) + base, *V = static_cast<const __bf16*>(p.V) + base;
            if (!PAD && tiles.whole(p, j0)) {
                loader.load(K + (long)j0 * p.k_n, stage);
                loader.load(V + (long)j0 * p.k_n, stage + 2 * kBytes);
            } else {
#pragma unroll
                for (int u = 0; u < kInst; ++u) {
                    const int inst = u * 4 + w, row = CopyLane<D>::row_of(inst, lane);
                    const long at = (long)tiles.row(p, j0 + row) * p.k_n;
                    copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(K + at), row, lane, p.d), lds_address(stage + inst * 1024));
                    copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(V + at), row, lane, p.d),
                             lds_address(stage + 2 * kBytes + inst * 1024));
                }
            }
        } else {
            pages.cover(p, b, tiles.row(p, j0), tiles.row(p, j0 + 63), tiles.end, lane);
            if (kEven && even && (j0 & 63) == 0 && tiles.whole(p, j0)) {
                if constexpr (SRC == kPages) {
                    const unsigned t0 = lds_address(stage) + w * 1024u;
#pragma unroll
                    for (int u = 0; u < kInst; ++u) {
                        const long at = scalar_row(p, kvh, j0 + (u * 4 + w) * kWaveRows).at * 2;
                        copy_to_lds<16, true>(t0, u * 4096, off[u % kOffs], static_cast<const char*>(p.K) + at);
                        copy_to_lds<16, true>(t0, u * 4096 + 2 * kBytes, off[u % kOffs], static_cast<const char*>(p.V) + at);
                    }
                } else {
#pragma unroll
                    for (int x = 0; x < kChunks; ++x) {
                        const PageRow r = scalar_row(p, kvh, j0 + (x * 4 + w) * kWaveRows);
                        kc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.K) + r.at + off[0]);
                        vc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.V) + r.at + off[0]);
                        kc[x].scale = exp_value(p.K_exp[r.exp + lane / (D / 16)]);
                        vc[x].scale = exp_value(p.V_exp[r.exp + lane / (D / 16)]);
                    }
                }
            } else if constexpr (SRC == kPages) {
#pragma unroll
                for (int u = 0; u < kInst; ++u) {
                    const int inst = u * 4 + w, row = CopyLane<D>::row_of(inst, lane), j = tiles.row(p, j0 + row);
                    const long at = win_page_row(p, pages.page(p, j), kvh, j).at * 2;
                    copy_row(CopyLane<D>::template at<PAD>(static_cast<const char*>(p.K) + at, row, lane, p.d), lds_address(stage + inst * 1024));
                    copy_row(CopyLane<D>::template at<PAD>(static_cast<const char*>(p.V) + at, row, lane, p.d),
                             lds_address(stage + 2 * kBytes + inst * 1024));
                }
            } else {
#pragma unroll
                for (int x = 0; x < kChunks; ++x) {
                    const int idx = x * kThreads + tid, j = tiles.row(p, j0 + idx / (D / 16));
                    const PageRow r = win_page_row(p, pages.page(p, j), kvh, j);
                    const long at = r.at + 16 * (idx % (D / 16));
                    kc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.K) + at);
                    vc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.V) + at);
                    kc[x].scale = exp_value(p.K_exp[r.exp]);
                    vc[x].scale = exp_value(p.V_exp[r.exp]);
                }
            }
        }
    }
    // the requested tile is in its stage once this and a barrier are past
    __device__ __forceinline__ void arrive(char* stage, int tid) const {
        if constexpr (SRC == kCodes) {
#pragma unroll
            for (int x = 0; x < kChunks; ++x) {
                const int idx = x * kThreads + tid, row = idx / (D / 16), c = 2 * (idx % (D / 16));
                kc[x].to_lds(stage + tile_off<D>(row, c), stage + tile_off<D>(row, c + 1));
                vc[x].to_lds(stage + 2 * kBytes + tile_off<D>(row, c), stage + 2 * kBytes + tile_off<D>(row, c + 1));
            }
        } else {
            wait_direct_loads();
        }
    }
};

template <int D, int SRC, int SPLIT, bool PAD, bool TREE>
__device__ __forceinline__ void win_out(const WinParams& p, int row_blocks) {
    constexpr int KS = D / 16, MT = D / 32, kTile = 64 * D * 2, BR = 128 / SPLIT;
    extern __shared__ __attribute__((aligned(1024))) char smem[];  // [K stage 0][K stage 1][V stage 0][V stage 1]
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wq = SPLIT == 1 ? w : w & 1, wk = SPLIT == 1 ? 0 : w >> 1;
    int b, kvh, blk;
    Share<BR, 64, TREE> at;
    if constexpr (SRC == kTensors) {
        int bk;
        decode_block(blockIdx.x, row_blocks, p.batch * p.kv_heads, bk, blk);
        b = bk / p.kv_heads;
        kvh = bk % p.kv_heads;
        blk = row_blocks - 1 - blk;  // the last rows see most keys
    } else {  // (a key head's blocks on as few XCDs as its number allows)
        at.init(p, TREE ? (int)(blockIdx.x / p.kv_heads) : p.blocks - 1 - (int)(blockIdx.x / p.kv_heads), lane);
        if (!at.any) return;
        b = at.b;
        kvh = blockIdx.x % p.kv_heads;
        blk = at.blk;
    }
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = blk * BR;
    if (r0 >= rows) return;
    const int w0 = min(r0 + 32 * wq, rows - 1), w1 = min(r0 + 32 * wq + 31, rows - 1);  // rows of this wave (repeated past the end)
    int t, head;
    win_place(p, kvh, min(w0 + l32, rows - 1), t, head);
    Sight<64, TREE> see;
    see.init(p, s, t, win_token(p, w0), win_token(p, w1), win_token(p, r0), win_token(p, min(r0 + BR - 1, rows - 1)));
    const auto& tiles = see.tiles;
    const int it0 = at.first(p, tiles.count), it1 = at.last(p, tiles.count);

    TileFeed<D, SRC, PAD> feed;
    feed.init(p, tid);
    // the Q rows come through a piece of the second stage that only this wave reads
    char* mine = smem + (w < 2 ? 1 : 3) * kTile + (w & 1) * (32 * D * 2);
#pragma unroll
    for (int u = 0; u < 32 / CopyLane<D>::kRows; ++u) {
        const int row = CopyLane<D>::row_of(u, lane);
        int qt, qh;
        win_place(p, kvh, min(w0 + row, rows - 1), qt, qh);
        const __bf16* from = static_cast<const __bf16*>(p.Q) + s.q_base + (long)qh * p.q_h + (long)qt * p.q_n;
        copy_row(CopyLane<D>::template at<PAD>(reinterpret_cast<const char*>(from), row, lane, p.d), lds_address(mine + u * 1024));
    }
    if (it0 < it1) feed.request(p, tiles, b, kvh, tiles.start(it0), smem, tid);
    FragOffsets<D> offsets;
    offsets.init(lane);
    bf16x8 qf[KS];
    wait_direct_loads();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = offsets.frag(mine, 0, 0, ks);
    win_sign(p.scale, qf);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) settle(qf[ks]);
    const float cs = win_scale(p.scale);
    WinRows<D> acc;
    acc.init();
    FragAddrs<D> fo;
    fo.init(offsets);
    if constexpr (SPLIT > 1) fo.shift_rows(32 * wk);
    fo.shift_transposed(2 * kTile);
    if (it0 < it1) feed.arrive(smem, tid);
    __syncthreads();

    constexpr int kPrioScores = 2, kPrioSoftmax = 0, kPrioPV = 1;  // see the forward without a window
    // d = 256: the 32-key halves of a tile one after the other (both at once need 530 registers)
    constexpr int kTurns = D == 256 && SPLIT == 1 ? 2 : 1, NT = SPLIT == 2 ? 1 : 2 / kTurns;
    auto tile = [&](auto stage_off, int it, int j0, bool masked) {
        const int off = stage_off;
#pragma unroll
        for (int turn = 0; turn < kTurns; ++turn) {
            __builtin_amdgcn_s_setprio(kPrioScores);
            f32x16 st[NT];
#pragma unroll
            for (int T = 0; T < NT; ++T)
#pragma unroll
                for (int i = 0; i < 16; ++i) st[T][i] = 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int T = 0; T < NT; ++T) st[T] = mfma32(fo.frag(smem, off, 32 * (turn + T), ks), qf[ks], st[T]);
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(kPrioSoftmax);
            acc.weights(st, cs, masked, [&] { return see.template keys<NT>(p, it, j0 + 32 * turn, 4 * h); });
            bf16x8 pb[NT][2];
#pragma unroll
            for (int T = 0; T < NT; ++T)
#pragma unroll
                for (int x = 0; x < 2; ++x) pb[T][x] = acc_to_operand(st[T], x);
            __builtin_amdgcn_s_setprio(kPrioPV);
            // the V^T fragments of the next 16 keys are requested in front of the products of these
            bf16x8 va[2][MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) va[0][mt] = fo.frag_t(smem, off, mt, 32 * turn);
#pragma unroll
            for (int g = 0; g < 2 * NT; ++g) {
                if (g + 1 < 2 * NT) {
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) va[(g + 1) & 1][mt] = fo.frag_t(smem, off, mt, 32 * turn + 16 * (g + 1));
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) acc.o[mt] = mfma32(va[g & 1][mt], pb[g >> 1][g & 1], acc.o[mt]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto step = [&](auto stage_off, int it) {
        const int off = stage_off;
        const int j0 = tiles.start(it) + 32 * wk;  // of the keys that this wave looks at
        if (it + 1 < it1) feed.request(p, tiles, b, kvh, tiles.start(it + 1), smem + (kTile - off), tid);
        // what this wave's rows see of the tile: nothing, all of it, or a part
        constexpr int kLast = 64 / SPLIT - 1;
        const bool none = see.none(p, it, j0, kLast) || r0 + 32 * wq >= rows;
        if (D == 256 || !none) tile(stage_off, it, j0, !see.all(p, it, j0, kLast));  // (d = 256: the branch costs 150 to 420 bytes of scratch)
        if (it + 1 < it1) feed.arrive(smem + (kTile - off), tid);
        __syncthreads();
    };
    if constexpr (D == 256) {  // one copy of the body, with a run-time stage (two: 96 to 360 bytes of scratch)
        for (int it = it0; it < it1; ++it) step((it - it0) & 1 ? kTile : 0, it);
    } else
    for (int it = it0; it < it1; it += 2) {
        step(std::integral_constant<int, 0>{}, it);
        if (it + 1 < it1) step(std::integral_constant<int, kTile>{}, it + 1);
    }

    float l = acc.l + __shfl_xor(acc.l, 32, 64);
    if constexpr (SPLIT == 2) {
        // the two waves of a row meet in LDS (the stages are free: every wave is past the last barrier): [wave][4 MT groups][64 lanes] x 16 bytes, m, l
        auto slot = [&](int g) { return reinterpret_cast<f32x4*>(smem) + (wq * 4 * MT + g) * 64 + lane; };
        float* ml = reinterpret_cast<float*>(smem + 2 * 4 * MT * 1024) + wq * 128;
        if (wk == 1) {
#pragma unroll
            for (int g = 0; g < 4 * MT; ++g) {
                const f32x16& a = acc.o[g / 4];
                *slot(g) = f32x4{a[4 * (g % 4)], a[4 * (g % 4) + 1], a[4 * (g % 4) + 2], a[4 * (g % 4) + 3]};
            }
            ml[lane] = acc.m;
            ml[64 + lane] = l;
        }
        __syncthreads();
        if (wk == 1) return;
        const float m_other = ml[lane], m = __builtin_elementwise_maximum(acc.m, m_other), m_use = m == -__builtin_inff() ? 0.f : m;
        const float mine = __builtin_amdgcn_exp2f(acc.m - m_use), other = __builtin_amdgcn_exp2f(m_other - m_use);
        l = l * mine + ml[64 + lane] * other;
        acc.m = m;
#pragma unroll
        for (int g = 0; g < 4 * MT; ++g) {
            const f32x4 a = *slot(g);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc.o[g / 4][4 * (g % 4) + e] = acc.o[g / 4][4 * (g % 4) + e] * mine + a[e] * other;
        }
    }
    const bool ok = r0 + 32 * wq + l32 < rows, some = l != 0.f;  // (NaN: some)
    if (!at.whole(p, tiles.count)) {  // (its sums meet those of the other parts in a launch of their own)
        const long row = at.sums(p, s.lse_base + (long)t * p.heads + head, 32 * wq + l32);
        if (!ok) return;
        float* ml = p.part_ml + row * 2;
        if (h == 0) {
            ml[0] = acc.m;
            ml[1] = l;
        }
        if (some) {
            const int d = PAD ? p.d : D;
            float* dst = p.part_o + row * d + 4 * h;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    if (32 * mt + 8 * g < d)
                        *reinterpret_cast<f32x4*>(dst + 32 * mt + 8 * g) = f32x4{acc.o[mt][4 * g], acc.o[mt][4 * g + 1], acc.o[mt][4 * g + 2], acc.o[mt][4 * g + 3]};
        }
        return;
    }
    const float inv = some ? 1.f / l : 0.f;
    if (ok && h == 0)
        p.LSE[s.lse_base + (long)head * s.lse_h + (long)t * s.lse_t] = some ? (acc.m + __builtin_amdgcn_logf(l)) * kLn2 : -__builtin_inff();
    typedef RowStage<D> Rows;  // (behind what the waves of a row exchange)
    constexpr int kMeet = SPLIT == 2 ? 2 * 4 * MT * 1024 + 1024 : 0;
    static_assert(kMeet + 4 / SPLIT * Rows::kBytes <= 4 * kTile, "the rows fit the stages");
    char* out = smem + kMeet + wq * Rows::kBytes;
#pragma unroll
    for (int g = 0; g < 4 * MT; ++g) {
        const f32x16& a = acc.o[g / 4];
        Rows::put(out, g, u32x2{pack_bf16(a[4 * (g % 4)] * inv, a[4 * (g % 4) + 1] * inv), pack_bf16(a[4 * (g % 4) + 2] * inv, a[4 * (g % 4) + 3] * inv)}, lane);
    }
    wave_exchange();
#pragma unroll
    for (int x = 0; x < 32; x += 64 / Rows::kLanes) {
        const int row = x + lane / Rows::kLanes, c = lane % Rows::kLanes, r = r0 + 32 * wq + row;
        if (r < rows && (!PAD || 8 * c < p.d)) {
            int qt, qh;
            win_place(p, kvh, r, qt, qh);
            *reinterpret_cast<u32x4*>(static_cast<__bf16*>(p.O) + s.q_base + (long)qh * p.q_h + (long)qt * p.q_n + 8 * c) =
                *reinterpret_cast<const u32x4*>(out + row * Rows::kPitch + 16 * c);
        }
    }
}

// Rows r0 .. r1 of a workgroup from its waves' sums in LDS ([wave][ROWS][D + 4] fp32 and [wave][ROWS][m, l]): to O and LSE, or to the parts.
template <int D, int NW, int ROWS, bool PAD, typename S>
__device__ __forceinline__ void few_store(const WinParams& p, const WinSeq& s, const char* smem, const float* ml, int kvh, int r0, int r1, const S& share, int tiles) {
    constexpr int kPitch = D * 4 + 16;
    const int tid = threadIdx.x, d = PAD ? p.d : D;
    constexpr int kLanes = D / 4;  // threads per row
    for (int row = tid / kLanes; row < ROWS; row += 64 * NW / kLanes) {
        const int r = r0 + row, c = 4 * (tid % kLanes);
        if (r > r1 || c >= d) break;
        float m = -__builtin_inff();
#pragma unroll
        for (int x = 0; x < NW; ++x) m = __builtin_elementwise_maximum(m, ml[(x * ROWS + row) * 2]);
        const float m_use = m == -__builtin_inff() ? 0.f : m;
        float sum_l = 0.f;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < NW; ++x) {
            const float f = __builtin_amdgcn_exp2f(ml[(x * ROWS + row) * 2] - m_use);
            sum_l += f * ml[(x * ROWS + row) * 2 + 1];
            sum += *reinterpret_cast<const f32x4*>(smem + (x * ROWS + row) * kPitch + c * 4) * f;
        }
        int rt, rh;
        win_place(p, kvh, r, rt, rh);
        const long at = s.lse_base + (long)rt * p.heads + rh;
        const bool some = sum_l != 0.f;
        if (!share.whole(p, tiles)) {
            const long part = share.sums(p, at, row);
            if (c == 0) {
                p.part_ml[part * 2] = m;
                p.part_ml[part * 2 + 1] = sum_l;
            }
            if (some) *reinterpret_cast<f32x4*>(p.part_o + part * d + c) = sum;
        } else {
            const float inv = some ? 1.f / sum_l : 0.f;
            if (c == 0) p.LSE[at] = some ? (m + __builtin_amdgcn_logf(sum_l)) * kLn2 : -__builtin_inff();
            *reinterpret_cast<u32x2*>(static_cast<__bf16*>(p.O) + s.q_base + (long)rh * p.q_h + (long)rt * p.q_n + c) =
                u32x2{pack_bf16(sum[0] * inv, sum[1] * inv), pack_bf16(sum[2] * inv, sum[3] * inv)};
        }
    }
}

// -------------------------------------------------------------------------------------------------------- few rows
template <int D, int SRC>
constexpr int kFewWaves = D == 256 && SRC == kPages ? 2 : 4;
template <int D, int SRC>
constexpr int kFewStages = SRC == kPages ? 2 : 1;
template <int D, int SRC>
constexpr int kFewLds = [] {
    constexpr int stages = kFewWaves<D, SRC> * kFewStages<D, SRC> * 2 * 32 * D * 2;
    constexpr int meet = kFewWaves<D, SRC> * (32 * (D * 4 + 16) + 32 * 2 * 4);
    return stages > meet ? stages : meet;
}();

template <int D, int SRC, bool PAD, bool TREE>
__device__ __forceinline__ void win_few(const WinParams& p) {
    constexpr int NW = kFewWaves<D, SRC>, KS = D / 16, MT = D / 32, kTile = 32 * D * 2;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, l32 = lane & 31;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    Share<32, 32, TREE> at;
    at.init(p, (int)(blockIdx.x / p.kv_heads), lane);
    if (!at.any) return;
    const int b = at.b, kvh = blockIdx.x % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = at.blk * 32;
    if (r0 >= rows) return;
    const int r1 = min(r0 + 31, rows - 1);
    int t, head;
    win_place(p, kvh, min(r0 + l32, r1), t, head);
    const int t_lo = win_token(p, r0), t_hi = win_token(p, r1);
    Sight<32, TREE> see;
    see.init(p, s, t, t_lo, t_hi, t_lo, t_hi);
    const auto& tiles = see.tiles;
    const int it0 = at.first(p, tiles.count), it1 = at.last(p, tiles.count);

    bf16x8 qf[KS];
    const char* q = reinterpret_cast<const char*>(static_cast<const __bf16*>(p.Q) + s.q_base + (long)head * p.q_h + (long)t * p.q_n);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, load_chunk<PAD>(q, 2 * ks + h, p.d));
    win_sign(p.scale, qf);
    const float cs = win_scale(p.scale);
    WinRows<D> acc;
    acc.init();
    FragAddrs<D> fo;
    FragOffsets<D> offsets;
    offsets.init(lane);
    fo.init(offsets);
    fo.shift_transposed(kTile);
    char* mine = smem + w * (kFewStages<D, SRC> * 2 * kTile);  // [stage][K, V]
    PageWindow pages;
    pages.init();

    constexpr int kInst = 32 / CopyLane<D>::kRows, kChunks = D / 32;
    CodeChunk kc[SRC == kCodes ? kChunks : 1], vc[SRC == kCodes ? kChunks : 1];
    auto request = [&](int it, char* stage) {
        const int j0 = tiles.start(it);
        pages.cover(p, b, tiles.row(p, j0), tiles.row(p, j0 + 31), tiles.end, lane);
        if constexpr (SRC == kPages) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was read from the stage is in registers
#pragma unroll
            for (int u = 0; u < kInst; ++u) {
                const int row = CopyLane<D>::row_of(u, lane), j = tiles.row(p, j0 + row);
                const long at = win_page_row(p, pages.page(p, j), kvh, j).at * 2;
                copy_row(CopyLane<D>::template at<PAD>(static_cast<const char*>(p.K) + at, row, lane, p.d), lds_address(stage + u * 1024));
                copy_row(CopyLane<D>::template at<PAD>(static_cast<const char*>(p.V) + at, row, lane, p.d), lds_address(stage + kTile + u * 1024));
            }
        } else {
#pragma unroll
            for (int x = 0; x < kChunks; ++x) {
                const int idx = x * 64 + lane, j = tiles.row(p, j0 + idx / (D / 16));
                const PageRow r = win_page_row(p, pages.page(p, j), kvh, j);
                const long at = r.at + 16 * (idx % (D / 16));
                kc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.K) + at);
                vc[x].codes = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p.V) + at);
                kc[x].scale = exp_value(p.K_exp[r.exp]);
                vc[x].scale = exp_value(p.V_exp[r.exp]);
            }
        }
    };
    int it = it0 + w, stage = 0;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) settle(qf[ks]);
    if (it < it1) request(it, mine);
    for (; it < it1; it += NW) {
        const int j0 = tiles.start(it);
        const bool more = it + NW < it1;
        const char* lds = mine + stage;
        if constexpr (SRC == kPages) {
            stage ^= 2 * kTile;
            if (more) {
                request(it + NW, mine + stage);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * kInst) : "memory");
            } else {
                wait_direct_loads();
            }
        } else {
#pragma unroll
            for (int x = 0; x < kChunks; ++x) {
                const int idx = x * 64 + lane, row = idx / (D / 16), c = 2 * (idx % (D / 16));
                kc[x].to_lds(mine + tile_off<D>(row, c), mine + tile_off<D>(row, c + 1));
                vc[x].to_lds(mine + kTile + tile_off<D>(row, c), mine + kTile + tile_off<D>(row, c + 1));
            }
            wave_exchange();
            if (more) request(it + NW, mine);
        }
        f32x16 st[1];
#pragma unroll
        for (int i = 0; i < 16; ++i) st[0][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) st[0] = mfma32(fo.frag(lds, 0, 0, ks), qf[ks], st[0]);
        settle_products(st[0]);
        acc.weights(st, cs, !see.all(p, it, j0, 31), [&] { return see.template keys<1>(p, it, j0, 4 * h); });
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bf16x8 pb = acc_to_operand(st[0], x);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc.o[mt] = mfma32(fo.frag_t(lds, 0, mt, 16 * x), pb, acc.o[mt]);
        }
        wave_exchange();
    }

    // the waves meet: [wave][32 rows][D + 4] fp32, then [wave][32][m, l]
    constexpr int kPitch = D * 4 + 16;
    float l = acc.l + __shfl_xor(acc.l, 32, 64);
    __syncthreads();
    float* ml = reinterpret_cast<float*>(smem + NW * 32 * kPitch);
    if (h == 0) {
        ml[(w * 32 + l32) * 2] = acc.m;
        ml[(w * 32 + l32) * 2 + 1] = l;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            *reinterpret_cast<f32x4*>(smem + (w * 32 + l32) * kPitch + (32 * mt + 8 * g + 4 * h) * 4) =
                f32x4{acc.o[mt][4 * g], acc.o[mt][4 * g + 1], acc.o[mt][4 * g + 2], acc.o[mt][4 * g + 3]};
    __syncthreads();
    few_store<D, NW, 32, PAD>(p, s, smem, ml, kvh, r0, r1, at, tiles.count);
}

// ---------------------------------------------------------------------------------------------------------- a row tile
// Single tokens: at most 16 rows of a (sequence, key head), on 16x16x32 products, with half the registers, half the matrix cycles and half the
// softmax arithmetic of 32 rows.  K goes from memory straight into operands: lane (l % 16, q = l / 16) reads 16 bytes of key l % 16, and
// 64 bytes of each of 16 rows make an instruction.  The order of d inside a product is free as long as Q has the same:
//   bf16   product ks: columns 32 ks + 8 q ..             codes   products 2 kk, 2 kk + 1: columns 64 kk + 16 q .., + 8 ..
// V goes through 32 rows of LDS that only this wave uses, for the transposing reads.  The next tile is in registers or on its way to them while
// this one is worked on.  C: column l % 16 (query), register i of group g <-> key 16 g + 4 q + i, and as an operand with k = 4 g + i.
template <int D, int SRC>
constexpr int kOneLds = 4 * (32 * D * 2 > 16 * (D * 4 + 16) + 128 ? 32 * D * 2 : 16 * (D * 4 + 16) + 128);
// workgroups of four waves on a CU that the registers allow
template <int D, int SRC>
constexpr int kOnePerCu = D == 64 ? 4 : D == 128 ? 3 : SRC == kCodes ? 2 : 1;

template <int D, int SRC, bool PAD, bool TREE>
__device__ __forceinline__ void win_one(const WinParams& p) {
    constexpr int NW = 4, MT = D / 16, KS = D / 32, kTile = 32 * D * 2;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, l16 = lane & 15;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    Share<16, 32, TREE> at;
    at.init(p, (int)(blockIdx.x / p.kv_heads), lane);
    if (!at.any) return;
    const int b = at.b, kvh = blockIdx.x % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = at.blk * 16;
    if (r0 >= rows) return;
    const int r1 = min(r0 + 15, rows - 1);
    int t, head;
    win_place(p, kvh, min(r0 + l16, r1), t, head);
    const int t_lo = win_token(p, r0), t_hi = win_token(p, r1);
    Sight<32, TREE> see;
    see.init(p, s, t, t_lo, t_hi, t_lo, t_hi);
    const auto& tiles = see.tiles;
    const int it0 = at.first(p, tiles.count), it1 = at.last(p, tiles.count);

    PageWindow pages;
    pages.init();
    // bf16: kr[g * KS + ks], vr[x]: 16 bytes of rows x * 64 / (D / 8) ..   codes: kr[g * KS / 2 + kk], with the scales of the rows
    constexpr int kK = SRC == kCodes ? KS : 2 * KS, kV = SRC == kCodes ? D / 32 : D / 16, kChunksPerRow = SRC == kCodes ? D / 16 : D / 8;
    u32x4 kr[kK], vr[kV];
    uint8_t ke[2], ve[SRC == kCodes ? kV : 1];
    auto request = [&](int it) {
        constexpr int es = SRC == kCodes ? 1 : 2;
        const int j0 = tiles.start(it);
        pages.cover(p, b, tiles.row(p, j0), tiles.row(p, j0 + 31), tiles.end, lane);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int j = tiles.row(p, j0 + 16 * g + l16);
            const PageRow r = win_page_row(p, pages.page(p, j), kvh, j);
            const char* src = static_cast<const char*>(p.K) + r.at * es;
#pragma unroll
            for (int x = 0; x < kK / 2; ++x) kr[g * (kK / 2) + x] = load_chunk<PAD>(src, 4 * x + q, p.d);
            if constexpr (SRC == kCodes) ke[g] = p.K_exp[r.exp];
        }
#pragma unroll
        for (int x = 0; x < kV; ++x) {
            const int idx = x * 64 + lane, j = tiles.row(p, j0 + idx / kChunksPerRow);
            const PageRow r = win_page_row(p, pages.page(p, j), kvh, j);
            vr[x] = load_chunk<PAD>(static_cast<const char*>(p.V) + r.at * es, idx % kChunksPerRow, p.d);
            if constexpr (SRC == kCodes) ve[x] = p.V_exp[r.exp];
        }
    };
    int it = it0 + w;
    if (it < it1) request(it);

    bf16x8 qf[KS];
    const char* qrow = reinterpret_cast<const char*>(static_cast<const __bf16*>(p.Q) + s.q_base + (long)head * p.q_h + (long)t * p.q_n);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = __builtin_bit_cast(bf16x8, load_chunk<PAD>(qrow, SRC == kCodes ? 8 * (ks >> 1) + 2 * q + (ks & 1) : 4 * ks + q, p.d));
    win_sign(p.scale, qf);
    const float cs = win_scale(p.scale);
    f32x4 o[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -__builtin_inff(), l = 0.f;  // l: this lane's quarter of the sum
    char* mine = smem + w * kTile;
    // column 16 mt + l % 16 of keys 4 q .. + 3 (and 16 further): see load_frag_t
    const int tr_row = 4 * q + (l16 >> 2), tr = tile_off<D>(tr_row, (l16 & 3) >> 1) + ((l16 & 1) << 3);

    for (; it < it1; it += NW) {
        const int j0 = tiles.start(it);
        f32x4 st[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int x = 0; x < kK / 2; ++x) {
                const u32x4 v = kr[g * (kK / 2) + x];
                if constexpr (SRC == kCodes) {
                    const float scale = exp_value(ke[g]);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        u32x4 a;
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * half + y], scale, false);
                            const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * half + y], scale, true);
                            a[2 * y] = __builtin_bit_cast(uint32_t, lo);
                            a[2 * y + 1] = __builtin_bit_cast(uint32_t, hi);
                        }
                        st[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), qf[2 * x + half], st[g], 0, 0, 0);
                    }
                } else {
                    st[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v), qf[x], st[g], 0, 0, 0);
                }
            }
        }
#pragma unroll
        for (int x = 0; x < kV; ++x) {
            const int idx = x * 64 + lane, row = idx / kChunksPerRow, c = idx % kChunksPerRow;
            if constexpr (SRC == kCodes) {
                CodeChunk chunk;
                chunk.codes = vr[x];
                chunk.scale = exp_value(ve[x]);
                chunk.to_lds(mine + tile_off<D>(row, 2 * c), mine + tile_off<D>(row, 2 * c + 1));
            } else {
                *reinterpret_cast<u32x4*>(mine + tile_off<D>(row, c)) = vr[x];
            }
        }
        wave_exchange();
        if (it + NW < it1) request(it + NW);
        if (!see.all(p, it, j0, 31)) {
            const auto seen = see.template keys<1>(p, it, j0, 4 * q);
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) st[g][i] = seen(0, 16 * g + i) ? st[g][i] : -__builtin_inff();
        }
        float mx = max3(max3(st[0][0], st[0][1], st[0][2]), max3(st[0][3], st[1][0], st[1][1]), __builtin_elementwise_maximum(st[1][2], st[1][3]));
        constexpr float kSlack = 8.f;  // see WinRows
        if (__builtin_amdgcn_ballot_w64(mx * cs > m + kSlack) != 0) {
            mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 16, 64));
            mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 32, 64));
            const float cand = mx * cs, m_new = cand > m + kSlack ? cand : m;
            const float alpha = __builtin_amdgcn_exp2f(m - (m_new == -__builtin_inff() ? 0.f : m_new));
            l *= alpha;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt] *= alpha;
            m = m_new;
        }
        const float m_use = m == -__builtin_inff() ? 0.f : m;
        float f[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            f[x] = __builtin_amdgcn_exp2f(fmaf(st[x >> 2][x & 3], cs, -m_use));
            l += f[x];
        }
        const u32x4 pb = {pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const int at = (tr ^ ((mt & 7) << 5)) + 256 * (mt >> 3);
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 ATTN_LDS*)(mine + at));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((i16x4 ATTN_LDS*)(mine + at + 16 * D * 2));
            typedef short i16x8 __attribute__((ext_vector_type(8)));
            const i16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, pb), o[mt], 0, 0, 0);
        }
        wave_exchange();
    }

    constexpr int kPitch = D * 4 + 16;  // the waves meet: [wave][16 rows][D + 4] fp32, then [wave][16][m, l]
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    __syncthreads();
    float* ml = reinterpret_cast<float*>(smem + NW * 16 * kPitch);
    if (q == 0) {
        ml[(w * 16 + l16) * 2] = m;
        ml[(w * 16 + l16) * 2 + 1] = l;
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) *reinterpret_cast<f32x4*>(smem + (w * 16 + l16) * kPitch + (16 * mt + 4 * q) * 4) = o[mt];
    __syncthreads();
    few_store<D, NW, 16, PAD>(p, s, smem, ml, kvh, r0, r1, at, tiles.count);
}

}  // namespace
}  // namespace attn
