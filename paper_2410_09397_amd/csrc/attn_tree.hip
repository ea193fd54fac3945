// Trees of drafted tokens: which of them each sees, from the token that each follows; and their attention in 32-bit arithmetic (the kernels of
// attn_win_plain.hpp with the tiles and masks of a tree).
#include "attn_win_plain.hpp"

namespace attn {
namespace {

// (three sequences of 50 to 777 tokens with 21 to 37 drafted, h6 k2 d = 80, window 128: 16 us, waits for operands as without a tree)
template <typename T, typename E, int DP>
__global__ void __launch_bounds__(kThreads, DP <= 96 ? 2 : 1) tree_plain_out_kernel(WinParams p) {
    constexpr int MT = DP / 32;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Share<32, 32, true> share;
    share.init(p, (int)(blockIdx.x / p.kv_heads), lane);
    if (!share.any) return;
    const int b = share.b, kvh = blockIdx.x % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = share.blk * 32;
    if (r0 >= rows) return;
    const RowPlace at = place(p, kvh, min(r0 + l32, rows - 1));
    Sight<32, true> see;
    see.init(p, s, at.t, 0, 0, 0, 0);
    const auto& tiles = see.tiles;
    const int it0 = share.first(p, tiles.count), it1 = share.last(p, tiles.count);

    RowOperand<T, DP> q;
    q.init(static_cast<const T*>(p.Q) + s.q_base + (long)at.head * p.q_h + (long)at.t * p.q_n, p.d, h);
    f32x16 o[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] = 0.f;
    float m_run = -__builtin_inff(), l_run = 0.f;  // of scale log2(e) s; this lane's half of the sum
    const float cs = p.scale * kLog2e;
    for (int it = it0 + w; it < it1; it += 4) {
        const int j0 = tiles.start(it);
        KeyTile<E, true> keys;
        keys.init(p, tiles, b, kvh, j0, l32);
        f32x16 st;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = 0.f;
        TileRow<E, DP> key;
        key.init(keys.K + keys.at, p.d, h);
        scores(st, key, keys.sk, q);
        const auto seen = see.template keys<1>(p, it, j0, 4 * h);
        float mx = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            st[e] = seen(0, 8 * (e >> 2) + (e & 3)) ? st[e] * cs : -__builtin_inff();
            mx = __builtin_elementwise_maximum(mx, st[e]);
        }
        plain_weights<E, DP, true>(p, keys, h, l32, st, mx, o, m_run, l_run);
    }
    plain_store<T, MT>(p, s, at, share, tiles.count, r0, rows, w, lane, o, m_run, l_run);
}

// The sums of a row's parts, as win_join_kernel, for the parts of TreeItems.  A workgroup takes `many` rows of a row block, so that its sequence, its parts and their
// places are looked up once for all of them; 16 to 64 lanes have a row.  Row blocks of one part are written where they are worked on.  34 MB of sums of one sequence of 65536 tokens: 8 us.
template <typename T, int BR, int LANES>
__global__ void __launch_bounds__(kThreads) tree_join_kernel(WinParams p, int many) {
    constexpr int BC = tree_tile(BR), kPer = 64 / LANES;
    const int turns = BR / many, lane = threadIdx.x & 63, in_row = threadIdx.x & (LANES - 1), idx = blockIdx.x / (p.kv_heads * turns);
    const int kvh = blockIdx.x / turns % p.kv_heads, row0 = blockIdx.x % turns * many;
    TreeItems<BR, BC> items;
    items.init(p, lane);
    int start, blocks = 1, parts = 0, blk = 0;
    const int b = items.find_block(p, idx, lane, start, blocks, parts, blk);
    if (b < 0 || parts <= 1) return;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group;
    const long step = (long)blocks * p.kv_heads * BR, first = ((long)(start + blk) * p.kv_heads + kvh) * BR;  // row x, part k: first + x + k * step
    for (int x = row0 + (int)threadIdx.x / LANES; x < row0 + many; x += kThreads / LANES) {
        const int r = blk * BR + x;
        if (r >= rows) break;
        float m_k[kPer], l_k[kPer], m = -__builtin_inff(), l = 0.f;
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
            const int k = y * LANES + in_row;
            const float* ml = p.part_ml + (first + x + (long)min(k, parts - 1) * step) * 2;
            m_k[y] = k < parts ? ml[0] : -__builtin_inff();
            l_k[y] = k < parts ? ml[1] : 0.f;
            m = __builtin_elementwise_maximum(m, m_k[y]);
        }
#pragma unroll
        for (int y = 1; y < LANES; y <<= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, y, 64));
        const float m_use = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
        for (int y = 0; y < kPer; ++y) {
            m_k[y] = l_k[y] != 0.f ? __builtin_amdgcn_exp2f(m_k[y] - m_use) : 0.f;  // (NaN: not 0)
            l += m_k[y] * l_k[y];
        }
#pragma unroll
        for (int y = 1; y < LANES; y <<= 1) l += __shfl_xor(l, y, 64);
        const bool none = l == 0.f;
        const float inv = none ? 0.f : 1.f / l;
        const int c = 4 * in_row, at = lane & ~(LANES - 1);
        const float* src = p.part_o + (first + x) * p.d;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        constexpr int kAhead = 8;
#pragma unroll
        for (int y = 0; y < kPer; ++y)
            for (int k0 = 0; k0 < LANES && y * LANES + k0 < parts; k0 += kAhead) {
                f32x4 part[kAhead];
                float weight[kAhead];
#pragma unroll
                for (int a = 0; a < kAhead; ++a) {
                    const int k = min(y * LANES + k0 + a, parts - 1);
                    weight[a] = __shfl(m_k[y], at + k0 + a, 64);  // (0 behind the last part)
                    part[a] = load4(src + (long)k * step * p.d, c, p.d);
                }
#pragma unroll
                for (int a = 0; a < kAhead; ++a)
                    if (weight[a] != 0.f) sum += part[a] * weight[a];
            }
        const int t = win_token(p, r), head = kvh * p.group + r - t * p.group;
        if (c < p.d) store4(static_cast<T*>(p.O) + s.q_base + (long)head * p.q_h + (long)t * p.q_n, c, p.d, sum * inv);
        if (in_row == 0) p.LSE[(s.row0 + t) * p.heads + head] = none ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}

// One workgroup per sequence.  A token's row of words is written from the last word down, as the way up its branch passes the tokens of each: the steps are
// reads of LDS that wait for one another, as many as the branch is long, and every word is written once, without a word of LDS for it.  A
// token that does not follow an earlier one of its sequence follows the context, so the way up always ends.  2 us, 5 with cold caches (doubling the step of the
// way up instead, on masks of a wave's lanes, changed neither).
__global__ void __launch_bounds__(kThreads) tree_mask_kernel(WinParams p, const int32_t* parents, uint32_t* mask) {
    __shared__ int up[kMostDrafted];
    const int b = blockIdx.x;
    const int row0 = p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n;
    const int count = min(p.q_ptr ? min(max(p.q_ptr[b + 1] - row0, 0), p.total_q - row0) : p.n, p.n), words = (p.n + 31) >> 5;
    for (int t = threadIdx.x; t < count; t += kThreads) {
        const int v = parents[row0 + t];
        up[t] = v < t ? max(v, -1) : -1;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += kThreads) {
        uint32_t* row = mask + (long)(row0 + t) * p.tree_stride;
        int at = t;
        for (int w = words - 1; w >= 0; --w) {
            uint32_t bits = 0;
            while (at >= 32 * w) {  // (at < 0: the context, below every word)
                bits |= 1u << (at & 31);
                at = up[at];
            }
            row[w] = bits;
        }
    }
}

template <typename T, typename E>
hipError_t fwd(long grid, const WinParams& p, hipStream_t stream) {
    return with_width(p.d, [&](auto width) {
        constexpr int DP = decltype(width)::value;
        hipLaunchKernelGGL((tree_plain_out_kernel<T, E, DP>), dim3((unsigned)grid), dim3(kThreads), DP * 128 + 1024, stream, p);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_tree_plain_fwd(bool is_bf16, bool fp8, long grid, const WinParams& p, hipStream_t stream) {
    if (!p.table || !p.tree) return hipErrorInvalidValue;
    if (fp8) return is_bf16 ? fwd<__bf16, uint8_t>(grid, p, stream) : fwd<float, uint8_t>(grid, p, stream);
    return fwd<float, float>(grid, p, stream);
}
hipError_t launch_tree_join(bool is_bf16, int rows, const WinParams& p, hipStream_t stream) {
    if (!tree_rows_exist(is_bf16, rows)) return hipErrorInvalidValue;
    const int many = join_rows((int64_t)p.blocks * p.kv_heads, rows);
    auto with = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        auto fn = !is_bf16 ? tree_join_kernel<float, 32, L> : rows == 16 ? tree_join_kernel<__bf16, 16, L> : rows == 32 ? tree_join_kernel<__bf16, 32, L>
                  : tree_join_kernel<__bf16, 128, L>;
        hipLaunchKernelGGL(fn, dim3((unsigned)((long)p.blocks * p.kv_heads * (rows / many))), dim3(kThreads), 0, stream, p, many);
    };
    if (p.d <= 64) with(std::integral_constant<int, 16>{});
    else if (p.d <= 128) with(std::integral_constant<int, 32>{});
    else with(std::integral_constant<int, 64>{});
    return hipGetLastError();
}
hipError_t launch_tree_mask(const WinParams& p, const int32_t* parents, uint32_t* mask, hipStream_t stream) {
    if (p.n > kMostDrafted) return hipErrorInvalidValue;
    hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)p.batch), dim3(kThreads), 0, stream, p, parents, mask);
    return hipGetLastError();
}

}  // namespace attn
