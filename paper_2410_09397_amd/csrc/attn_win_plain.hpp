// Windowed attention in 32-bit arithmetic (attn_win_plain.hip says how): how its operands are read, and what the forward kernels, over tensors, over
// pages and over pages whose last tokens are a tree of drafted ones, have in common.  HIP device code only.
#pragma once
#include <type_traits>

#include "attn_internal.hpp"
#include "attn_win_tiles.hpp"

namespace attn {
namespace {

__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(8)));

// A kernel of width DP serves head dimensions in (kFull<DP>, DP]: the columns below kFull<DP> exist without a question.  The others are read from inside
// the row and replaced by 0 where they do not exist: a load behind a condition is waited for where it stands, and the loads of a tile have
// to be on their way together.
template <int DP>
constexpr int kFull = DP == 192 ? 128 : DP == 256 ? 192 : DP - 32;

// columns c .. c + 3 of a row, c a multiple of 4
template <int DP>
__device__ __forceinline__ f32x4 load4(const float* row, int c, bool exists, int d) {
    if (exists) return *reinterpret_cast<const f32x4u*>(row + c);
    f32x4 v;
    if constexpr (DP == 32) {  // (d may be less than 4)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = row[min(c + e, d - 1)];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c + e < d ? v[e] : 0.f;
    } else {
        // four values that end with the row's last one, moved down by as many places as they start early
        const int start = min(c, d - 4), s = c - start;
        v = *reinterpret_cast<const f32x4u*>(row + start);
        if (s & 1) v = f32x4{v[1], v[2], v[3], 0.f};
        if (s & 2) v = f32x4{v[2], v[3], 0.f, 0.f};
        if (s >= 4) v = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    return v;
}
template <int DP>
__device__ __forceinline__ f32x4 load4(const __bf16* row, int c, bool exists, int d) {  // (d is a multiple of 8)
    const f32x4 v = __builtin_convertvector(*reinterpret_cast<const bf16x4u*>(row + (exists ? c : min(c, d - 4))), f32x4), zero = {0.f, 0.f, 0.f, 0.f};
    return exists || c < d ? v : zero;
}
template <int DP>
__device__ __forceinline__ f32x4 load4(const uint8_t* row, int c, bool exists, int d) {
    int u = *reinterpret_cast<const int*>(row + (exists ? c : min(c, d - 4)));
    u = exists || c < d ? u : 0;
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(u, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint8_t x) { return __builtin_amdgcn_cvt_f32_fp8((int)x, 0); }
// column 32 m + l of a row; CHECK, first: m counts from a group of columns that the compiler does not know
template <int DP, bool CHECK = false, typename E>
__device__ __forceinline__ float load1(const E* row, int m, int l, int d, int first = 0) {
    const int c = 32 * (first + m) + l;
    if (!CHECK && 32 * m + 32 <= kFull<DP>) return value(row[c]);
    const float v = value(row[min(c, d - 1)]);
    return c < d ? v : 0.f;
}
// of any width, for the small kernels
__device__ __forceinline__ f32x4 load4(const float* row, int c, int d) {
    if (c + 4 <= d) return *reinterpret_cast<const f32x4u*>(row + c);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (c + e < d) v[e] = row[c + e];
    return v;
}
__device__ __forceinline__ void store4(float* row, int c, int d, f32x4 v) {
    if (c + 4 <= d) {
        *reinterpret_cast<f32x4u*>(row + c) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (c + e < d) row[c + e] = v[e];
}
__device__ __forceinline__ void store4(__bf16* row, int c, int d, f32x4 v) {
    if (c < d) *reinterpret_cast<u32x2*>(row + c) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
}

// A resident row as the contraction over d takes it: 4 values of columns 8 c + 4 h .. for every c.  bf16 rows stay packed; rows that
// have no registers to stay in are read again for every tile.
template <typename T, int DP>
struct RowOperand {
    static constexpr bool kResident = DP <= (std::is_same_v<T, __bf16> ? 192 : 128);
    typedef std::conditional_t<std::is_same_v<T, __bf16>, u32x2, f32x4> Chunk;
    Chunk v[kResident ? DP / 8 : 1];
    const T* row;
    int d, h;
    __device__ __forceinline__ f32x4 load(int c) const { return load4<DP>(row, 8 * c + 4 * h, 8 * c + 8 <= kFull<DP>, d); }
    __device__ __forceinline__ void init(const T* row_, int d_, int h_) {
        row = row_;
        d = d_;
        h = h_;
        if constexpr (kResident) {
#pragma unroll
            for (int c = 0; c < DP / 8; ++c) {
                const f32x4 x = load(c);
                if constexpr (std::is_same_v<T, __bf16>) v[c] = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
                else v[c] = x;
            }
        }
    }
    __device__ __forceinline__ f32x4 get(int c) const {
        if constexpr (!kResident) return load(c);
        else if constexpr (std::is_same_v<T, __bf16>) return __builtin_convertvector(__builtin_bit_cast(bf16x4, v[c]), f32x4);
        else return v[c];
    }
};

// The 32 rows of a key tile as a lane sees them: row l % 32 for the contraction over d, every row for the contraction over keys.  Rows of
// tensors are 32-bit offsets from the tile's first (q_n, k_n < 2^22), rows of pages lie anywhere.
template <typename E, bool PAGED>
struct KeyTile {
    static constexpr bool kCodes = std::is_same_v<E, uint8_t>;
    std::conditional_t<PAGED, long, unsigned> at;  // element offset of row l % 32
    const E *K, *V;
    float sk, sv;  // quantised: what its codes are multiplied with
    template <typename Tiles>
    __device__ __forceinline__ void init(const WinParams& p, const Tiles& tiles, int b, int kvh, int j0, int l32) {
        const int j = tiles.row(p, j0 + l32);
        K = static_cast<const E*>(p.K);
        V = static_cast<const E*>(p.V);
        if constexpr (PAGED) {
            const PageRow r = win_page_row(p, win_page(p, b, j), kvh, j);
            at = r.at;
            if constexpr (kCodes) {
                sk = exp_value(p.K_exp[r.exp]);
                sv = exp_value(p.V_exp[r.exp]);
            }
        } else {
            const long base = (long)b * p.k_b + (long)kvh * p.k_h + (long)j0 * p.k_n;
            K += base;
            V += base;
            at = (unsigned)(j - j0) * (unsigned)p.k_n;
        }
    }
    // offset of the row that another lane holds
    __device__ __forceinline__ auto row_of(int row) const {
        if constexpr (PAGED) {
            const int lo = __shfl((int)at, row, 64), hi = __shfl((int)(at >> 32), row, 64);
            return ((long)hi << 32) | (unsigned)lo;
        } else {
            return (unsigned)__shfl((int)at, row, 64);
        }
    }
};

// Wide rows: the loads of at most `every` steps are on the way together (of more the compiler spills the addresses).
template <int DP>
__device__ __forceinline__ void pause(int step, int every) {
    if (DP >= 192 && step % every == every - 1) __builtin_amdgcn_sched_barrier(0);
}

// A row of the tile (l % 32) for the contraction over d.  Narrow widths: all of its loads are requested by init(), so that those of
// several rows and of what follows are on their way together; wide ones read it as they go.
template <typename E, int DP>
struct TileRow {
    static constexpr bool kAhead = DP <= 128;
    f32x4 v[kAhead ? DP / 8 : 1];
    const E* row;
    int d, h;
    __device__ __forceinline__ f32x4 load(int c) const { return load4<DP>(row, 8 * c + 4 * h, 8 * c + 8 <= kFull<DP>, d); }
    __device__ __forceinline__ void init(const E* row_, int d_, int h_) {
        row = row_;
        d = d_;
        h = h_;
        if constexpr (kAhead) {
#pragma unroll
            for (int c = 0; c < DP / 8; ++c) v[c] = load(c);
        }
    }
    __device__ __forceinline__ f32x4 get(int c) const {
        if constexpr (kAhead) return v[c];
        else return load(c);
    }
};

// s += A B^T over d: a's rows are the tile's, b's the resident ones
template <typename E, typename T, int DP>
__device__ __forceinline__ void scores(f32x16& s, const TileRow<E, DP>& row, float scale, const RowOperand<T, DP>& b) {
#pragma unroll
    for (int c = 0; c < DP / 8; ++c) {
        f32x4 a = row.get(c);
        if constexpr (std::is_same_v<E, uint8_t>) a *= scale;
        const f32x4 q = b.get(c);
#pragma unroll
        for (int e = 0; e < 4; ++e) s = mfma_f32(a[e], q[e], s);
        pause<DP>(c, 8);
    }
}

// Products over the rows of a tile, in groups of 4 accumulator registers: use(e, x) has what load(e, x) gave for x < N (columns of one or two tensors);
// the loads of a group are requested in front of the products of the one before.
template <int N, int DP, typename Load, typename Use>
__device__ __forceinline__ void by_rows(Load load, Use use) {
    float v[2][4][N];
    auto request = [&](int g) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int x = 0; x < N; ++x) v[g & 1][e][x] = load(4 * g + e, x);
    };
    request(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (g < 3) request(g + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int x = 0; x < N; ++x) use(4 * g + e, x, v[g & 1][e][x]);
    }
}

struct RowPlace {  // of query row r of a (sequence, key head)
    int t, head;
};
__device__ __forceinline__ RowPlace place(const WinParams& p, int kvh, int r) {
    const int t = win_token(p, r);
    return {t, kvh * p.group + r - t * p.group};
}

// a: the sum of the four waves' accumulators, for wave 0, in the order of the waves; `meet`: 4 MT KB
template <int MT>
__device__ __forceinline__ void meet_waves(f32x16 (&a)[MT], float* meet, int w, int lane) {
    auto slot = [&](int m, int x) { return reinterpret_cast<f32x4*>(meet) + (m * 4 + x) * 64 + lane; };
    for (int from = 1; from < 4; ++from) {
        if (w == from) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int x = 0; x < 4; ++x) *slot(m, x) = f32x4{a[m][4 * x], a[m][4 * x + 1], a[m][4 * x + 2], a[m][4 * x + 3]};
        }
        __syncthreads();
        if (w == 0) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const f32x4 other = *slot(m, x);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[m][4 * x + e] += other[e];
                }
        }
        __syncthreads();
    }
}

// --------------------------------------------------------------------------------------------------------- forward
// What the forward kernels (attn_win_plain.hip, and over trees attn_tree.hip) have in common.  A tile's rows and which of its keys a row sees stand in the kernels themselves
// (win_plain_out_kernel says why).

// A tile's scores times scale log2(e) (-inf: not seen; mx: the lane's largest) become weights of the running reference, and their products with V are added to O.
template <typename E, int DP, bool PAGED>
__device__ __forceinline__ void plain_weights(const WinParams& p, const KeyTile<E, PAGED>& keys, int h, int l32, f32x16& st, float mx, f32x16 (&o)[DP / 32], float& m_run,
                                              float& l_run) {
    constexpr int MT = DP / 32;
    mx = __builtin_elementwise_maximum(mx, __shfl_xor(mx, 32, 64));
    const float m_new = __builtin_elementwise_maximum(m_run, mx), m_use = m_new == -__builtin_inff() ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
    m_run = m_new;
    l_run *= alpha;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] *= alpha;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        st[e] = __builtin_amdgcn_exp2f(st[e] - m_use);
        l_run += st[e];
    }
    if constexpr (KeyTile<E, PAGED>::kCodes) {
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] *= __shfl(keys.sv, acc_row(e, h), 64);
    }
    by_rows<MT, DP>([&](int e, int m) { return load1<DP>(keys.V + keys.row_of(acc_row(e, h)), m, l32, p.d); },
                    [&](int e, int m, float v) { o[m] = mfma_f32(v, st[e], o[m]); });
}

// The waves' sums of 32 rows meet and are stored, as O and LSE or (share) as those of a part.  at: the lane's row, r0: the workgroup's first.
template <typename T, int MT, typename S>
__device__ __forceinline__ void plain_store(const WinParams& p, const WinSeq& s, const RowPlace& at, const S& share, int tiles, int r0, int rows, int w, int lane,
                                            f32x16 (&o)[MT], float m_run, float l_run) {
    const int h = lane >> 5, l32 = lane & 31;
    // every wave's m and l, then its O in units of the common reference
    float l = l_run + __shfl_xor(l_run, 32, 64);
    extern __shared__ __attribute__((aligned(16))) float meet[];  // [MT][4][64] x 16 bytes, [4][m, l][32]
    float* stats = meet + MT * 4 * 64 * 4;
    if (h == 0) {
        stats[w * 64 + l32] = m_run;
        stats[w * 64 + 32 + l32] = l;
    }
    __syncthreads();
    float m_all = stats[l32];
#pragma unroll
    for (int x = 1; x < 4; ++x) m_all = __builtin_elementwise_maximum(m_all, stats[x * 64 + l32]);
    const float m_ref = m_all == -__builtin_inff() ? 0.f : m_all, mine = __builtin_amdgcn_exp2f(m_run - m_ref);
    l = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) l += __builtin_amdgcn_exp2f(stats[x * 64 + l32] - m_ref) * stats[x * 64 + 32 + l32];
    m_run = m_all;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[m][e] *= mine;
    meet_waves<MT>(o, meet, w, lane);
    if (w != 0 || r0 + l32 >= rows) return;
    if (!share.whole(p, tiles)) {
        const long row = share.sums(p, s.lse_base + (long)at.t * p.heads + at.head, l32);
        float* ml = p.part_ml + row * 2;
        if (h == 0) {
            ml[0] = m_run;
            ml[1] = l;
        }
        if (l > 0.f || l != l) {
            float* dst = p.part_o + row * p.d;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    store4(dst, 32 * m + 8 * g + 4 * h, p.d, f32x4{o[m][4 * g], o[m][4 * g + 1], o[m][4 * g + 2], o[m][4 * g + 3]});
        }
        return;
    }
    const bool none = l == 0.f;  // no key: O = 0, LSE = -inf
    const float inv = none ? 0.f : 1.f / l;
    T* dst = static_cast<T*>(p.O) + s.q_base + (long)at.head * p.q_h + (long)at.t * p.q_n;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            store4(dst, 32 * m + 8 * g + 4 * h, p.d,
                   f32x4{o[m][4 * g] * inv, o[m][4 * g + 1] * inv, o[m][4 * g + 2] * inv, o[m][4 * g + 3] * inv});
    if (h == 0)
        p.LSE[s.lse_base + (long)at.head * s.lse_h + (long)at.t * s.lse_t] =
            none ? -__builtin_inff() : (m_run + __builtin_amdgcn_logf(l)) * kLn2;
}

// f(width): see kFull
template <typename F>
hipError_t with_width(int d, F f) {
    if (d <= 32) return f(std::integral_constant<int, 32>{});
    if (d <= 64) return f(std::integral_constant<int, 64>{});
    if (d <= 96) return f(std::integral_constant<int, 96>{});
    if (d <= 128) return f(std::integral_constant<int, 128>{});
    if (d <= 192) return f(std::integral_constant<int, 192>{});
    return f(std::integral_constant<int, 256>{});
}

}  // namespace
}  // namespace attn
