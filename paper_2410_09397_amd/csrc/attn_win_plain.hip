// Windowed attention in 32-bit arithmetic: forward over tensors or pages and backward for fp32 storage at any d <= 256, and the forward
// over quantised pages at the head dimensions that attn_win_fwd.hip does not have.
//
// Products are v_mfma_f32_32x32x2_f32.  Operand layout (lane l, h = l / 32): A row l % 32, k = h; B column l % 32, k = h; C as for the
// bf16 form (column l % 32, register i <-> row 8 (i / 4) + 4 h + i % 4).  The order of k is free as long as both operands have the same:
//   contraction over d     step (c, e) takes columns 8 c + e (h = 0) and 8 c + 4 + e (h = 1): a lane reads 4 values at a time
//   contraction over rows  step i takes the rows of accumulator register i, which is then an operand as it stands
// A workgroup owns 32 rows of queries or keys; its four waves take the tiles that stream past in turn, each reading its operands straight from memory
// (any layout of the rows will do) into accumulators of its own, which meet in LDS at the end: a short window is only a handful of tiles, and a tile
// takes a wave 64 cycles for every 2 x 32 of its products.  What bounds them is the wait for those reads, not the products (four dependent trips to a tile: 49 to 63 % of the
// wave cycles wait, the matrix pipe is 16 to 19 % busy; the kernels of attn_stream.hip, which stage whole rows in LDS, keep it 45 to 65 % busy).  us of a step, full causal
// through those -> windowed through these, b2 h6: n777 d80 w128 81 -> 101 (two key heads) and 118 (six), w64 81 -> 81, n1500 d64 w128 159 -> 135,
// n2048 d64 w128 278 -> 149; without a window b2 h16 n1000 d96 287 -> 840.
#include <type_traits>

#include "attn_internal.hpp"
#include "attn_window.hpp"

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
    __device__ __forceinline__ void init(const WinParams& p, const WinTiles<32>& tiles, int b, int kvh, int j0, int l32) {
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
template <typename T, typename E, int DP, bool PAGED>
__global__ void __launch_bounds__(kThreads, DP <= 96 ? 2 : 1) win_plain_out_kernel(WinParams p, int row_blocks) {
    constexpr int MT = DP / 32;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int b, kvh, blk;
    if constexpr (PAGED) {
        WinBlock block;
        block.init(p, (int)(blockIdx.x / p.kv_heads), 32, lane);
        if (!block.any) return;
        b = block.b;
        kvh = blockIdx.x % p.kv_heads;
        blk = block.blk;
    } else {
        const int bk = blockIdx.x / row_blocks;
        b = bk / p.kv_heads;
        kvh = bk % p.kv_heads;
        blk = blockIdx.x % row_blocks;
    }
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = blk * 32;
    if (r0 >= rows) return;
    const int r = min(r0 + l32, rows - 1);
    const RowPlace at = place(p, kvh, r);
    const int i = s.first + at.t;
    const int hi = i < s.len ? i : -1, lo = i - p.window + 1;  // this row sees lo .. hi, and the sinks up to hi
    WinTiles<32> tiles;
    tiles.init(p, s.len, s.first + place(p, kvh, r0).t, s.first + place(p, kvh, min(r0 + 31, rows - 1)).t);
    const int it0 = blockIdx.y * p.chunk, it1 = min(tiles.count, it0 + p.chunk);

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
        KeyTile<E, PAGED> keys;
        keys.init(p, tiles, b, kvh, j0, l32);
        f32x16 st;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = 0.f;
        TileRow<E, DP> key;
        key.init(keys.K + keys.at, p.d, h);
        scores(st, key, keys.sk, q);
        float mx = -__builtin_inff();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = j0 + acc_row(e, h);
            const bool seen = j <= hi && (j >= lo || j < p.sinks);
            st[e] = seen ? st[e] * cs : -__builtin_inff();
            mx = __builtin_elementwise_maximum(mx, st[e]);
        }
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
    if (p.splits > 1) {
        const long row = s.lse_base + (long)at.t * p.heads + at.head;
        float* ml = p.part_ml + (row * p.splits + blockIdx.y) * 2;
        if (h == 0) {
            ml[0] = m_run;
            ml[1] = l;
        }
        if (l > 0.f || l != l) {
            float* dst = p.part_o + (row * p.splits + blockIdx.y) * p.d;
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

// The sums of the parts of a row: O = sum_k 2^(m_k - m) O_k / l, l = sum_k 2^(m_k - m) l_k, always in the same order.  WAVES waves per row; every
// one reads all m_k, l_k (at most 64, one per lane); 16 to 64 lanes share a part's O_k, so that a row has 1 to 16 parts on the way
// at a time.  Parts that saw no key have no O_k.  (One wave per row and one part at a time: 21 us for 32 rows of 63 parts, now 5.)
template <typename T, int WAVES>
__global__ void __launch_bounds__(kThreads) win_join_kernel(WinParams p) {
    __shared__ f32x4 meet[kThreads];
    const int lane = threadIdx.x & 63, in_row = threadIdx.x % (64 * WAVES);
    const long row = ((long)blockIdx.x * kThreads + threadIdx.x) / (64 * WAVES);
    const int token = (int)(row / p.heads), head = (int)(row % p.heads);
    if (token >= p.total_q) return;  // (all waves of a row)
    const float* ml = p.part_ml + row * p.splits * 2;
    const bool mine = lane < p.splits;
    const float m_k = mine ? ml[2 * lane] : -__builtin_inff(), l_k = mine ? ml[2 * lane + 1] : 0.f;
    // which sequence the row belongs to is looked up while its sums are on their way; of a row of no sequence they mean nothing, and nothing is written
    const int b = win_sequence_of(p, __builtin_amdgcn_readfirstlane(token), lane);
    const WinSeq s = win_sequence(p, max(b, 0));
    const int t = b < 0 ? -1 : token - (int)(s.lse_base / p.heads);
    float m = m_k;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) m = __builtin_elementwise_maximum(m, __shfl_xor(m, x, 64));
    const float m_use = m == -__builtin_inff() ? 0.f : m;
    const float f_k = l_k != 0.f ? __builtin_amdgcn_exp2f(m_k - m_use) : 0.f;  // (NaN: not 0)
    float l = f_k * l_k;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x, 64);
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    const int lanes = p.d <= 64 ? 16 : p.d <= 128 ? 32 : 64, slots = 64 * WAVES / lanes, slot = in_row / lanes, c = 4 * (in_row % lanes);
    const float* src = p.part_o + row * p.splits * p.d;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAhead = 4;  // parts per lane on the way
    for (int k0 = 0; k0 < p.splits; k0 += kAhead * slots) {
        f32x4 part[kAhead];
        float weight[kAhead];
#pragma unroll
        for (int x = 0; x < kAhead; ++x) {
            const int k = k0 + x * slots + slot, kc = min(k, p.splits - 1);
            weight[x] = __shfl(f_k, kc, 64);  // (by all lanes)
            if (k >= p.splits) weight[x] = 0.f;
            part[x] = load4(src + (long)kc * p.d, c, p.d);
        }
#pragma unroll
        for (int x = 0; x < kAhead; ++x)
            if (weight[x] != 0.f) sum += part[x] * weight[x];
    }
    for (int x = lanes; x < 64; x <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], x, 64);
    if constexpr (WAVES > 1) {
        meet[threadIdx.x] = sum;
        __syncthreads();
        if (in_row >= 64) return;
#pragma unroll
        for (int x = 1; x < WAVES; ++x) sum += meet[threadIdx.x + 64 * x];
    }
    if (t < 0 || t >= s.nq || lane >= lanes) return;
    T* dst = static_cast<T*>(p.O) + s.q_base + (long)head * p.q_h + (long)t * p.q_n;
    if (c < p.d) store4(dst, c, p.d, sum * inv);
    if (lane == 0) p.LSE[row] = none ? -__builtin_inff() : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// -------------------------------------------------------------------------------------------------------- backward
// delta = rowsum(dO o O) of every query inside its sequence, [batch, heads, n]; eight lanes per row.
__global__ void __launch_bounds__(kThreads) win_rows_kernel(WinParams p) {
    const long f = ((long)blockIdx.x * kThreads + threadIdx.x) >> 3, rows = (long)p.batch * p.heads * p.n;
    const int c0 = 4 * (threadIdx.x & 7);
    float sum = 0.f;
    if (f < rows) {
        const int t = (int)(f % p.n), bh = (int)(f / p.n);
        const long at = (long)(bh / p.heads) * p.q_b + (long)(bh % p.heads) * p.q_h + (long)t * p.q_n;
        if (!p.lens || t < p.lens[bh / p.heads])
            for (int c = c0; c < p.d; c += 32) {
                const f32x4 x = load4(static_cast<const float*>(p.O_in) + at, c, p.d), g = load4(static_cast<const float*>(p.dO) + at, c, p.d);
                sum += x[0] * g[0] + x[1] * g[1] + x[2] * g[2] + x[3] * g[3];
            }
    }
#pragma unroll
    for (int x = 1; x < 8; x <<= 1) sum += __shfl_xor(sum, x, 64);
    if (f < rows && (threadIdx.x & 7) == 0) p.delta[f] = sum;
}

// dQ: a workgroup owns 32 query rows, its waves take the key tiles in turn and their sums meet in LDS; dS^T = P^T o (V dO^T - delta), dQ^T += K^T dS^T.
template <int DP>
__global__ void __launch_bounds__(kThreads, DP <= 96 ? 2 : 1) win_plain_dq_kernel(WinParams p, int row_blocks) {
    constexpr int MT = DP / 32;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bk = blockIdx.x / row_blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, r0 = (blockIdx.x % row_blocks) * 32;
    if (r0 >= rows) return;
    const int r = min(r0 + l32, rows - 1);
    const RowPlace at = place(p, kvh, r);
    const int i = s.first + at.t;
    const int hi = i < s.len ? i : -1, lo = i - p.window + 1;
    WinTiles<32> tiles;
    tiles.init(p, s.len, s.first + place(p, kvh, r0).t, s.first + place(p, kvh, min(r0 + 31, rows - 1)).t);
    const long off = s.q_base + (long)at.head * p.q_h + (long)at.t * p.q_n, stat = s.lse_base + (long)at.head * s.lse_h + at.t;
    RowOperand<float, DP> q, g;
    q.init(static_cast<const float*>(p.Q) + off, p.d, h);
    g.init(static_cast<const float*>(p.dO) + off, p.d, h);
    const float lse = hi >= 0 ? p.LSE_in[stat] * kLog2e : 0.f, delta = hi >= 0 ? p.delta[stat] : 0.f;
    f32x16 dq[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[m][e] = 0.f;
    const float cs = p.scale * kLog2e;
    for (int it = w; it < tiles.count; it += 4) {
        const int j0 = tiles.start(it);
        KeyTile<float, false> keys;
        keys.init(p, tiles, b, kvh, j0, l32);
        f32x16 st, dp;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = dp[e] = 0.f;
        TileRow<float, DP> key, val;
        key.init(keys.K + keys.at, p.d, h);
        val.init(keys.V + keys.at, p.d, h);
        scores(st, key, 1.f, q);
        scores(dp, val, 1.f, g);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int j = j0 + acc_row(e, h);
            const bool seen = j <= hi && (j >= lo || j < p.sinks);
            dp[e] = seen ? __builtin_amdgcn_exp2f(fmaf(st[e], cs, -lse)) * (dp[e] - delta) : 0.f;
        }
        by_rows<MT, DP>([&](int e, int m) { return load1<DP>(keys.K + keys.row_of(acc_row(e, h)), m, l32, p.d); },
                        [&](int e, int m, float v) { dq[m] = mfma_f32(v, dp[e], dq[m]); });
    }
    extern __shared__ __attribute__((aligned(16))) float meet[];
    meet_waves<MT>(dq, meet, w, lane);
    if (w != 0 || r0 + l32 >= rows) return;
    float* dst = static_cast<float*>(p.dQ) + off;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            store4(dst, 32 * m + 8 * x + 4 * h, p.d,
                   f32x4{dq[m][4 * x] * p.scale, dq[m][4 * x + 1] * p.scale, dq[m][4 * x + 2] * p.scale, dq[m][4 * x + 3] * p.scale});
}

// dK, dV: a workgroup owns 32 keys; its waves take the 32-token tiles of all heads of the group in turn, with scores [query][key], which
// are the operands of dV^T += dO^T P and dK^T += Q^T dS as they stand.  The waves' sums meet in LDS.  d > 128: the columns of the gradients are shared by two workgroups
// (blockIdx.y), which both form the scores; one would need 600 registers per lane.
template <int DP>
__global__ void __launch_bounds__(kThreads, 1) win_plain_dkdv_kernel(WinParams p, int key_blocks) {
    constexpr int MT = DP >= 192 ? DP / 64 : DP / 32;
    extern __shared__ __attribute__((aligned(16))) float meet[];  // [MT][4][64] x 16 bytes
    const int m0 = MT * blockIdx.y, c0 = 32 * m0;  // first column of the gradients
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bk = blockIdx.x / key_blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    WinKeys own;
    own.init(p, blockIdx.x % key_blocks, 32, s.len);
    const int j0 = own.j0, i0 = own.i0, i1 = own.i1, j = j0 + l32;
    const long kv = (long)b * p.k_b + (long)kvh * p.k_h;
    const int t_tiles = (i1 - i0 + 31) / 32, jobs = t_tiles * p.group;
    const int jr = max(0, min(j, s.len - 1));
    RowOperand<float, DP> k, v;
    k.init(static_cast<const float*>(p.K) + kv + (long)jr * p.k_n, p.d, h);
    v.init(static_cast<const float*>(p.V) + kv + (long)jr * p.k_n, p.d, h);
    f32x16 dk[MT], dv[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[m][e] = dv[m][e] = 0.f;
    const float cs = p.scale * kLog2e;
    for (int job = w; job < jobs; job += 4) {
        const int head = kvh * p.group + job / t_tiles, t0 = i0 + 32 * (job % t_tiles);
        // 32-bit offsets from the tile's first row; rows past the end repeat the last one
        const long base = s.q_base + (long)head * p.q_h + (long)t0 * p.q_n, stat = s.lse_base + (long)head * s.lse_h + t0;
        const float *Q = static_cast<const float*>(p.Q) + base, *G = static_cast<const float*>(p.dO) + base;
        const float *lse = p.LSE_in + stat, *delta = p.delta + stat;
        const int last = i1 - 1 - t0;
        const unsigned q_n = (unsigned)p.q_n, mine = (unsigned)min(l32, last) * q_n;
        f32x16 st, dp;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = dp[e] = 0.f;
        TileRow<float, DP> query, grad;
        query.init(Q + mine, p.d, h);
        grad.init(G + mine, p.d, h);
        float lse_x[16], delta_x[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            lse_x[e] = lse[min(acc_row(e, h), last)];
            delta_x[e] = delta[min(acc_row(e, h), last)];
        }
        __builtin_amdgcn_sched_barrier(0);
        scores(st, query, 1.f, k);
        scores(dp, grad, 1.f, v);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int x = acc_row(e, h), i = t0 + x;
            const bool seen = x <= last && j <= i && (i - j < p.window || j < p.sinks);
            st[e] = seen ? __builtin_amdgcn_exp2f(fmaf(st[e], cs, -lse_x[e] * kLog2e)) : 0.f;
            dp[e] = seen ? st[e] * (dp[e] - delta_x[e]) : 0.f;
        }
        by_rows<2 * MT, DP>(
            [&](int e, int x) {
                const unsigned row = (unsigned)min(acc_row(e, h), last) * q_n;
                return load1<DP, (DP >= 192)>((x < MT ? G : Q) + row, x % MT, l32, p.d, m0);
            },
            [&](int e, int x, float y) {
                if (x < MT) dv[x] = mfma_f32(y, st[e], dv[x]);
                else dk[x - MT] = mfma_f32(y, dp[e], dk[x - MT]);
            });
    }
    meet_waves<MT>(dk, meet, w, lane);
    meet_waves<MT>(dv, meet, w, lane);
    if (w != 0 || j >= p.n) return;
    if (own.slot >= 0) {
        float* dst = p.part_kv + ((long)bk * p.slots + own.slot) * 2 * 32 * p.d + (long)l32 * p.d;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                store4(dst, c0 + 32 * m + 8 * x + 4 * h, p.d, f32x4{dk[m][4 * x], dk[m][4 * x + 1], dk[m][4 * x + 2], dk[m][4 * x + 3]} * p.scale);
                store4(dst + 32 * p.d, c0 + 32 * m + 8 * x + 4 * h, p.d, f32x4{dv[m][4 * x], dv[m][4 * x + 1], dv[m][4 * x + 2], dv[m][4 * x + 3]});
            }
        return;
    }
    const long out = kv + (long)j * p.k_n;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            store4(static_cast<float*>(p.dK) + out, c0 + 32 * m + 8 * x + 4 * h, p.d, f32x4{dk[m][4 * x], dk[m][4 * x + 1], dk[m][4 * x + 2], dk[m][4 * x + 3]} * p.scale);
            store4(static_cast<float*>(p.dV) + out, c0 + 32 * m + 8 * x + 4 * h, p.d, f32x4{dv[m][4 * x], dv[m][4 * x + 1], dv[m][4 * x + 2], dv[m][4 * x + 3]});
        }
}

// dK and dV of keys whose tiles several workgroups work on: the sum of the parts, in their order.  16 to 64 lanes per row.
template <typename T>
__global__ void __launch_bounds__(kThreads) win_keys_kernel(WinParams p, int tile, int keys) {
    const int lanes = p.d <= 64 ? 16 : p.d <= 128 ? 32 : 64;
    const long f = ((long)blockIdx.x * kThreads + threadIdx.x) / lanes;
    const int c = 4 * (int)(threadIdx.x & (lanes - 1));
    if (f >= (long)p.batch * p.kv_heads * keys * 2 || c >= p.d) return;
    const int which = (int)(f & 1), j = (int)((f >> 1) % keys), bk = (int)((f >> 1) / keys), x = j / tile;
    const bool sink = x < p.sink_tiles;
    const int parts = sink ? p.parts : p.rest_parts, slot = sink ? x * p.parts : p.sink_tiles * p.parts + (x - p.sink_tiles) * p.rest_parts;
    const float* src = p.part_kv + (((long)bk * p.slots + slot) * 2 + which) * tile * p.d + (long)(j % tile) * p.d;
    T* dst = static_cast<T*>(which ? p.dV : p.dK) + (long)(bk / p.kv_heads) * p.k_b + (long)(bk % p.kv_heads) * p.k_h + (long)j * p.k_n;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    constexpr int kAhead = 8;  // parts on the way
    for (int k0 = 0; k0 < parts; k0 += kAhead) {
        f32x4 v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) v[k] = load4(src + (long)min(k0 + k, parts - 1) * 2 * tile * p.d, c, p.d);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (k0 + k < parts) sum += v[k];
    }
    store4(dst, c, p.d, sum);
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

template <typename T, typename E, bool PAGED>
hipError_t fwd(const WinParams& p, hipStream_t stream) {
    const int blocks = (int)(((long)p.n * p.group + 31) / 32);
    return with_width(p.d, [&](auto width) {
        hipLaunchKernelGGL((win_plain_out_kernel<T, E, decltype(width)::value, PAGED>), dim3((unsigned)((PAGED ? (long)p.blocks : (long)blocks * p.batch) * p.kv_heads), (unsigned)p.splits),
                           dim3(kThreads), decltype(width)::value * 128 + 1024, stream, p, blocks);
        return hipGetLastError();
    });
}

hipError_t bwd(const WinParams& p, hipStream_t stream) {
    const int blocks = (int)(((long)p.n * p.group + 31) / 32), keys = p.sink_tiles * p.parts + ((p.n + 31) / 32 - p.sink_tiles) * p.rest_parts;
    return with_width(p.d, [&](auto width) {
        constexpr int DP = decltype(width)::value;
        hipLaunchKernelGGL((win_plain_dq_kernel<DP>), dim3((unsigned)((long)blocks * p.batch * p.kv_heads)), dim3(kThreads), DP * 128, stream, p, blocks);
        hipLaunchKernelGGL((win_plain_dkdv_kernel<DP>), dim3((unsigned)((long)keys * p.batch * p.kv_heads), DP >= 192 ? 2 : 1), dim3(kThreads),
                           (DP >= 192 ? DP / 2 : DP) * 128, stream, p, keys);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_win_plain_fwd(bool is_bf16, bool fp8, const WinParams& p, hipStream_t stream) {
    if (fp8) return is_bf16 ? fwd<__bf16, uint8_t, true>(p, stream) : fwd<float, uint8_t, true>(p, stream);
    return p.table ? fwd<float, float, true>(p, stream) : fwd<float, float, false>(p, stream);
}
hipError_t launch_win_plain_bwd(const WinParams& p, hipStream_t stream) { return bwd(p, stream); }
hipError_t launch_win_join(bool is_bf16, const WinParams& p, hipStream_t stream) {
    // four waves for a row that has many parts
    const int waves = p.splits > 8 ? 4 : 1;
    const dim3 grid((unsigned)(((long)p.total_q * p.heads * waves + 3) / 4));
    auto fn = is_bf16 ? (waves == 4 ? win_join_kernel<__bf16, 4> : win_join_kernel<__bf16, 1>)
                      : (waves == 4 ? win_join_kernel<float, 4> : win_join_kernel<float, 1>);
    hipLaunchKernelGGL(fn, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}
hipError_t launch_win_rows(const WinParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)(((long)p.batch * p.heads * p.n * 8 + kThreads - 1) / kThreads));
    hipLaunchKernelGGL(win_rows_kernel, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
}
hipError_t launch_win_keys(bool is_bf16, int tile, const WinParams& p, hipStream_t stream) {
    const int keys = p.rest_parts > 1 || p.sink_tiles * tile > p.n ? p.n : p.sink_tiles * tile;
    const dim3 grid((unsigned)(((long)p.batch * p.kv_heads * keys * 2 * (p.d <= 64 ? 16 : p.d <= 128 ? 32 : 64) + kThreads - 1) / kThreads));
    if (is_bf16) hipLaunchKernelGGL(win_keys_kernel<__bf16>, grid, dim3(kThreads), 0, stream, p, tile, keys);
    else hipLaunchKernelGGL(win_keys_kernel<float>, grid, dim3(kThreads), 0, stream, p, tile, keys);
    return hipGetLastError();
}

}  // namespace attn
