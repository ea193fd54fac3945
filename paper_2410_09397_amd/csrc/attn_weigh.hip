// How much attention the new tokens pay to every token of the paged cache: weight_j = decay weight_j + sum_r exp(scale <q_r, k_j> - LSE_r) over the rows r
// (new tokens times heads of a group, see attn_window.hpp) that see token j.  LSE is the attention's own, so one pass over K is all there is: no
// maximum, no second product, and the weights stay in 32 bits.
//
// S = Q K^T with keys in the columns: a lane has one key and some rows in its registers, so that the sum over rows is an addition per value and ends
// with one exchange between the lanes of a key.  No two workgroups add to the same weight: the same call gives the same bits.
#include "attn_win_plain.hpp"

namespace attn {
namespace {

// Rows r0 .. r1 - 1 are those that see some of the keys j0 .. j1 of a sequence (j1 < len), in multiples of BR.
template <int BR>
struct WeighRows {
    int r0, r1;
    __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s, int j0, int j1) {
        const int t0 = max(0, j0 - s.first);
        const int t1 = j0 < p.sinks ? s.nq : (int)min((long)s.nq, max(0l, (long)j1 + p.window - s.first));
        r0 = t0 * p.group / BR * BR;
        r1 = t1 * p.group;
    }
};

// Row r of a (sequence, key head): its position, or -1 where it sees nothing or adds nothing (whatever its Q holds), and what its exponents are relative to (+inf: weights 0).
struct WeighRow {
    int i;
    float lse2;
    __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s, int kvh, int r, int rows) {
        const int x = min(r, rows - 1), t = win_token(p, x), head = kvh * p.group + x - t * p.group;
        const float lse = p.LSE_in[(s.row0 + t) * p.heads + head];
        const bool adds = r < rows && s.first + t < s.len && lse != -__builtin_inff();
        i = adds ? s.first + t : -1;
        lse2 = adds ? lse * kLog2e : __builtin_inff();
    }
};
__device__ __forceinline__ bool weigh_sees(const WinParams& p, int i, int j) { return j <= i && (i - j < p.window || j < p.sinks); }

__device__ __forceinline__ void weigh_store(const WeighParams& w, const WinSeq& s, int b, int kvh, int j, float sum) {
    if (j >= s.len) return;
    float v = sum;
    if (w.in && j < s.first) v = fmaf(w.decay, w.in[(long)b * w.in_b + (long)kvh * w.in_h + j], sum);
    w.out[(long)b * w.out_b + (long)kvh * w.out_h + j] = v;
}

// Which keys a workgroup takes: chunk `part` of a sequence.  The chunks of all sequences are counted, so that those of short ones leave no workgroups idle
// among those of long ones; what the host has launched too many lies at the end.  (More than 64 sequences fill the chip whatever their lengths are, and each has w.blocks.)
struct WeighShare {
    int b, part;
    bool any;
    __device__ __forceinline__ void init(const WinParams& p, int idx, int chunk, int blocks, int lane) {
        if (p.batch > 64) {
            b = idx / blocks;
            part = idx - b * blocks;
            any = part * (long)chunk < min(max(p.lens[b], 0), p.max_len);
            return;
        }
        any = true;
        const int own = lane < p.batch ? (min(max(p.lens[lane], 0), p.max_len) + chunk - 1) / chunk : 0;
        int upto = own;
        for (int x = 1; x < p.batch; x <<= 1) {
            const int before = __shfl_up(upto, x, 64);
            upto += lane >= x ? before : 0;
        }
        const unsigned long who = __builtin_amdgcn_ballot_w64(lane < p.batch && upto > idx);
        if (who) {
            b = __builtin_ctzl(who);
            part = idx - __builtin_amdgcn_readlane(upto - own, b);
            return;
        }
        any = false;
        b = part = 0;
    }
};

// 16 codes as two chunks of 8 bf16, exactly
__device__ __forceinline__ bf16x8 code_half(u32x4 v, int half, float scale) {
    u32x4 a;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const bf16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * half + y], scale, false);
        const bf16x2 hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[2 * half + y], scale, true);
        a[2 * y] = __builtin_bit_cast(uint32_t, lo);
        a[2 * y + 1] = __builtin_bit_cast(uint32_t, hi);
    }
    return __builtin_bit_cast(bf16x8, a);
}

// Keys of GROUP columns of a product (16: 16x16x32, 32: 32x32x16), straight from memory into operands: lane l has key l % GROUP, and of it 16 bytes of every 64 / GROUP.  The
// order of d inside a product is free as long as Q has the same: operand x of codes that lie together (a lane's 16 bytes are 8 columns twice).
template <int D, int SRC, int GROUP, bool PAD>
struct KeyOperand {
    static constexpr int kProducts = D * GROUP / 512, kLoads = SRC == kCodes ? kProducts / 2 : kProducts, kQuarters = 64 / GROUP;
    u32x4 raw[kLoads];
    uint8_t exp;
    // key j (clamped by the caller) in page `page`
    __device__ __forceinline__ void request(const WinParams& p, int page, int kvh, int j, int lane) {
        const PageRow r = win_page_row(p, page, kvh, j);
        const char* src = static_cast<const char*>(p.K) + r.at * (SRC == kCodes ? 1 : 2);
#pragma unroll
        for (int x = 0; x < kLoads; ++x) raw[x] = load_chunk<PAD>(src, kQuarters * x + lane / GROUP, p.d);
        if constexpr (SRC == kCodes) exp = p.K_exp[r.exp];
    }
    __device__ __forceinline__ bf16x8 operand(int x, float scale) const {
        if constexpr (SRC == kCodes) return code_half(raw[x / 2], x % 2, scale);
        else return __builtin_bit_cast(bf16x8, raw[x]);
    }
    // the 8 columns of a row of Q that go with operand x: their number in units of 8
    static __device__ __forceinline__ int chunk_of(int x, int lane) {
        return SRC == kCodes ? 2 * (kQuarters * (x / 2) + lane / GROUP) + x % 2 : kQuarters * x + lane / GROUP;
    }
};

// At most 16 rows (ONE), on 16x16x32 products with Q in registers, or any number, 16 at a time from memory (rows that the other kernels' tiles do not hold).  32 keys to a wave, the
// next ones on their way.  Memory bounds it: the newest token of 64 sequences of 100 to 8192, h32 k8 d = 128, quantised, 31 us, 4.3 TB/s.
template <int D, int SRC, bool PAD, bool ONE>
__global__ void __launch_bounds__(kThreads) weigh_one_kernel(WeighParams w) {
    const WinParams& p = w.p;
    typedef KeyOperand<D, SRC, 16, PAD> Keys;
    constexpr int KS = Keys::kProducts;
    const int lane = threadIdx.x & 63, q = lane >> 4, l16 = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kvh = blockIdx.x % p.kv_heads;
    WeighShare share;
    share.init(p, blockIdx.x / p.kv_heads, w.chunk, w.blocks, lane);
    if (!share.any) return;
    const int b = share.b;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, end = min(s.len, (share.part + 1) * w.chunk);
    const float cs = p.scale * kLog2e;
    int j0 = share.part * w.chunk + 32 * wave;
    PageWindow pages;
    pages.init();
    Keys keys[2];
    auto request = [&] {
        pages.cover(p, b, j0, min(j0 + 31, s.len - 1), s.len, lane);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int j = min(j0 + 16 * g + l16, s.len - 1);
            keys[g].request(p, pages.page(p, j), kvh, j, lane);
        }
    };
    if (j0 < end) request();
    bf16x8 qf[KS];
    WeighRow at[4];
    auto load_rows = [&](int r0) {
        const int x = min(r0 + l16, rows - 1), t = win_token(p, x), head = kvh * p.group + x - t * p.group;
        const char* row = reinterpret_cast<const char*>(static_cast<const __bf16*>(p.Q) + s.q_base + (long)head * p.q_h + (long)t * p.q_n);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, load_chunk<PAD>(row, Keys::chunk_of(ks, lane), p.d));
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i].init(p, s, kvh, r0 + 4 * q + i, rows);
    };
    if (ONE && rows > 0) load_rows(0);
    while (j0 < end) {
        const int here = j0;
        bf16x8 kf[2][KS];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const float scale = SRC == kCodes ? exp_value(keys[g].exp) : 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[g][ks] = keys[g].operand(ks, scale);
        }
        j0 += 128;
        if (j0 < end) request();
        float sum[2] = {0.f, 0.f};
        WeighRows<16> range;
        range.init(p, s, here, min(here + 31, s.len - 1));
        for (int r0 = range.r0; r0 < range.r1; r0 += 16) {
            if (!ONE) load_rows(r0);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                f32x4 st = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], kf[g][ks], st, 0, 0, 0);
                const int j = here + 16 * g + l16;
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[g] += weigh_sees(p, at[i].i, j) ? __builtin_amdgcn_exp2f(fmaf(st[i], cs, -at[i].lse2)) : 0.f;
            }
        }
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            sum[g] += __shfl_xor(sum[g], 16, 64);
            sum[g] += __shfl_xor(sum[g], 32, 64);
        }
        const float v = q & 1 ? sum[1] : sum[0];
        if (q < 2) weigh_store(w, s, b, kvh, here + 16 * q + l16, v);
    }
}

// ----------------------------------------------------------------------------------------------------- rows in tiles
// More rows lie in LDS as tiles of 128: TT tokens with their heads, TT = 128 / group, so that a tile's rows are at the same distances from its first as every other tile's.
// Beside each row: its position (-1: none, or nothing that it adds) and what its exponents are relative to.
typedef int i32x4 __attribute__((ext_vector_type(4)));
constexpr int kWeighTile = 128;
template <int D>
struct WeighStage {
    __bf16 rows[kWeighTile * D];  // swizzled as the tiles of attn_common.hpp
    float lse2[kWeighTile];
    int pos[kWeighTile];
    int whole[4];  // of 32 rows each: every one has a position
};

// 32 rows of a stage times 32 NG keys: the weights that these rows give the lane's keys.  masked: not every row sees every key.
template <int D, int SRC, int NG, bool PAD>
__device__ __forceinline__ void weigh_rows(const WinParams& p, const WeighStage<D>& stage, int row0, const bf16x8 (&kf)[NG][D / 16], int j, float cs, bool masked, int lane,
                                           float (&sum)[NG]) {
    typedef KeyOperand<D, SRC, 32, PAD> Keys;
    const int h = lane >> 5, row = row0 + (lane & 31);
    const char* lds = reinterpret_cast<const char*>(stage.rows) + row * (2 * D);
    f32x16 st[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) st[g][i] = 0.f;
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const bf16x8 q = *reinterpret_cast<const bf16x8*>(lds + ((Keys::chunk_of(x, lane) ^ swz<D>(row)) << 4));
#pragma unroll
        for (int g = 0; g < NG; ++g) st[g] = mfma32(q, kf[g][x], st[g]);
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) settle_products(st[g]);
    f32x4 lse[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) lse[x] = *reinterpret_cast<const f32x4*>(stage.lse2 + row0 + 8 * x + 4 * h);
    if (masked) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const i32x4 pos = *reinterpret_cast<const i32x4*>(stage.pos + row0 + 8 * x + 4 * h);
#pragma unroll
            for (int g = 0; g < NG; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sum[g] += weigh_sees(p, pos[i], j + 32 * g) ? __builtin_amdgcn_exp2f(fmaf(st[g][4 * x + i], cs, -lse[x][i])) : 0.f;
        }
        return;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
        float a = 0.f, c = 0.f;  // (two chains: an addition waits for the one before)
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                a += __builtin_amdgcn_exp2f(fmaf(st[g][4 * x + i], cs, -lse[x][i]));
                c += __builtin_amdgcn_exp2f(fmaf(st[g][4 * x + i + 1], cs, -lse[x][i + 1]));
            }
        sum[g] += a + c;
    }
}

// A whole stage of rows (128 / group has no remainder, d up to 128) that all see all of 64 keys: the products of 32 rows and 32 keys are issued between the exponentials of the 32 keys before (the vector arithmetic takes
// longer than the matrix pipe: an exponential is four instructions' time).
template <int D, int SRC, bool PAD>
__device__ __forceinline__ void weigh_stage(const WeighStage<D>& stage, const bf16x8 (&kf)[2][D / 16], float cs, int lane, float (&sum)[2]) {
    typedef KeyOperand<D, SRC, 32, PAD> Keys;
    constexpr int KS = D / 16;
    const int h = lane >> 5, l32 = lane & 31;
    const char* lds = reinterpret_cast<const char*>(stage.rows) + l32 * (2 * D);
    bf16x8 q[2][KS];
    f32x16 st[2];
    f32x4 lse[4];
    auto fetch = [&](int x) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[x & 1][ks] = *reinterpret_cast<const bf16x8*>(lds + x * (64 * D) + ((Keys::chunk_of(ks, lane) ^ swz<D>(l32)) << 4));
    };
    auto products = [&](int x, int g) {
#pragma unroll
        for (int i = 0; i < 16; ++i) st[g][i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) st[g] = mfma32(q[x & 1][ks], kf[g][ks], st[g]);
    };
    auto weights = [&](int g) {
        float a = 0.f, c = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            a += __builtin_amdgcn_exp2f(fmaf(st[g][i], cs, -lse[i >> 2][i & 3]));
            c += __builtin_amdgcn_exp2f(fmaf(st[g][i + 1], cs, -lse[i >> 2][(i & 3) + 1]));
        }
        sum[g] += a + c;
    };
    auto mix = [&] {
#pragma unroll
        for (int y = 0; y < KS; ++y) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);        // one product
            __builtin_amdgcn_sched_group_barrier(0x2, 48 / KS, 0);  // and its share of the vector arithmetic
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    fetch(0);
    products(0, 0);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
#pragma unroll
        for (int y = 0; y < 4; ++y) lse[y] = *reinterpret_cast<const f32x4*>(stage.lse2 + 32 * x + 8 * y + 4 * h);
        if (x < 3) fetch(x + 1);
        __builtin_amdgcn_sched_barrier(0);
        products(x, 1);
        weights(0);
        mix();
        if (x < 3) products(x + 1, 0);
        weights(1);
        mix();
    }
}

// Brings tiles of rows into stages.  Tile `it` has tokens TT it .. of the sequence.
template <int D, bool PAD>
struct WeighFeed {
    static constexpr int kInst = kWeighTile / (4 * CopyLane<D>::kRows);
    unsigned off[kInst];  // of the lane's 16 bytes from the tile's first row, bytes
    int tt, token, g;     // tokens of a tile; of threads 0 .. 127: token and head of row `tid`
    float lse;
    int pos;
    __device__ __forceinline__ void init(const WinParams& p, int tid) {
        const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
        tt = kWeighTile / p.group;
#pragma unroll
        for (int u = 0; u < kInst; ++u) {
            const int row = CopyLane<D>::row_of(u * 4 + w, lane), t = min(win_token(p, row), tt - 1), g = min(row - t * p.group, p.group - 1);
            off[u] = ((unsigned)t * (unsigned)p.q_n + (unsigned)g * (unsigned)p.q_h) * 2u + 16u * ((lane % (D / 8)) ^ swz<D>(row));
        }
        token = win_token(p, tid & (kWeighTile - 1));
        g = (tid & (kWeighTile - 1)) - token * p.group;
    }
    __device__ __forceinline__ void request(const WinParams& p, const WinSeq& s, int kvh, int it, WeighStage<D>* stage, int tid) {
        const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), t0 = it * tt;
        if (tid < kWeighTile) {
            const bool is = token < tt && t0 + token < s.nq;
            lse = is ? p.LSE_in[(s.row0 + t0 + token) * p.heads + kvh * p.group + g] : -__builtin_inff();
            pos = is && lse != -__builtin_inff() && s.first + t0 + token < s.len ? s.first + t0 + token : -1;
        }
        const char* first = reinterpret_cast<const char*>(static_cast<const __bf16*>(p.Q) + s.q_base + (long)(kvh * p.group) * p.q_h + (long)t0 * p.q_n);
        const unsigned to = lds_address(stage->rows);
        if (!PAD && t0 + tt <= s.nq) {
#pragma unroll
            for (int u = 0; u < kInst; ++u) copy_to_lds<16, true>(to + w * 1024u, u * 4096, off[u], TileLoader<D, 64>::uniform(reinterpret_cast<const __bf16*>(first)));
        } else {
#pragma unroll
            for (int u = 0; u < kInst; ++u) {
                const int row = CopyLane<D>::row_of(u * 4 + w, lane), t = min(min(win_token(p, row), tt - 1), s.nq - 1 - t0), g = min(row - win_token(p, row) * p.group, p.group - 1);
                copy_row(CopyLane<D>::template at<PAD>(first + ((long)t * p.q_n + (long)g * p.q_h) * 2, row, lane, p.d), to + (u * 4 + w) * 1024u);
            }
        }
    }
    // the requested tile is in its stage once this and a barrier are past
    __device__ __forceinline__ void arrive(WeighStage<D>* stage, int tid) const {
        wait_direct_loads();
        if (tid < kWeighTile) {
            stage->lse2[tid] = lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;
            stage->pos[tid] = pos;
            const unsigned long has = __builtin_amdgcn_ballot_w64(pos >= 0);
            if ((tid & 31) == 0) stage->whole[tid >> 5] = (unsigned)(has >> (tid & 32)) == ~0u;
        }
    }
};

// Whether every row of a stage sees all of the keys j0 .. j1: t0 .. t1 - 1 are its tokens; none of its rows is without a position.
__device__ __forceinline__ bool weigh_whole(const WinParams& p, const WinSeq& s, int t0, int t1, int j0, int j1) {
    const int i0 = s.first + t0, i1 = s.first + t1 - 1;
    return j1 <= i0 && i1 < s.len && (i1 - j0 < p.window || j1 < p.sinks);
}

// Rows of one tile (a few new tokens): they stay in LDS, and the keys stream past, 32 to a wave, the next ones on their way.  Memory and the first tile's latency: the last 32
// tokens of 8 prompts, h32 k8 d = 128, 16 us, 3.2 TB/s.
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads, 2) weigh_few_kernel(WeighParams w) {
    const WinParams& p = w.p;
    typedef KeyOperand<D, SRC, 32, PAD> Keys;
    constexpr int KS = Keys::kProducts;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    WeighStage<D>* stage = reinterpret_cast<WeighStage<D>*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kvh = blockIdx.x % p.kv_heads;
    WeighShare share;
    share.init(p, blockIdx.x / p.kv_heads, w.chunk, w.blocks, lane);
    if (!share.any) return;
    const int b = share.b;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, end = min(s.len, (share.part + 1) * w.chunk);
    const float cs = p.scale * kLog2e;
    int j0 = share.part * w.chunk + 32 * wave;
    PageWindow pages;
    pages.init();
    Keys key;
    auto request = [&] {
        pages.cover(p, b, j0, min(j0 + 31, s.len - 1), s.len, lane);
        const int j = min(j0 + l32, s.len - 1);
        key.request(p, pages.page(p, j), kvh, j, lane);
    };
    if (rows > 0) {
        WeighFeed<D, PAD> feed;
        feed.init(p, tid);
        feed.request(p, s, kvh, 0, stage, tid);
        if (j0 < end) request();
        feed.arrive(stage, tid);
    } else if (j0 < end) {
        request();
    }
    __syncthreads();
    while (j0 < end) {
        const int here = j0;
        bf16x8 kf[1][KS];
        const float scale = SRC == kCodes ? exp_value(key.exp) : 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[0][ks] = key.operand(ks, scale);
        j0 += 128;
        if (j0 < end) request();
        float sum[1] = {0.f};
        WeighRows<32> range;
        range.init(p, s, here, min(here + 31, s.len - 1));
        const bool whole = weigh_whole(p, s, 0, s.nq, here, here + 31);
        for (int r0 = range.r0; r0 < range.r1; r0 += 32)
            weigh_rows<D, SRC, 1, PAD>(p, *stage, r0, kf, here + l32, cs, !whole || !__builtin_amdgcn_readfirstlane(stage->whole[r0 >> 5]), lane, sum);
        sum[0] += __shfl_xor(sum[0], 32, 64);
        if (lane < 32) weigh_store(w, s, b, kvh, here + l32, sum[0]);
    }
}

// Many rows: a workgroup has 256 keys, 64 in the operands of each wave, and tiles of rows stream past all of them.  Few keys, or those of a prompt that most rows see, are
// shared out: a workgroup takes one of w.parts shares of the tiles, and weigh_join_kernel adds up the sums, in their order.
// Exponentials and conversions bound it beside the matrix pipe (33 % busy): all of a prompt of 4096 tokens, h32 k8 d = 128, 97 us, 710 TFLOP/s.
constexpr int kWeighKeys = 256;
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads, (D == 256 ? 1 : 2)) weigh_many_kernel(WeighParams w) {
    const WinParams& p = w.p;
    typedef KeyOperand<D, SRC, 32, PAD> Keys;
    constexpr int KS = Keys::kProducts;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    WeighStage<D>* stages = reinterpret_cast<WeighStage<D>*>(smem);
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // most rows see the first keys of a sequence: these workgroups come first, and where all are on the chip at once the later half comes back from the last
    const int bk_total = p.batch * p.kv_heads, bk = blockIdx.x % bk_total, b = bk / p.kv_heads, kvh = bk % p.kv_heads, all = w.blocks * w.parts;
    int idx = blockIdx.x / bk_total;
    if ((long)all * bk_total <= 512 && idx >= (all + 1) / 2) idx = all - 1 - (idx - (all + 1) / 2);
    const int blk = idx / w.parts, part = idx - blk * w.parts;
    const WinSeq s = win_sequence(p, b);
    const int b0 = kWeighKeys * blk, b1 = min(b0 + kWeighKeys - 1, s.len - 1), j0 = b0 + 64 * wave, j1 = j0 + 63;
    if (b0 >= s.len) return;
    const float cs = p.scale * kLog2e;
    WeighFeed<D, PAD> feed;
    feed.init(p, tid);
    // tiles of tokens that see some of the keys, and this workgroup's share of them
    const int t_lo = max(0, b0 - s.first), t_hi = b0 < p.sinks ? s.nq : (int)min((long)s.nq, max(0l, (long)b1 + p.window - s.first));
    const int first = t_lo / feed.tt, tiles = t_hi > t_lo ? (t_hi + feed.tt - 1) / feed.tt - first : 0;
    const int it0 = first + (int)((long)tiles * part / w.parts), it1 = first + (int)((long)tiles * (part + 1) / w.parts);
    int tok0[4], tok1[4];  // first and last token of 32 rows of a tile
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        tok0[x] = __builtin_amdgcn_readfirstlane(win_token(p, 32 * x));
        tok1[x] = __builtin_amdgcn_readfirstlane(win_token(p, 32 * x + 31));
    }
    float sum[2] = {0.f, 0.f};
    if (it0 < it1) {
        feed.request(p, s, kvh, it0, stages, tid);
        bf16x8 kf[2][KS];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int j = min(j0 + 32 * g + l32, s.len - 1);
            Keys key;
            key.request(p, win_page(p, b, j), kvh, j, lane);
            const float scale = SRC == kCodes ? exp_value(key.exp) : 0.f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) kf[g][ks] = key.operand(ks, scale);
        }
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) settle(kf[g][ks]);
        feed.arrive(stages, tid);
        __syncthreads();
        for (int it = it0; it < it1; ++it) {
            const WeighStage<D>& stage = stages[(it - it0) & 1];
            WeighStage<D>* next = stages + ((it - it0 + 1) & 1);
            if (it + 1 < it1) feed.request(p, s, kvh, it + 1, next, tid);
            const int t0 = it * feed.tt, i0 = s.first + t0, i_end = s.first + s.nq - 1;
            const int i1 = min(i0 + tok1[3], i_end);
            const bool full = D <= 128 && j1 <= i0 && (i1 - j0 < p.window || j1 < p.sinks) &&
                              __builtin_amdgcn_readfirstlane(stage.whole[0] & stage.whole[1] & stage.whole[2] & stage.whole[3]);
            if (full) {
                if constexpr (D <= 128) weigh_stage<D, SRC, PAD>(stage, kf, cs, lane, sum);
            } else
#pragma unroll 1
            for (int x = 0; x < 4; ++x) {
                const int lo = i0 + tok0[x], hi = min(i0 + tok1[x], i_end);
                if (lo > i_end || hi < j0 || (lo - j1 >= p.window && j0 >= p.sinks)) continue;  // none of the rows sees any of the keys
                const bool whole = __builtin_amdgcn_readfirstlane(stage.whole[x]) && j1 <= lo && (hi - j0 < p.window || j1 < p.sinks);
                weigh_rows<D, SRC, 2, PAD>(p, stage, 32 * x, kf, j0 + l32, cs, !whole, lane, sum);
            }
            if (it + 1 < it1) feed.arrive(next, tid);
            __syncthreads();
        }
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) sum[g] += __shfl_xor(sum[g], 32, 64);
    const float v = lane < 32 ? sum[0] : sum[1];
    const int j = j0 + lane;
    if (w.parts == 1) weigh_store(w, s, b, kvh, j, v);
    else if (j < s.len) w.sums[((long)part * bk_total + bk) * p.max_len + j] = v;
}
__global__ void __launch_bounds__(kThreads) weigh_join_kernel(WeighParams w, int blocks) {
    const WinParams& p = w.p;
    const int bk = blockIdx.x / blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads, j = blockIdx.x % blocks * kThreads + threadIdx.x;
    const WinSeq s = win_sequence(p, b);
    if (j >= s.len) return;
    float sum = 0.f;
    for (int x = 0; x < w.parts; ++x) sum += w.sums[((long)x * p.batch * p.kv_heads + bk) * p.max_len + j];
    weigh_store(w, s, b, kvh, j, sum);
}

// 32-bit arithmetic: 32x32x2 products of 32 keys and 32 rows, both straight from memory.  At most 32 rows: every wave has keys of its own.  More (SHARED): the four waves have the
// same keys and take the rows in turn, and their sums meet in LDS (a tile of rows is 64 cycles for every two columns, and a small model has few keys to fill the chip with: 50 new
// tokens of 3 sequences, h6 k2 d = 80, 16.6 us with keys to each wave, 9.0 so).
template <typename T, typename E, int DP, bool SHARED>
__global__ void __launch_bounds__(kThreads, 1) weigh_plain_kernel(WeighParams w) {
    const WinParams& p = w.p;
    __shared__ float meet[4][32];
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blk = blockIdx.x % w.blocks, bk = blockIdx.x / w.blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, j0 = blk * w.chunk + (SHARED ? 0 : 32 * wave);
    if (j0 >= s.len) return;  // (SHARED: all waves)
    const int j = j0 + l32, at_j = min(j, s.len - 1);
    const PageRow place = win_page_row(p, win_page(p, b, at_j), kvh, at_j);
    RowOperand<E, DP> key;
    key.init(static_cast<const E*>(p.K) + place.at, p.d, h);
    float cs = p.scale * kLog2e;
    if constexpr (std::is_same_v<E, uint8_t>) cs *= exp_value(p.K_exp[place.exp]);
    float sum = 0.f;
    WeighRows<32> range;
    range.init(p, s, j0, min(j0 + 31, s.len - 1));
    for (int r0 = range.r0 + (SHARED ? 32 * wave : 0); r0 < range.r1; r0 += SHARED ? 128 : 32) {
        const int x = min(r0 + l32, rows - 1), t = win_token(p, x), head = kvh * p.group + x - t * p.group;
        TileRow<T, DP> row;
        row.init(static_cast<const T*>(p.Q) + s.q_base + (long)head * p.q_h + (long)t * p.q_n, p.d, h);
        WeighRow mine;
        mine.init(p, s, kvh, r0 + l32, rows);
        f32x16 st;
#pragma unroll
        for (int e = 0; e < 16; ++e) st[e] = 0.f;
        scores(st, row, 1.f, key);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int i = __shfl(mine.i, acc_row(e, h), 64);
            const float lse2 = __shfl(mine.lse2, acc_row(e, h), 64);
            sum += weigh_sees(p, i, j) ? __builtin_amdgcn_exp2f(fmaf(st[e], cs, -lse2)) : 0.f;
        }
    }
    sum += __shfl_xor(sum, 32, 64);
    if constexpr (SHARED) {
        if (h == 0) meet[wave][l32] = sum;
        __syncthreads();
        if (wave != 0) return;
        sum = (meet[0][l32] + meet[1][l32]) + (meet[2][l32] + meet[3][l32]);
    }
    if (h == 0) weigh_store(w, s, b, kvh, j, sum);
}

dim3 grid_of(const WeighParams& w) { return dim3((unsigned)((long)w.blocks * w.parts * w.p.batch * w.p.kv_heads)); }

template <int D, int SRC, bool PAD>
hipError_t launch_from(WeighRowsKind kind, const WeighParams& w, hipStream_t stream) {
    auto run = [&](auto kernel, int lds) {
        const hipError_t e = lds ? allow_lds(kernel, lds) : hipSuccess;
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid_of(w), dim3(kThreads), lds, stream, w);
        return hipGetLastError();
    };
    if (kind == kWeighOne) return run(weigh_one_kernel<D, SRC, PAD, true>, 0);
    if (kind == kWeighAny) return run(weigh_one_kernel<D, SRC, PAD, false>, 0);
    if (kind == kWeighFew) return run(weigh_few_kernel<D, SRC, PAD>, (int)sizeof(WeighStage<D>));
    const hipError_t e = run(weigh_many_kernel<D, SRC, PAD>, 2 * (int)sizeof(WeighStage<D>));
    if (e != hipSuccess || w.parts == 1) return e;
    const int blocks = (w.p.max_len + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(weigh_join_kernel, dim3((unsigned)((long)blocks * w.p.batch * w.p.kv_heads)), dim3(kThreads), 0, stream, w, blocks);
    return hipGetLastError();
}
template <int D>
hipError_t launch(bool fp8, WeighRowsKind kind, const WeighParams& w, hipStream_t stream) {
    if (fp8) return launch_from<D, kCodes, false>(kind, w, stream);
    return w.p.d < D ? launch_from<D, kPages, true>(kind, w, stream) : launch_from<D, kPages, false>(kind, w, stream);
}
template <typename T, typename E>
hipError_t plain(const WeighParams& w, hipStream_t stream) {
    return with_width(w.p.d, [&](auto width) {
        constexpr int DP = decltype(width)::value;
        auto fn = w.chunk == 32 ? weigh_plain_kernel<T, E, DP, true> : weigh_plain_kernel<T, E, DP, false>;
        hipLaunchKernelGGL(fn, grid_of(w), dim3(kThreads), 0, stream, w);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_weigh(bool fp8, WeighRowsKind kind, const WeighParams& w, hipStream_t stream) {
    if (fp8 && w.p.d != 64 && w.p.d != 128 && w.p.d != 256) return hipErrorInvalidValue;
    return w.p.d <= 64 ? launch<64>(fp8, kind, w, stream) : w.p.d <= 128 ? launch<128>(fp8, kind, w, stream) : launch<256>(fp8, kind, w, stream);
}
hipError_t launch_weigh_plain(bool is_bf16, bool fp8, const WeighParams& w, hipStream_t stream) {
    if (fp8) return is_bf16 ? plain<__bf16, uint8_t>(w, stream) : plain<float, uint8_t>(w, stream);
    return plain<float, float>(w, stream);
}

}  // namespace attn
