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

// Row r of a (sequence, key head): its position, or -1 where it sees nothing, and what its exponents are relative to (+inf: weights 0).
struct WeighRow {
    int i;
    float lse2;
    __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s, int kvh, int r, int rows) {
        const int x = min(r, rows - 1), t = win_token(p, x), head = kvh * p.group + x - t * p.group;
        const float lse = p.LSE_in[(s.row0 + t) * p.heads + head];
        i = r < rows && s.first + t < s.len ? s.first + t : -1;
        lse2 = r >= rows || lse == -__builtin_inff() ? __builtin_inff() : lse * kLog2e;
    }
};
__device__ __forceinline__ bool weigh_sees(const WinParams& p, int i, int j) { return j <= i && (i - j < p.window || j < p.sinks); }

__device__ __forceinline__ void weigh_store(const WeighParams& w, const WinSeq& s, int b, int kvh, int j, float sum) {
    if (j >= s.len) return;
    float v = sum;
    if (w.in && j < s.first) v = fmaf(w.decay, w.in[(long)b * w.in_b + (long)kvh * w.in_h + j], sum);
    w.out[(long)b * w.out_b + (long)kvh * w.out_h + j] = v;
}

// 16x16x32 products: 32 keys on a wave, straight from memory into operands (lane l: key l % 16, 16 bytes of it), rows 16 at a time.
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads) weigh_kernel(WeighParams w) {
    const WinParams& p = w.p;
    constexpr int KS = D / 32;
    const int lane = threadIdx.x & 63, q = lane >> 4, l16 = lane & 15, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blk = blockIdx.x % w.blocks, bk = blockIdx.x / w.blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, end = min(s.len, (blk + 1) * w.chunk);
    const float cs = p.scale * kLog2e;
    for (int j0 = blk * w.chunk + 32 * wave; j0 < end; j0 += 128) {
        bf16x8 kf[2][KS];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int j = min(j0 + 16 * g + l16, s.len - 1);
            const PageRow r = win_page_row(p, win_page(p, b, j), kvh, j);
            if constexpr (SRC == kCodes) {
                const char* src = static_cast<const char*>(p.K) + r.at;
                const float scale = exp_value(p.K_exp[r.exp]);
#pragma unroll
                for (int x = 0; x < KS / 2; ++x) {
                    const u32x4 v = load_chunk<PAD>(src, 4 * x + q, p.d);
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
                        kf[g][2 * x + half] = __builtin_bit_cast(bf16x8, a);
                    }
                }
            } else {
                const char* src = static_cast<const char*>(p.K) + r.at * 2;
#pragma unroll
                for (int x = 0; x < KS; ++x) kf[g][x] = __builtin_bit_cast(bf16x8, load_chunk<PAD>(src, 4 * x + q, p.d));
            }
        }
        float sum[2] = {0.f, 0.f};
        WeighRows<16> range;
        range.init(p, s, j0, min(j0 + 31, s.len - 1));
        for (int r0 = range.r0; r0 < range.r1; r0 += 16) {
            const int x = min(r0 + l16, rows - 1), t = win_token(p, x), head = kvh * p.group + x - t * p.group;
            const char* row = reinterpret_cast<const char*>(static_cast<const __bf16*>(p.Q) + s.q_base + (long)head * p.q_h + (long)t * p.q_n);
            bf16x8 qf[KS];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
                qf[ks] = __builtin_bit_cast(bf16x8, load_chunk<PAD>(row, SRC == kCodes ? 8 * (ks >> 1) + 2 * q + (ks & 1) : 4 * ks + q, p.d));
            WeighRow at[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) at[i].init(p, s, kvh, r0 + 4 * q + i, rows);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                f32x4 st = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) st = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[ks], kf[g][ks], st, 0, 0, 0);
                const int j = j0 + 16 * g + l16;
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
        if (q < 2) weigh_store(w, s, b, kvh, j0 + 16 * q + l16, v);
    }
}

// 32-bit arithmetic: 32x32x2 products of 32 keys on a wave, rows 32 at a time, both straight from memory.
template <typename T, typename E, int DP>
__global__ void __launch_bounds__(kThreads, 1) weigh_plain_kernel(WeighParams w) {
    const WinParams& p = w.p;
    const int lane = threadIdx.x & 63, h = lane >> 5, l32 = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int blk = blockIdx.x % w.blocks, bk = blockIdx.x / w.blocks, b = bk / p.kv_heads, kvh = bk % p.kv_heads;
    const WinSeq s = win_sequence(p, b);
    const int rows = s.nq * p.group, end = min(s.len, (blk + 1) * w.chunk);
    for (int j0 = blk * w.chunk + 32 * wave; j0 < end; j0 += 128) {
        const int j = j0 + l32, at_j = min(j, s.len - 1);
        const PageRow place = win_page_row(p, win_page(p, b, at_j), kvh, at_j);
        RowOperand<E, DP> key;
        key.init(static_cast<const E*>(p.K) + place.at, p.d, h);
        float cs = p.scale * kLog2e;
        if constexpr (std::is_same_v<E, uint8_t>) cs *= exp_value(p.K_exp[place.exp]);
        float sum = 0.f;
        WeighRows<32> range;
        range.init(p, s, j0, min(j0 + 31, s.len - 1));
        for (int r0 = range.r0; r0 < range.r1; r0 += 32) {
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
        if (h == 0) weigh_store(w, s, b, kvh, j, sum);
    }
}

dim3 grid_of(const WeighParams& w) { return dim3((unsigned)((long)w.blocks * w.p.batch * w.p.kv_heads)); }

template <int D>
hipError_t launch(bool fp8, const WeighParams& w, hipStream_t stream) {
    auto fn = fp8 ? weigh_kernel<D, kCodes, false> : w.p.d < D ? weigh_kernel<D, kPages, true> : weigh_kernel<D, kPages, false>;
    hipLaunchKernelGGL(fn, grid_of(w), dim3(kThreads), 0, stream, w);
    return hipGetLastError();
}
template <typename T, typename E>
hipError_t plain(const WeighParams& w, hipStream_t stream) {
    return with_width(w.p.d, [&](auto width) {
        hipLaunchKernelGGL((weigh_plain_kernel<T, E, decltype(width)::value>), grid_of(w), dim3(kThreads), 0, stream, w);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_weigh(bool fp8, const WeighParams& w, hipStream_t stream) {
    if (fp8 && w.p.d != 64 && w.p.d != 128 && w.p.d != 256) return hipErrorInvalidValue;
    return w.p.d <= 64 ? launch<64>(fp8, w, stream) : w.p.d <= 128 ? launch<128>(fp8, w, stream) : launch<256>(fp8, w, stream);
}
hipError_t launch_weigh_plain(bool is_bf16, bool fp8, const WeighParams& w, hipStream_t stream) {
    if (fp8) return is_bf16 ? plain<__bf16, uint8_t>(w, stream) : plain<float, uint8_t>(w, stream);
    return plain<float, float>(w, stream);
}

}  // namespace attn
