// The paged cache: keys and values of new tokens go into its pages (quantised on the way where the pages hold codes), and come back out.
//
// A quantised row (one token, one head, K or V) is d e4m3 codes and one exponent byte e: a code c stands for c 2^(e - 127), with the
// smallest power of two that brings the row's largest magnitude to 448, the largest value of the format, or less.  A power of
// two costs no precision in a floating-point format, makes scaling exact in both directions (the code is the only rounding,
// to nearest, ties to even) and takes one byte.  A NaN or an infinity is stored as NaN and does not count for the largest magnitude.
//
// Bound by memory: every value is read once and written once.  8 to 32 lanes share a row, 16 bytes of it each.
#include "attn_internal.hpp"
#include "attn_window.hpp"

namespace attn {
namespace {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ f32x8 load8(const __bf16* at, int) {
    return __builtin_convertvector(*reinterpret_cast<const bf16x8*>(at), f32x8);
}
__device__ __forceinline__ f32x8 load8(const float* at, int count) {  // count: values of the row from `at` on
    f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (count >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4u*>(at), b = *reinterpret_cast<const f32x4u*>(at + 4);
        v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < count) v[e] = at[e];
    }
    return v;
}
__device__ __forceinline__ void store8(__bf16* at, int, f32x8 v) {
    *reinterpret_cast<u32x4*>(at) = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* at, int count, f32x8 v) {
    if (count >= 8) {
        *reinterpret_cast<f32x4u*>(at) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        *reinterpret_cast<f32x4u*>(at + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < count) at[e] = v[e];
    }
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Which row a lane works on: row u of the new tokens' rows of a sequence, u = (t * kv_heads + kvh) * 2 + (0: K, 1: V).
struct CacheRow {
    bool inside, in_page;  // a row of this sequence; that has a place in the pages
    int t, kvh, which;
    long at, exp;
};
__device__ __forceinline__ CacheRow cache_row(const WinParams& p, const WinSeq& s, int b, long u) {
    CacheRow r;
    r.which = (int)(u & 1);
    const long x = u >> 1;
    r.t = (int)(x / p.kv_heads);
    r.kvh = (int)(x - (long)r.t * p.kv_heads);
    r.inside = r.t < s.nq;
    r.in_page = false;
    r.at = r.exp = 0;
    const int pos = s.first + r.t;
    if (r.inside && pos >= 0) {
        const int page = p.table[(long)b * p.table_stride + (pos >> p.page_shift)];
        if ((unsigned)page < (unsigned)p.num_pages) {
            const PageRow at = win_page_row(p, page, r.kvh, pos);
            r.at = at.at;
            r.exp = at.exp;
            r.in_page = true;
        }
    }
    return r;
}

template <typename T, bool FP8>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(WinParams p, const void* K, const void* V, long s_n, long s_h, int lanes) {
    const int b = blockIdx.y;
    const WinSeq s = win_sequence(p, b);
    const long u = ((long)blockIdx.x * kThreads + threadIdx.x) / lanes;
    const int c = 8 * (int)(threadIdx.x & (lanes - 1));
    const CacheRow r = cache_row(p, s, b, u);
    const bool mine = r.in_page && c < p.d;
    f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int row0 = p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n;
    if (mine) v = load8(static_cast<const T*>(r.which ? V : K) + (row0 + (long)r.t) * s_n + (long)r.kvh * s_h + c, p.d - c);
    void* pages = const_cast<void*>(r.which ? p.V : p.K);
    if constexpr (FP8) {
        constexpr uint32_t kInf = 0x7f800000u;
        uint32_t top = 0;  // magnitudes order as their bits do
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t a = magnitude(v[e]);
            if (a < kInf) top = a > top ? a : top;
        }
        for (int x = 1; x < lanes; x <<= 1) {
            const uint32_t other = (uint32_t)__shfl_xor((int)top, x, 64);
            top = other > top ? other : top;
        }
        // top = f 2^k with 1 <= f < 2, and 448 = 1.75 2^8
        int e2 = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
        e2 = top == 0 ? 0 : e2 < -126 ? -126 : e2;
        const float scale = __builtin_bit_cast(float, (uint32_t)(127 - e2) << 23);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = magnitude(v[e]) < kInf ? v[e] * scale : __builtin_nanf("");
        }
        if (mine) {
            int lo = 0, hi = 0;
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
            *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(pages) + r.at + c) = u32x2{(uint32_t)lo, (uint32_t)hi};
            if (c == 0) const_cast<uint8_t*>(r.which ? p.V_exp : p.K_exp)[r.exp] = (uint8_t)(e2 + 127);
        }
    } else if (mine) {
        store8(static_cast<T*>(pages) + r.at + c, p.d - c, v);
    }
}

// Rows without a place in the pages (a position in front of the first token, a page that is gone) come back as zeros.
template <typename T, bool FP8>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(WinParams p, void* K, void* V, long s_n, long s_h, int lanes) {
    const int b = blockIdx.y;
    const WinSeq s = win_sequence(p, b);
    const long u = ((long)blockIdx.x * kThreads + threadIdx.x) / lanes;
    const int c = 8 * (int)(threadIdx.x & (lanes - 1));
    const CacheRow r = cache_row(p, s, b, u);
    if (!r.inside || c >= p.d) return;
    f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const void* pages = r.which ? p.V : p.K;
    if (r.in_page) {
        if constexpr (FP8) {
            const u32x2 codes = *reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pages) + r.at + c);
            const float scale = exp_value((r.which ? p.V_exp : p.K_exp)[r.exp]);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[x], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[x], true);
                v[4 * x] = lo[0] * scale;
                v[4 * x + 1] = lo[1] * scale;
                v[4 * x + 2] = hi[0] * scale;
                v[4 * x + 3] = hi[1] * scale;
            }
        } else {
            v = load8(static_cast<const T*>(pages) + r.at + c, p.d - c);
        }
    }
    const int row0 = p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n;
    store8(static_cast<T*>(r.which ? V : K) + (row0 + (long)r.t) * s_n + (long)r.kvh * s_h + c, p.d - c, v);
}

int lanes_of(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }
dim3 grid_of(const WinParams& p) {
    return dim3((unsigned)(((long)p.n * p.kv_heads * 2 * lanes_of(p.d) + kThreads - 1) / kThreads), (unsigned)p.batch);
}

}  // namespace

hipError_t launch_cache_write(bool is_bf16, bool fp8, const WinParams& p, const void* K, const void* V, long s_n, long s_h, hipStream_t stream) {
    auto fn = is_bf16 ? (fp8 ? cache_write_kernel<__bf16, true> : cache_write_kernel<__bf16, false>)
                      : (fp8 ? cache_write_kernel<float, true> : cache_write_kernel<float, false>);
    hipLaunchKernelGGL(fn, grid_of(p), dim3(kThreads), 0, stream, p, K, V, s_n, s_h, lanes_of(p.d));
    return hipGetLastError();
}
hipError_t launch_cache_read(bool is_bf16, bool fp8, const WinParams& p, void* K, void* V, long s_n, long s_h, hipStream_t stream) {
    auto fn = is_bf16 ? (fp8 ? cache_read_kernel<__bf16, true> : cache_read_kernel<__bf16, false>)
                      : (fp8 ? cache_read_kernel<float, true> : cache_read_kernel<float, false>);
    hipLaunchKernelGGL(fn, grid_of(p), dim3(kThreads), 0, stream, p, K, V, s_n, s_h, lanes_of(p.d));
    return hipGetLastError();
}

}  // namespace attn
