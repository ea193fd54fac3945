// The paged cache: keys and values of new tokens go into its pages (quantised on the way where the pages hold codes), and come back out.
//
// A quantised row (one token, one head, K or V) is d e4m3 codes and one exponent byte e: a code c stands for c 2^(e - 127), with the
// smallest power of two that brings the row's largest magnitude to 448, the largest value of the format, or less.  A power of
// two costs no precision in a floating-point format, makes scaling exact in both directions (the code is the only rounding,
// to nearest, ties to even) and takes one byte.  A NaN or an infinity is stored as NaN and does not count for the largest magnitude.
//
// Bound by memory: every value is read once and written once.  8 to 32 lanes share a row, 16 bytes of it each.
#include "attn_internal.hpp"
#include "attn_win_rules.hpp"
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

// The rows of a token and head that a lane works on, K and V alike: u = t * kv_heads + kvh counts those of a sequence.
struct CacheRow {
    bool inside, in_page;  // a row of this sequence; that has a place in the pages
    long given, at, exp;   // its offset among the new tokens' rows, in the pages, among the exponents
};
__device__ __forceinline__ CacheRow cache_row(const WinParams& p, const WinSeq& s, int b, int row0, long u, long s_n, long s_h) {
    CacheRow r;
    const int t = (int)(u / p.kv_heads), kvh = (int)(u - (long)t * p.kv_heads), pos = s.first + t;
    r.inside = t < s.nq;
    r.in_page = false;
    r.given = (row0 + (long)t) * s_n + (long)kvh * s_h;
    r.at = r.exp = 0;
    if (r.inside && pos >= 0) {
        const int page = p.table[(long)b * p.table_stride + (pos >> p.page_shift)];
        if ((unsigned)page < (unsigned)p.num_pages) {
            const PageRow at = win_page_row(p, page, kvh, pos);
            r.at = at.at;
            r.exp = at.exp;
            r.in_page = true;
        }
    }
    return r;
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// Codes and exponent of a row that `lanes` lanes share.
__device__ __forceinline__ u32x2 quantise(f32x8 v, int lanes, int& e2) {
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
    e2 = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    e2 = top == 0 ? 0 : e2 < -126 ? -126 : e2;
    const float scale = __builtin_bit_cast(float, (uint32_t)(127 - e2) << 23);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = magnitude(v[e]) < kInf ? v[e] * scale : __builtin_nanf("");
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], hi, true);
    return u32x2{(uint32_t)lo, (uint32_t)hi};
}
__device__ __forceinline__ f32x8 dequantise(u32x2 codes, float scale) {
    f32x8 v;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[x], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[x], true);
        v[4 * x] = lo[0] * scale;
        v[4 * x + 1] = lo[1] * scale;
        v[4 * x + 2] = hi[0] * scale;
        v[4 * x + 3] = hi[1] * scale;
    }
    return v;
}

__device__ __forceinline__ int first_row(const WinParams& p, int b) { return p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n; }

template <typename T, bool FP8, int kRowsPerThread>
__global__ void __launch_bounds__(kThreads) cache_write_kernel(WinParams p, const void* K, const void* V, long s_n, long s_h, int lanes) {
    const int b = blockIdx.y, row0 = first_row(p, b), per = kThreads / lanes;
    const WinSeq s = win_sequence(p, b);
    const long u0 = (long)blockIdx.x * (per * kRowsPerThread);
    if (u0 >= (long)s.nq * p.kv_heads) return;
    const int c = 8 * (int)(threadIdx.x & (lanes - 1));
    CacheRow r[kRowsPerThread];
    f32x8 k[kRowsPerThread], v[kRowsPerThread];
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) r[x] = cache_row(p, s, b, row0, u0 + x * per + threadIdx.x / lanes, s_n, s_h);
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) {
        k[x] = v[x] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (r[x].in_page && c < p.d) {
            k[x] = load8(static_cast<const T*>(K) + r[x].given + c, p.d - c);
            v[x] = load8(static_cast<const T*>(V) + r[x].given + c, p.d - c);
        }
    }
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) {
        const bool mine = r[x].in_page && c < p.d;
        if constexpr (FP8) {
            int ke, ve;
            const u32x2 kc = quantise(k[x], lanes, ke), vc = quantise(v[x], lanes, ve);
            if (mine) {
                *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(const_cast<void*>(p.K)) + r[x].at + c) = kc;
                *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(const_cast<void*>(p.V)) + r[x].at + c) = vc;
                if (c == 0) {
                    const_cast<uint8_t*>(p.K_exp)[r[x].exp] = (uint8_t)(ke + 127);
                    const_cast<uint8_t*>(p.V_exp)[r[x].exp] = (uint8_t)(ve + 127);
                }
            }
        } else if (mine) {
            store8(static_cast<T*>(const_cast<void*>(p.K)) + r[x].at + c, p.d - c, k[x]);
            store8(static_cast<T*>(const_cast<void*>(p.V)) + r[x].at + c, p.d - c, v[x]);
        }
    }
}

// Rows without a place in the pages (a position in front of the first token, a page that is gone) come back as zeros.
template <typename T, bool FP8, int kRowsPerThread>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(WinParams p, void* K, void* V, long s_n, long s_h, int lanes) {
    const int b = blockIdx.y, row0 = first_row(p, b), per = kThreads / lanes;
    const WinSeq s = win_sequence(p, b);
    const long u0 = (long)blockIdx.x * (per * kRowsPerThread);
    const int c = 8 * (int)(threadIdx.x & (lanes - 1));
    if (u0 >= (long)s.nq * p.kv_heads || c >= p.d) return;
    CacheRow r[kRowsPerThread];
    f32x8 k[kRowsPerThread], v[kRowsPerThread];
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) r[x] = cache_row(p, s, b, row0, u0 + x * per + threadIdx.x / lanes, s_n, s_h);
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) {
        k[x] = v[x] = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (!r[x].in_page) continue;
        if constexpr (FP8) {
            k[x] = dequantise(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p.K) + r[x].at + c), exp_value(p.K_exp[r[x].exp]));
            v[x] = dequantise(*reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(p.V) + r[x].at + c), exp_value(p.V_exp[r[x].exp]));
        } else {
            k[x] = load8(static_cast<const T*>(p.K) + r[x].at + c, p.d - c);
            v[x] = load8(static_cast<const T*>(p.V) + r[x].at + c, p.d - c);
        }
    }
#pragma unroll
    for (int x = 0; x < kRowsPerThread; ++x) {
        if (!r[x].inside) continue;
        store8(static_cast<T*>(K) + r[x].given + c, p.d - c, k[x]);
        store8(static_cast<T*>(V) + r[x].given + c, p.d - c, v[x]);
    }
}

template <int ROWS>
dim3 grid_of(const WinParams& p) {
    const long rows = kThreads / cache_lanes(p.d) * ROWS;
    return dim3((unsigned)(((long)p.n * p.kv_heads + rows - 1) / rows), (unsigned)p.batch);
}

}  // namespace

hipError_t launch_cache_write(bool is_bf16, bool fp8, const WinParams& p, const void* K, const void* V, long s_n, long s_h, hipStream_t stream) {
    auto launch = [&](auto rows) {
        constexpr int R = decltype(rows)::value;
        auto fn = is_bf16 ? (fp8 ? cache_write_kernel<__bf16, true, R> : cache_write_kernel<__bf16, false, R>)
                          : (fp8 ? cache_write_kernel<float, true, R> : cache_write_kernel<float, false, R>);
        hipLaunchKernelGGL(fn, grid_of<R>(p), dim3(kThreads), 0, stream, p, K, V, s_n, s_h, cache_lanes(p.d));
    };
    if (cache_rows_per_thread(p.kv_heads, p.total_q, p.d) > 1) launch(std::integral_constant<int, kManyRows>{});
    else launch(std::integral_constant<int, 1>{});
    return hipGetLastError();
}
hipError_t launch_cache_read(bool is_bf16, bool fp8, const WinParams& p, void* K, void* V, long s_n, long s_h, hipStream_t stream) {
    auto launch = [&](auto rows) {
        constexpr int R = decltype(rows)::value;
        auto fn = is_bf16 ? (fp8 ? cache_read_kernel<__bf16, true, R> : cache_read_kernel<__bf16, false, R>)
                          : (fp8 ? cache_read_kernel<float, true, R> : cache_read_kernel<float, false, R>);
        hipLaunchKernelGGL(fn, grid_of<R>(p), dim3(kThreads), 0, stream, p, K, V, s_n, s_h, cache_lanes(p.d));
    };
    if (cache_rows_per_thread(p.kv_heads, p.total_q, p.d) > 1) launch(std::integral_constant<int, kManyRows>{});
    else launch(std::integral_constant<int, 1>{});
    return hipGetLastError();
}

}  // namespace attn
