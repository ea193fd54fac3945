// Windowed attention on bf16-MFMA, d in {64, 128, 256}: how rows of a tile come from tensors or pages into the swizzled LDS tiles of
// attn_common.hpp.  HIP device code only.
#pragma once
#include "attn_window.hpp"

namespace attn {

enum WinSource { kTensors = 0, kPages = 1, kCodes = 2 };  // bf16 tensors, bf16 pages, quantised pages

// What lane `lane` of copy instruction `inst` (1 KB of a [rows x D] tile) fetches: its row, and where in the row.  PAD: the rows have d < D
// columns (a multiple of 8); the others are filled with zeros, which change no product.
static __device__ const u32x4 win_zeros = {0, 0, 0, 0};
template <int D>
struct CopyLane {
    static constexpr int kRows = 512 / D;  // rows per instruction
    __device__ __forceinline__ static int row_of(int inst, int lane) { return inst * kRows + lane / (D / 8); }
    // from: the first byte of row `row` of the tile
    template <bool PAD>
    __device__ __forceinline__ static const char* at(const char* from, int row, int lane, int d) {
        const int c = (lane % (D / 8)) ^ swz<D>(row);
        if (PAD && 8 * c >= d) return reinterpret_cast<const char*>(&win_zeros);
        return from + 16 * c;
    }
};
// 16 bytes from column 8 c on of a row
template <bool PAD>
__device__ __forceinline__ u32x4 load_chunk(const char* row, int c, int d) {
    return *reinterpret_cast<const u32x4*>(PAD && 8 * c >= d ? reinterpret_cast<const char*>(&win_zeros) : row + 16 * c);
}

// 16 bytes per lane from `src` to LDS at dst + 16 lane.  Inline assembly as in load_tile_direct: the wait is the caller's.
__device__ __forceinline__ void copy_row(const char* src, unsigned dst) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(dst), "v"(src) : "memory", "m0");
}
__device__ __forceinline__ unsigned lds_address(const void* at) {
    return __builtin_amdgcn_readfirstlane((unsigned)(size_t)(ATTN_LDS const char*)at);
}

// The pages of up to 64 consecutive entries of a sequence's table, one per lane: a wave asks for the page of a key by a shuffle, and reads the
// table once per 64 entries (1024 keys in pages of 16), not once per tile: the wait for it drains the copies in flight.
struct PageWindow {
    int ids, first;
    __device__ __forceinline__ void init() { first = -128; }
    // keys j0 .. j1 of a tile, both of whose entries exist
    __device__ __forceinline__ void cover(const WinParams& p, int b, int j0, int j1, int end, int lane) {
        const int e0 = j0 >> p.page_shift, e1 = j1 >> p.page_shift;
        if (e0 >= first && e1 < first + 64) return;
        first = e0;
        const int e = min(first + lane, (end - 1) >> p.page_shift);
        ids = (int)min((unsigned)p.table[(long)b * p.table_stride + e], (unsigned)(p.num_pages - 1));
    }
    __device__ __forceinline__ int page(const WinParams& p, int j) const { return __shfl(ids, (j >> p.page_shift) - first, 64); }
};

// 16 codes of a row as two chunks of 8 bf16, exactly: 2^(e - 127) is a power of two and a code has 4 bits.
struct CodeChunk {
    u32x4 codes;
    float scale;
    __device__ __forceinline__ void to_lds(char* lo, char* hi) const {
        u32x4 v[2];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[x], scale, false);
            const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[x], scale, true);
            v[x >> 1][2 * (x & 1)] = __builtin_bit_cast(uint32_t, a);
            v[x >> 1][2 * (x & 1) + 1] = __builtin_bit_cast(uint32_t, b);
        }
        *reinterpret_cast<u32x4*>(lo) = v[0];
        *reinterpret_cast<u32x4*>(hi) = v[1];
    }
};

// Which keys a lane's query sees, relative to a tile: key j0 + c + 4 h is seen iff c <= hi and (c >= lo or c < sink).
struct LaneBounds {
    int hi, lo;
    __device__ __forceinline__ void init(const WinParams& p, int i, int len) {
        hi = i < len ? i : -1;
        lo = i - p.window + 1;
    }
};

}  // namespace attn
