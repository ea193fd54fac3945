// Windowed attention over tensors or over a paged cache: the arguments of its kernels and what they share.
//
// A query at position i of its sequence sees key j iff j <= i and (no window, or i - j < window, or j < sinks).  In tensors
// [batch, heads, n, d] token t has position t and a sequence may be shorter than n; in a paged cache the new tokens of a
// sequence are its last ones.  The heads of a group share keys and values: the queries of a (sequence, key head) are taken
// as rows r = t * group + g of one matrix, so that a tile of keys is read once for all of them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_common.hpp"

namespace attn {

struct WinParams {
    const void *Q, *K, *V, *dO, *O_in;  // K, V: tensors or pages
    void *O, *dQ, *dK, *dV;
    const float* LSE_in;
    float *LSE, *delta;
    long q_b, q_h, q_n;     // Q, O, dO, dQ; paged: q_b unused
    long k_b, k_h, k_n;     // K, V, dK, dV; paged: k_b is the stride of pages
    const uint8_t *K_exp, *V_exp;  // [page][kv head][token of the page]; nullptr: pages hold values
    const int32_t *table, *lens, *q_ptr;  // table == nullptr: tensors
    long table_stride;
    unsigned group_inv;     // ceil(2^32 / group) for group > 1: see win_token
    int batch, heads, kv_heads, group, n, d;  // n: tokens (tensors), largest number of new tokens of a sequence (paged)
    int page_shift, num_pages, total_q, max_len;
    float scale;
    int window, sinks;  // window > 0; no window: larger than any distance, and no sinks
    int row_blocks, blocks;  // paged: row blocks of the longest sequence, and at most of all of them
    // forward: work of a row block shared out over `splits` workgroups of `chunk` tiles each; their sums meet in win_join_kernel
    int splits, chunk;
    float *part_o, *part_ml;  // [row][split][d], [row][split][2], row = token row * heads + head
    // backward: the first `sink_tiles` key tiles are each worked on by `parts` workgroups, the others by `rest_parts`, each of which takes a
    // share of the tokens; where there are several, their sums meet in win_keys_kernel
    int sink_tiles, parts, rest_parts;
    int slots;  // workgroups of a (sequence, key head) whose sums are parts
    float* part_kv;  // [batch * kv_heads][slot][dK, dV][keys of a tile][d]
};

// r / group for 0 <= r < 2^31: the product with ceil(2^32 / group) is the quotient or one more (a division takes some 25 instructions, and the rows of a
// block are placed one by one when they are read and written).
__device__ __forceinline__ int win_token(const WinParams& p, int r) {
    if (p.group == 1) return r;
    const unsigned q = __umulhi((unsigned)r, p.group_inv);
    return (int)(q - (q * (unsigned)p.group > (unsigned)r ? 1u : 0u));
}

// What a workgroup knows of its sequence.  Everything is uniform; lengths from device memory are brought into the range that the
// buffers allow, so that no value in them leads outside.
struct WinSeq {
    int len, nq, first;  // keys 0 .. len - 1; queries t = 0 .. nq - 1 at positions first + t
    long q_base, lse_base, lse_h, lse_t;
};
__device__ __forceinline__ WinSeq win_sequence(const WinParams& p, int b) {
    WinSeq s;
    if (p.table) {
        const int row0 = p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n;
        const int rows = p.q_ptr ? min(max(p.q_ptr[b + 1] - row0, 0), p.total_q - row0) : p.n;
        s.len = min(max(p.lens[b], 0), p.max_len);
        s.first = s.len - rows;
        s.nq = min(rows, p.n);
        s.q_base = (long)row0 * p.q_n;
        s.lse_base = (long)row0 * p.heads;
        s.lse_h = 1;
        s.lse_t = p.heads;
    } else {
        s.len = p.lens ? min(max(p.lens[b], 0), p.n) : p.n;
        s.first = 0;
        s.nq = p.n;
        s.q_base = (long)b * p.q_b;
        s.lse_base = (long)b * p.heads * p.n;
        s.lse_h = p.n;
        s.lse_t = 1;
    }
    return s;
}

// Row block `idx` of all sequences of a paged call, counting only those that have rows: the host knows no more than their number's bound, and a workgroup
// for every block that the longest sequence could have costs a batch of mixed lengths more than its work (16 sequences of 1 to 256 new tokens:
// 744 of 1024 without rows).  A wave adds up the sequences' blocks 64 at a time.
struct WinBlock {
    int b, blk;
    bool any;
    __device__ __forceinline__ void init(const WinParams& p, int idx, int rows_per_block, int lane) {
        any = true;
        if (!p.q_ptr || p.row_blocks == 1) {
            b = idx / p.row_blocks;
            blk = idx - b * p.row_blocks;
            return;
        }
        for (int base = 0; base < p.batch; base += 64) {
            const int mine = base + lane;
            int own = 0;
            if (mine < p.batch) {
                const int row0 = min(max(p.q_ptr[mine], 0), p.total_q), rows = min(max(p.q_ptr[mine + 1] - row0, 0), p.total_q - row0);
                own = (min(rows, p.n) * p.group + rows_per_block - 1) / rows_per_block;
            }
            int upto = own;
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) {
                const int before = __shfl_up(upto, x, 64);
                upto += lane >= x ? before : 0;
            }
            const int all = __builtin_amdgcn_readlane(upto, 63);
            if (idx < all) {
                const int who = __builtin_ctzl(__builtin_amdgcn_ballot_w64(upto > idx));
                b = base + who;
                blk = idx - __builtin_amdgcn_readlane(upto - own, who);
                return;
            }
            idx -= all;
        }
        any = false;
        b = blk = 0;
    }
};
// The sequence that row `row` of a paged call belongs to, or -1.
__device__ __forceinline__ int win_sequence_of(const WinParams& p, int row, int lane) {
    if (!p.q_ptr) return row < p.batch * p.n ? row / p.n : -1;
    for (int base = 0; base < p.batch; base += 64) {
        const int mine = base + lane;
        const bool hit = mine < p.batch && row >= p.q_ptr[mine] && row < p.q_ptr[mine + 1];
        const unsigned long who = __builtin_amdgcn_ballot_w64(hit);
        if (who) return base + __builtin_ctzl(who);
    }
    return -1;
}

// The key tiles of BC keys that queries at positions i_min .. i_max see some key of: those of the sinks, then those of the windows.
template <int BC>
struct WinTiles {
    int lo, end;    // keys lo .. end - 1, and 0 .. sinks - 1, are seen by some query
    int ns, first;  // sink tiles; first of the other tiles
    int count;
    __device__ __forceinline__ void init(const WinParams& p, int len, int i_min, int i_max) {
        end = min(i_max, len - 1) + 1;
        lo = max(0, i_min - p.window + 1);
        ns = (min(p.sinks, end) + BC - 1) / BC;
        first = max(lo / BC, ns);
        count = ns + max(0, (end + BC - 1) / BC - first);
        if (end <= 0 || i_min >= len) count = 0;
    }
    __device__ __forceinline__ int start(int it) const { return (it < ns ? it : it - ns + first) * BC; }
    // The row that is read for key j of a tile: rows that no query of the block sees (behind the end, before the windows, where pages
    // may be gone) are replaced by one of the same tile that some query sees.
    __device__ __forceinline__ int row(const WinParams& p, int j) const {
        j = min(j, end - 1);
        return j < lo && j >= p.sinks ? ((j & -BC) < p.sinks ? p.sinks - 1 : lo) : j;
    }
    __device__ __forceinline__ bool whole(const WinParams& p, int j0) const {  // every row of the tile is its own
        return j0 + BC <= end && (j0 >= lo || j0 + BC <= p.sinks);
    }
};

// Element offset of the first value of a key's row in pages, and of its exponent byte.  A page number outside the cache (of a token
// that a caller declared visible and has no page for) is brought inside it: the result is meaningless, the access is not.
struct PageRow {
    long at;
    long exp;
};
__device__ __forceinline__ int win_page(const WinParams& p, int b, int j) {
    const int page = p.table[(long)b * p.table_stride + (j >> p.page_shift)];
    return (int)min((unsigned)page, (unsigned)(p.num_pages - 1));
}
__device__ __forceinline__ PageRow win_page_row(const WinParams& p, int page, int kvh, int j) {
    const int slot = j & ((1 << p.page_shift) - 1);
    return {(long)page * p.k_b + (long)kvh * p.k_h + (long)slot * p.k_n,
            (((long)page * p.kv_heads + kvh) << p.page_shift) + slot};
}

// 2^(e - 127) for an exponent byte e of 1 .. 254 (0 and 255, which no row is written with, give 0 and infinity).
__device__ __forceinline__ float exp_value(uint8_t e) { return __builtin_bit_cast(float, (uint32_t)e << 23); }

// What a key owner of the backward works on: keys j0 .. and tokens i0 .. i1 - 1 (which see some of them); slot < 0: all of those, else one part.
struct WinKeys {
    int j0, i0, i1, slot;
    __device__ __forceinline__ void init(const WinParams& p, int blk, int tile, int len) {
        const int shared = p.sink_tiles * p.parts, r = blk - shared;
        const int parts = r < 0 ? p.parts : p.rest_parts, part = (r < 0 ? blk : r) % parts;
        j0 = tile * (r < 0 ? blk / parts : p.sink_tiles + r / parts);
        slot = parts > 1 ? blk : -1;
        i1 = j0 < p.sinks ? len : (int)min((long)len, (long)j0 + tile - 1 + p.window);
        i0 = j0;
        if (j0 >= len) {
            i1 = i0;
        } else if (parts > 1) {
            const int share = ((i1 - j0 + parts - 1) / parts + tile - 1) / tile * tile;
            i0 = min(i1, j0 + part * share);
            i1 = min(i1, i0 + share);
        }
    }
};

// ------------------------------------------------------------------------------------------------------------- host
// is_bf16: the type of Q, O and of tensors, and of pages that are not quantised (fp8).  The arguments have been checked.
hipError_t launch_win_plain_fwd(bool is_bf16, bool fp8, const WinParams& p, hipStream_t stream);
// bf16; quantised pages: d in {64, 128, 256}; rows of a workgroup: 16, 32 (pages), 64, 128
hipError_t launch_win_fwd(bool fp8, int rows, const WinParams& p, hipStream_t stream);
hipError_t launch_win_bwd(int rows, const WinParams& p, hipStream_t stream);                                // rows: 64, 128; forms delta itself
hipError_t launch_win_plain_bwd(const WinParams& p, hipStream_t stream);  // fp32
hipError_t launch_win_join(bool is_bf16, const WinParams& p, hipStream_t stream);
hipError_t launch_win_keys(bool is_bf16, int tile, const WinParams& p, hipStream_t stream);
hipError_t launch_win_rows(const WinParams& p, hipStream_t stream);       // fp32: delta
hipError_t launch_cache_write(bool is_bf16, bool fp8, const WinParams& p, const void* K, const void* V, long s_n, long s_h, hipStream_t stream);
hipError_t launch_cache_read(bool is_bf16, bool fp8, const WinParams& p, void* K, void* V, long s_n, long s_h, hipStream_t stream);

}  // namespace attn
