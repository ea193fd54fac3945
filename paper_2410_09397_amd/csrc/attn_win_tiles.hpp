// Windowed attention on bf16-MFMA, d in {64, 128, 256}: how rows of a tile come from tensors or pages into the swizzled LDS tiles of
// attn_common.hpp.  HIP device code only.
#pragma once
#include "attn_win_rules.hpp"
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

// Behind the last product of a sum whose next reader is on the other side of a branch.  A product of 8 passes is in its registers 11 states later; the
// compiler puts the states in between within a block, but on the way around a branch that is taken it has been seen to leave out all but three of them: at d = 256
// the last register, read first, then lacked the last products (one key of 32 with a wrong score).
__device__ __forceinline__ void settle_products(f32x16& sum) { asm volatile("s_nop 10" : "+v"(sum)); }

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

// The tiles of BC keys that a block of rows goes through, and which of a tile's keys the query of a lane sees.
//   init        t: the lane's token; t_lo .. t_hi: those of its wave; b_lo .. b_hi: those of its workgroup
//   all, none   every row of the wave sees all of the keys j0 .. j0 + last of tile `it`, or none of them
//   keys        seen(T, c): the lane's query sees key j0 + 32 T + shift + c (of NT accumulators of 32 keys)
template <int BC, bool TREE>
struct Sight {
    WinTiles<BC> tiles;
    LaneBounds see;
    int t_lo, t_hi, len;
    __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s, int t, int wave_lo, int wave_hi, int b_lo, int b_hi) {
        see.init(p, s.first + t, s.len);
        t_lo = s.first + wave_lo;
        t_hi = s.first + wave_hi;
        len = s.len;
        tiles.init(p, s.len, s.first + b_lo, s.first + b_hi);
    }
    __device__ __forceinline__ bool all(const WinParams& p, int, int j0, int last) const {
        return j0 + last <= t_lo && t_hi < len && (t_hi - j0 < p.window || j0 + last < p.sinks);
    }
    __device__ __forceinline__ bool none(const WinParams& p, int, int j0, int last) const {
        return j0 > t_hi || (j0 + last < t_lo - p.window + 1 && j0 >= p.sinks);
    }
    struct Keys {
        int hi, lo, sink;
        __device__ __forceinline__ bool operator()(int T, int c) const {
            c += 32 * T;
            return c <= hi && (c >= lo || c < sink);
        }
    };
    template <int NT>
    __device__ __forceinline__ Keys keys(const WinParams& p, int, int j0, int shift) const {
        const int j = j0 + shift;
        return {see.hi - j, see.lo - j, p.sinks - j};
    }
};

// A tree of drafted tokens behind a context: tiles of the context first (those of the sinks, then those of the windows), then tiles of the drafted
// tokens, which start with the first of them, so that a tile's keys are all told by position or all by mask.
template <int BC>
struct Sight<BC, true> {
    struct Tiles {
        int context, lo, end;  // slots 0 .. context - 1 and context .. end - 1; of the context lo .. and 0 .. sinks - 1 are seen by some query
        int ns, first, of_context, count;
        __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s) {
            context = max(0, s.first);
            end = max(context, min(s.len, s.first + s.nq));
            lo = max(0, context - p.window);  // (of a query that sees no drafted token)
            ns = (min(p.sinks, context) + BC - 1) / BC;
            first = max(lo / BC, ns);
            of_context = ns + max(0, (context + BC - 1) / BC - first);
            count = of_context + (end - context + BC - 1) / BC;
        }
        __device__ __forceinline__ int start(int it) const {
            return it < of_context ? (it < ns ? it : it - ns + first) * BC : context + (it - of_context) * BC;
        }
        __device__ __forceinline__ int row(const WinParams& p, int j) const {  // (as WinTiles)
            j = min(j, end - 1);
            return j < lo && j >= p.sinks ? ((j & -BC) < p.sinks ? p.sinks - 1 : lo) : j;
        }
        __device__ __forceinline__ bool whole(const WinParams& p, int j0) const { return j0 + BC <= end && (j0 >= lo || j0 + BC <= p.sinks); }
    } tiles;
    int row, lo;  // of the lane's query: its row of the mask, and under a window the first key of the context that is in it
    int first, nq;
    // x, in a way that what is made of it is made where it stands: kept over the loop, it costs registers that the kernels of single tokens do not have
    static __device__ __forceinline__ int here(int x) {
        asm volatile("" : "+v"(x));
        return x;
    }
    static __device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }
    // bits u .. u + 31 of the mask; tokens in front of slot 0 and behind the last one are none
    __device__ __forceinline__ uint32_t drafted(const WinParams& p, int u) const {
        const int w = u >> 5, words = (p.n + 31) >> 5;
        const uint32_t* mask = p.tree + (long)here(row) * p.tree_stride;
        const uint32_t a = w < words ? mask[w] : 0u, b = (u & 31) && w + 1 < words ? mask[w + 1] : 0u;
        return (uint32_t)((((uint64_t)b << 32) | a) >> (u & 31)) & below(nq - u) & ~below(-first - u);
    }
    __device__ __forceinline__ void init(const WinParams& p, const WinSeq& s, int t, int, int, int, int) {
        tiles.init(p, s);
        first = s.first;
        nq = s.nq;
        row = (int)s.row0 + t;
        int seen = 0;  // drafted tokens
        if (p.window < kNoWindow) {
            for (int u = 0; u < nq; u += 32) seen += __popc(drafted(p, u));
        }
        lo = tiles.context + seen - p.window;  // the query is at position context + seen - 1
    }
    __device__ __forceinline__ bool all(const WinParams& p, int it, int j0, int last) const {
        return it < tiles.of_context && j0 + last < tiles.context && (tiles.context + nq - 1 - j0 < p.window || j0 + last < p.sinks);
    }
    __device__ __forceinline__ bool none(const WinParams&, int it, int j0, int) const { return j0 >= (it < tiles.of_context ? tiles.context : tiles.end); }
    // keys j .. j + 31 of a tile
    __device__ __forceinline__ uint32_t bits(const WinParams& p, int it, int j) const {
        if (it < tiles.of_context) return below(tiles.context - j) & (~below(lo - j) | below(p.sinks - j));
        uint32_t v = drafted(p, j - first);
        if (p.window < kNoWindow) {  // the r-th drafted token that the query sees is at position context + r
            const int seen = here(lo) + p.window - tiles.context;
            int r = 0;
            for (int u = 0; u < j - first; u += 32) r += __popc(drafted(p, u) & below(j - first - u));
            uint32_t in = 0;
            for (uint32_t left = v; left; left &= left - 1, ++r)
                if (seen - 1 - r < p.window || tiles.context + r < p.sinks) in |= left & -left;
            v = in;
        }
        return v;
    }
    template <int NT>
    struct Keys {
        uint32_t v[NT];
        __device__ __forceinline__ bool operator()(int T, int c) const { return (v[T] >> c) & 1u; }
    };
    template <int NT>
    __device__ __forceinline__ Keys<NT> keys(const WinParams& p, int it, int j0, int shift) const {
        Keys<NT> k;
#pragma unroll
        for (int T = 0; T < NT; ++T) k.v[T] = bits(p, it, j0 + 32 * T) >> shift;
        return k;
    }
};

// How a call on trees is shared out.  An item is a row block of a sequence and a part of its tiles; the items of a key head are counted through the sequences, in
// a sequence part by part (so that the row blocks that read the same keys run together), and are as many workgroups.  The sequences' lengths differ
// more than anything else in such a call, and the host does not know them: a part is p.least tiles, or as many as a workgroup
// gets if all tiles are shared out over p.places of them (so that these and one for each row block are enough).  A wave looks at 64 sequences at a time.
template <int BR, int BC>
struct TreeItems {
    int chunk;
    struct Sequence {
        int blocks, tiles;
    };
    static __device__ __forceinline__ Sequence sequence(const WinParams& p, int b) {
        if (b >= p.batch) return {0, 0};
        const WinSeq s = win_sequence(p, b);
        typename Sight<BC, true>::Tiles tiles;
        tiles.init(p, s);
        return {(s.nq * p.group + BR - 1) / BR, tiles.count};
    }
    __device__ __forceinline__ int parts(int tiles) const { return max(1, (int)(((long)tiles + chunk - 1) / chunk)); }
    __device__ __forceinline__ void init(const WinParams& p, int lane) {
        chunk = 0x7fffffff;
        if (p.places == 0) return;  // no work is shared out
        unsigned long sum = 0;
        for (int base = 0; base < p.batch; base += 64) {
            const Sequence s = sequence(p, base + lane);
            unsigned long own = (unsigned long)s.blocks * (unsigned)s.tiles;
            for (int x = 1; x < min(64, p.batch - base); x <<= 1) own += __shfl_xor(own, x, 64);
            sum += (unsigned long)(unsigned)__builtin_amdgcn_readlane((int)(own >> 32), 0) << 32 | (unsigned)__builtin_amdgcn_readlane((int)own, 0);
        }
        chunk = max(p.least, (int)fminf(ceilf((float)sum / (float)p.places), 1e9f));
    }
    // the sequence that item idx belongs to (-1: there is none), the number of its first item, its row blocks and parts
    __device__ __forceinline__ int find(const WinParams& p, int idx, int lane, int& start, int& blocks, int& of_parts) const {
        start = 0;
        of_parts = 1;
        if (p.places == 0 && (!p.q_ptr || p.row_blocks == 1)) {  // (every sequence has as many workgroups: batches of thousands are not searched)
            blocks = p.row_blocks;
            start = idx / blocks * blocks;
            return idx < p.batch * blocks ? idx / blocks : -1;
        }
        for (int base = 0; base < p.batch; base += 64) {
            const Sequence s = sequence(p, base + lane);
            const int own = s.blocks * parts(s.tiles);
            int upto = own;
            for (int x = 1; x < min(64, p.batch - base); x <<= 1) {
                const int before = __shfl_up(upto, x, 64);
                upto += lane >= x ? before : 0;
            }
            const unsigned long who = __builtin_amdgcn_ballot_w64(base + lane < p.batch && start + upto > idx);
            if (who) {
                const int first = __builtin_ctzl(who);
                blocks = __builtin_amdgcn_readlane(s.blocks, first);
                of_parts = __builtin_amdgcn_readlane(parts(s.tiles), first);
                start += __builtin_amdgcn_readlane(upto - own, first);
                return (unsigned)(idx - start) < (unsigned)__builtin_amdgcn_readlane(own, first) ? base + first : -1;  // (no item: the numbers have passed 32 bits, by rows of several sequences)
            }
            start += __builtin_amdgcn_readlane(upto, min(64, p.batch - base) - 1);
        }
        return -1;
    }
    // Where all items are on the chip at once, two to a CU, the later half of them with the earlier one: those with most tiles come first, and of the later half those with fewest, so that
    // long ones share a CU with short ones.  The sequence of the idx-th in this order (-1: there is none), its row blocks and parts, which item of the sequence it is, and the number of
    // the sequence's first item in the order that the sums have.  Up to 64 sequences.
    __device__ __forceinline__ int find_folded(const WinParams& p, int idx, int lane, int& start, int& blocks, int& of_parts, int& within) const {
        const Sequence s = sequence(p, lane);
        const int of = parts(s.tiles), own = s.blocks * of, size = (s.tiles + of - 1) / of;
        TreeFold at;
        for (int x = 0; x < p.batch; ++x) at.count(lane, size, x, __builtin_amdgcn_readlane(own, x), __builtin_amdgcn_readlane(size, x));
        if (idx >= at.all || at.all > p.blocks + p.places + 1) return -1;  // (more items than the launch has: as in find_block)
        idx = TreeFold::place(idx, at.all, p.fold);
        const unsigned long who = __builtin_amdgcn_ballot_w64(at.has(idx, own));
        if (!who) return -1;
        const int b = __builtin_ctzl(who);
        blocks = __builtin_amdgcn_readlane(s.blocks, b);
        of_parts = __builtin_amdgcn_readlane(of, b);
        start = __builtin_amdgcn_readlane(at.before, b);
        within = idx - __builtin_amdgcn_readlane(at.first, b);
        return b;
    }
    // row block idx of all sequences: its sequence (-1: there is none), that one's first item, row blocks and parts, and which of them it is
    __device__ __forceinline__ int find_block(const WinParams& p, int idx, int lane, int& start, int& blocks, int& of_parts, int& blk) const {
        start = 0;
        for (int base = 0; base < p.batch; base += 64) {
            const Sequence s = sequence(p, base + lane);
            const int own = s.blocks * parts(s.tiles);
            int upto = own, rows = s.blocks;
            for (int x = 1; x < min(64, p.batch - base); x <<= 1) {
                const int before = __shfl_up(upto, x, 64), rows_before = __shfl_up(rows, x, 64);
                upto += lane >= x ? before : 0;
                rows += lane >= x ? rows_before : 0;
            }
            const unsigned long who = __builtin_amdgcn_ballot_w64(base + lane < p.batch && rows > idx);
            if (who) {
                const int first = __builtin_ctzl(who);
                start += __builtin_amdgcn_readlane(upto - own, first);
                blocks = __builtin_amdgcn_readlane(s.blocks, first);
                of_parts = __builtin_amdgcn_readlane(parts(s.tiles), first);
                blk = idx - __builtin_amdgcn_readlane(rows - s.blocks, first);
                // (all of its parts are among the launch's: not so only where q_ptr gives rows to several sequences)
                const long last_part = (long)start + blk + (long)(of_parts - 1) * blocks;
                return start >= 0 && (unsigned)blk < (unsigned)blocks && last_part <= (long)p.blocks + p.places ? base + first : -1;
            }
            const int last = min(64, p.batch - base) - 1;
            start += __builtin_amdgcn_readlane(upto, last);
            idx -= __builtin_amdgcn_readlane(rows, last);
        }
        return -1;
    }
};

// The work of a workgroup: a row block of a sequence and its part of the tiles.
template <int BR, int BC, bool TREE>
struct Share {
    int b, blk;
    bool any;
    __device__ __forceinline__ void init(const WinParams& p, int idx, int lane) {
        WinBlock at;
        at.init(p, idx, BR, lane);
        b = at.b;
        blk = at.blk;
        any = at.any;
    }
    __device__ __forceinline__ int first(const WinParams& p, int) const { return blockIdx.y * p.chunk; }
    __device__ __forceinline__ int last(const WinParams& p, int tiles) const { return (int)min((long)tiles, (long)first(p, tiles) + p.chunk); }
    __device__ __forceinline__ bool whole(const WinParams& p, int) const { return p.splits <= 1; }
    // where its sums lie among the parts: token_row = row of Q times heads + head, row = row of the block
    __device__ __forceinline__ long sums(const WinParams& p, long token_row, int) const { return token_row * p.splits + blockIdx.y; }
};
template <int BR, int BC>
struct Share<BR, BC, true> {
    int b, blk, part, parts, item;
    bool any;
    __device__ __forceinline__ void init(const WinParams& p, int idx, int lane) {
        TreeItems<BR, BC> items;
        items.init(p, lane);
        int start = 0, blocks = 1, within;
        if (BR == 128 && p.fold > 0) {
            b = items.find_folded(p, idx, lane, start, blocks, parts, within);
        } else {
            b = items.find(p, idx, lane, start, blocks, parts);
            within = idx - start;
        }
        any = b >= 0;
        b = max(b, 0);
        part = any ? __builtin_amdgcn_readfirstlane(within / blocks) : 0;  // (divisions are vector arithmetic)
        blk = any ? within - part * blocks : 0;
        item = start + within;
    }
    // (the parts of a sequence are as long as one another)
    __device__ __forceinline__ int share(int tiles, int x) const { return __builtin_amdgcn_readfirstlane((int)((unsigned long)tiles * (unsigned)x / (unsigned)parts)); }
    __device__ __forceinline__ int first(const WinParams&, int tiles) const { return share(tiles, part); }
    __device__ __forceinline__ int last(const WinParams&, int tiles) const { return share(tiles, part + 1); }
    __device__ __forceinline__ bool whole(const WinParams&, int) const { return parts <= 1; }
    __device__ __forceinline__ long sums(const WinParams& p, long, int row) const { return ((long)item * p.kv_heads + blockIdx.x % p.kv_heads) * BR + row; }
};

}  // namespace attn
