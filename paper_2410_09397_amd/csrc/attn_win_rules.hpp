// Rules that choose the kernels of windowed attention and of the paged cache by the size of the call, and share their work out: nothing of the
// device, so that the CPU tests run them as well.
#pragma once
#include <algorithm>
#include <cstdint>

namespace attn {

constexpr int kNoWindow = 0x3fffffff;           // larger than any distance; a position plus or minus it stays in range
constexpr int64_t kMostGroups = (1 << 24) - 1;  // workgroups of 256 threads in a launch

// Whether the bf16-MFMA kernels take a call: bf16 of any head dimension, quantised pages of those that fill a kernel's width.
inline bool win_is_wide(bool bf16, int d, bool fp8 = false) { return bf16 && (!fp8 || d == 64 || d == 128 || d == 256); }

// A window that hides nothing of a sequence of `longest` keys is none, and then nothing is a sink.
struct WinReach {
    int window, sinks;
};
inline WinReach win_reach(int window, int sinks, int longest) {
    const bool limits = window > 0 && window < longest && sinks < longest;
    return {limits ? window : kNoWindow, limits ? sinks : 0};
}

// Rows of a workgroup: 128, or 64 where blocks of 128 would not be more than three for two CUs.  us, forward / backward, 128 -> 64 rows, h heads on k key heads:
//   d = 64    h4 k4 n300 9.4 / 19.8 -> 8.4 / 17.7                d = 256   h8 k2 n1024 55 / 110 -> 36 / 87
//   d = 128   h8 k2 n1024 26 / 60 -> 20 / 50     h4 k1 n4096 w1024 31 / 74 -> 23 / 62     h16 k2 n2048 48 / 128 -> 39 / 115
//   16 sequences of 1 to 256 new tokens, h32 k8 w1024 d = 128 (280 to 336 blocks) 54 -> 44
//   beyond the line: d = 64 b2 h16 k4 n2048 w256 16.6 / 56 -> 18.3 / 59
inline int block_rows(int64_t blocks128) { return blocks128 <= 384 ? 64 : 128; }
inline int win_rows(int batch, int heads, int kv_heads, int n) {
    return block_rows(((int64_t)n * (heads / kv_heads) + 127) / 128 * batch * kv_heads);
}

// Keys of a tile of the backward's key owners.
inline int win_key_tile(bool wide) { return wide ? 64 : 32; }

// Workgroups of the key owners.  One streams window + tile tokens per head of its group, one of sink keys all of them: those are shared out over as
// many workgroups as make the shares about as long (at most 64, and fewer where there are many sink tiles).  Where all of them
// together are no more than half of the places that are counted here (512 up to d = 128, two on a CU; 256 beyond, one on a CU), the tokens of every tile are shared out: at least two
// tiles of tokens to each, and enough of them over all heads of the group (twelve; the 32-bit kernels, whose waves take them in turn, six) to pay for the
// sums' way through memory and the launch behind.  us of the backward, one workgroup per tile -> shared, h heads on k key heads:
//   d = 128, no window   h8 k2 n512 63 -> 39   h8 k2 n1024 114 -> 55   h16 k2 n2048 380 -> 128      d = 256, no window  h8 k2 n1024 211 -> 104
//   d = 128, window      h4 k1 n4096 w1024 135 -> 76   h16 k4 n2048 w512 85 -> 77   h8 k8 n1024 w256 (too few tiles) 35 -> 45
//   d = 64               h4 k4 n300 (too few tiles) 20 -> 22      d = 256, window     h8 k4 n2048 w300 (too few tiles) 73 -> 77
// Both numbers are one line for all calls, and other lines suit some of them better.  Twelve tiles -> ten: d = 64 w256, h16 k4 n2048 two sequences 42 -> 45
// (with sinks, whose sums make the launch anyway, 52 -> 53), one sequence 40 -> 37 (with sinks 48 -> 42); d = 128, the same, one sequence 52 -> 50 (59 -> 56); d = 40 h8 k2 n1031 42 -> 38.
// 512 places -> the 768 that the registers and LDS of d = 64 allow: no window h8 k2 n8192 462 -> 388, h6 k3 n2500 63 -> 62, w700 h12 k3 n6000 108 -> 91, w256 as it was.
// 256 places -> 512 for the padded rows of 129 to 255: h8 k2 n2048 d = 160 187 -> 166, h16 k4 n2048 d = 200 w512 173 -> 165.
// sink_tiles: how many of the first key tiles are shared out over `parts` workgroups each (0 where parts is 1); the others over rest_parts;
// slots: workgroups of a (sequence, key head) whose sums are parts.  window, sinks: as win_reach gives them.
struct WinParts {
    int sink_tiles, parts, rest_parts, slots;
};
inline WinParts win_parts(bool wide, int batch, int heads, int kv_heads, int n, int d, int window, int sinks) {
    const int tile = win_key_tile(wide);
    const int64_t places = wide && d > 128 ? 256 : 512;
    const int64_t tiles = (n + tile - 1) / tile, bk = (int64_t)batch * kv_heads;
    const int64_t span = std::min<int64_t>((int64_t)window + tile, n), token_tiles = (span + tile - 1) / tile;
    WinParts p = {sinks > 0 ? (int)std::min<int64_t>((sinks + tile - 1) / tile, tiles) : 0, 1, 1, 0};
    if (p.sink_tiles > 0) p.parts = (int)std::min<int64_t>(std::min<int64_t>((n + span - 1) / span, 64), std::max(1, 256 / p.sink_tiles));
    const int64_t rest = std::min(std::min(places / std::max<int64_t>(1, tiles * bk), token_tiles / 2), token_tiles * (heads / kv_heads) / (wide ? 12 : 6));
    if (rest > 1) {
        p.rest_parts = (int)rest;
        p.parts = std::min(64, (int)rest * p.parts);
    }
    // (the sums of the parts are a launch of up to 64 lanes for every key and gradient)
    if (bk * (p.rest_parts > 1 ? n : (int64_t)p.sink_tiles * tile) / 2 > kMostGroups) p.parts = p.rest_parts = 1;
    if (p.parts <= 1) p.sink_tiles = 0;
    p.slots = p.sink_tiles * (p.parts > 1 ? p.parts : 0) + (p.rest_parts > 1 ? (int)(tiles - p.sink_tiles) * p.rest_parts : 0);
    return p;
}

// Rows of a workgroup of the paged forward: see attn_win_fwd.hip.
inline int paged_rows(bool wide, int batch, int heads, int kv_heads, int total_q, int max_q) {
    const int64_t group = heads / kv_heads, rows = max_q * group;
    if (!wide) return 32;
    // (total_q bounds the row blocks that have rows where the sequences' new tokens differ in number)
    if (rows > 64) return block_rows(std::min((rows + 127) / 128 * batch, total_q * group / 128 + batch) * kv_heads);
    return rows > 16 ? 32 : 16;
}

// How the keys of a row block are shared out: with fewer row blocks than the chip has places for, a workgroup takes `chunk` tiles.
// row_blocks: of the longest sequence; blocks: at most of all of them.
struct PagedSplits {
    int row_blocks, blocks, splits, chunk;
};
inline PagedSplits paged_splits(bool wide, int batch, int heads, int kv_heads, int d, int total_q, int max_q, int max_len, int window, int sinks) {
    const int64_t group = heads / kv_heads, rows = paged_rows(wide, batch, heads, kv_heads, total_q, max_q), tile = rows >= 64 ? 64 : 32;
    const bool few = rows < 64;
    PagedSplits p = {(int)((max_q * group + rows - 1) / rows), 0, 1, 0x7fffffff};
    p.blocks = (int)std::min((int64_t)p.row_blocks * batch, total_q * group / rows + batch);
    const int64_t blocks = (int64_t)p.blocks * kv_heads;
    // (the windows of a block reach over window + its tokens - 1 keys, which lie in one tile more than they fill, as the sinks do)
    const int64_t keys = std::min<int64_t>(max_len, (int64_t)window + max_q) + sinks, tiles = keys / tile + 3;
    // How many: as many as there are places (some more for few rows, whose lengths differ), but not in pieces so small that the launch that
    // joins them costs more than they save.  us, split -> not: one token of b sequences of L keys, d = 128, quantised: b1 L600 11.0 -> 10.4,
    // b1 L1000 11.2 -> 13.6, b64 L1000 33 -> 24; d = 256: b1 L300 12.9 -> 11.4, b1 L600 13.0 -> 14.9
    const int64_t want = std::min<int64_t>(64, (few ? 2048 : 512) / std::max<int64_t>(1, blocks));
    const int64_t least = !few ? 16 : blocks >= 256 ? 32 : d > 128 ? 8 : 12;  // tiles
    const int64_t splits = (int64_t)total_q * heads <= kMostGroups ? std::min(want, tiles / least) : 1;
    if (splits > 1) {
        p.chunk = (int)((tiles + splits - 1) / splits);
        p.splits = (int)((tiles + p.chunk - 1) / p.chunk);
    }
    return p;
}

// (The times below, of trees, weights and eviction, compare two or more forms of the code as it stood when a line was drawn.  Later steps have made the calls shorter, and the same call
// stands with different times in different comments: what counts is the ratio within a comment.)
//
// Trees of drafted tokens: rows of a workgroup.  Unlike the new tokens of a batch in their order, whose blocks are as many as their tokens make them, a tree has one or two
// blocks, and what fills the chip are the parts of the context: more than 64 rows always take blocks of 128, which convert and read a tile half as often.  us of a call
// with 128 / 64 rows, h32 k8 d = 128, 64 drafted tokens: 16 sequences of 100 to 8192 tokens 84 / 144 (quantised), 74 / 119; one of 65536 102 / 124; one of 1000 (where
// the chip is not full) 25.7 / 23.5; d = 256 h16 k4, 4 sequences 64 / 75.
constexpr int kMostDrafted = 1024;  // drafted tokens of a sequence: their masks are 32 words
// The kernels there are, and keys of their tiles.
inline bool tree_rows_exist(bool bf16, int rows) { return rows == 32 || (bf16 && (rows == 16 || rows == 128)); }
constexpr int tree_tile(int rows) { return rows == 128 ? 64 : 32; }
inline int tree_rows(bool wide, int batch, int heads, int kv_heads, int total_q, int max_q) {
    const int64_t group = heads / kv_heads, rows = max_q * group;
    if (!wide || rows <= 64) return paged_rows(wide, batch, heads, kv_heads, total_q, max_q);
    return 128;
}
// How a call on trees is shared out (see TreeItems): a part is `least` tiles, or as many as make `places` of all (0: nothing is shared out, and there are no sums to
// join).  grid: workgroups, each of which has a block of sums if there are any to join.
// Where the row blocks leave places free, parts are sized to fill them once (a round and a half, two, three: 16 sequences with 64 drafted 81 -> 89, 87, 96 us, one of 65536 tokens
// 106 -> 128, 124, 121). Where row blocks alone are more than the chip's places, parts come in two rounds, so that the last ones are short.  us: parts of at least 4 tiles of 64 keys / of 8, one sequence of
// 1000 tokens with 64 drafted 25.8 / 30.6, 8 sequences of 500 to 4000 with 30 38.5 / 40.8; at least 16 tiles of 32 keys, of four waves / 32, 16 sequences with 8 drafted 44.8 /
// 47.2; two rounds / one / four, 64 sequences of 100 to 2000 tokens with 40 drafted 135 / 140 / 139.
// fold: one round of 128 rows, two workgroups to a CU, of several sequences: long parts share a CU with short ones (see find_folded; 16 sequences with 64 drafted, quantised 82.3 -> 79.3, not 70.4 -> 67.6;
// 8 sequences of 500 to 4000 with 30 38.4 -> 38.2).
constexpr int64_t kTreeLeast = 4, kTreeLeastFew = 16, kTreeRounds = 2;
struct TreeShares {
    int row_blocks, blocks, places, least, fold;
    int64_t grid;
};
inline TreeShares tree_shares(bool wide, int batch, int heads, int kv_heads, int d, int total_q, int max_q, int max_len, int window, int sinks) {
    const int64_t group = heads / kv_heads, rows = tree_rows(wide, batch, heads, kv_heads, total_q, max_q), tile = tree_tile((int)rows);
    TreeShares p = {(int)((max_q * group + rows - 1) / rows), 0, 0, 0x7fffffff, 0, 0};
    p.blocks = (int)std::min((int64_t)p.row_blocks * batch, total_q * group / rows + batch);
    p.grid = (int64_t)p.blocks * kv_heads;
    const int64_t chip = rows == 16 && d <= 128 ? 1024 : d > 128 ? 256 : 512, of_head = std::max<int64_t>(1, chip / kv_heads);
    // (the windows reach over window keys, the sinks and the drafted tokens have tiles of their own, and each kind may fill one more than its keys)
    const int64_t keys = std::min<int64_t>(max_len, (int64_t)window + max_q) + sinks, tiles = keys / tile + 4, least = rows == 128 ? kTreeLeast : kTreeLeastFew;
    if (tiles < 2 * least || p.grid > 8 * chip || (int64_t)total_q * heads > kMostGroups) return p;
    p.places = (int)(p.blocks <= of_head ? of_head - p.blocks / 2 : kTreeRounds * of_head);
    if (rows == 128 && d <= 128 && p.blocks <= of_head && batch > 1 && batch <= 64) p.fold = (int)(256 / kv_heads);
    p.least = (int)std::max(least, (tiles + 63) / 64);  // (64 parts at most: the joining launch has a lane for each)
    p.grid += (p.places + 1) * (int64_t)kv_heads;  // (one more: the device divides in 32-bit floating point)
    return p;
}

// The folded order of the items of a key head (see find_folded): what the sequence `own`, with parts of `size` tiles, learns of the others, each counted once.
struct TreeFold {
    int all = 0, before = 0, first = 0;  // items of all sequences; in front of its own in the order of the sequences (that of the sums); and in that of the parts' sizes
    constexpr void count(int own, int size, int other, int items, int tiles) {
        all += items;
        before += other < own ? items : 0;
        first += tiles > size || (tiles == size && other < own) ? items : 0;
    }
    // which item workgroup idx has in the order of the sizes: the later half comes back from the last
    static constexpr int place(int idx, int all, int fold) { return idx < fold ? idx : all - 1 - (idx - fold); }
    constexpr bool has(int place, int items) const { return place >= first && place - first < items; }
};

// Rows of a workgroup of the joining launch, out of blocks of `rows`: 8, or as many as leave 2048 workgroups (each looks its sequence up first).  us of a call with
// 512 / 1024 / 2048 / 4096 / any number of them: 64 sequences with 40 drafted tokens 129 / 130 / 121 / 119 / 139, 16 with 64 84 / 78 / 76 / 80 / 79.
constexpr int64_t kJoinGroups = 2048;
inline int join_rows(int64_t blocks, int rows) {
    int many = 8;
    while (many < rows && blocks * (rows / many) > kJoinGroups) many *= 2;
    return many;
}

// Kernels of attn_cache_weigh by the rows of a (sequence, key head): at most 16, one tile of 128, more of them; any: groups or strides that a tile does not hold (and the
// kernel of 32-bit arithmetic).  us of a call: one kernel for all, 16 rows at a time -> these, h32 k8 d = 128: newest token of 64 sequences (quantised) 72 -> 31, last 32
// tokens of 8 prompts 52 -> 18, a prompt of 4096 tokens 1101 -> 101.
// One tile or less: keys of a workgroup, as many as leave 2048 workgroups (512 / 1024 / 4096: last 32 tokens of 8 prompts 24.9 / 19.9 / 21.1 for 18.1).
// Groups of heads that do not divide 128 leave rows of a tile empty, and those tiles, like all of d = 256, take the rows 32 at a time, without the products between the exponentials: a prompt of
// 4096 tokens, d = 128, h32 k8 99 us (690 TFLOP/s), h24 k8 93 (560), h28 k4 120 (500); d = 256 h16 k4 149 (460).
// Many rows: the keys of a workgroup are 256, and the tiles of rows are shared out until there are some 768 workgroups, a round and a half, with two tiles each at least.  us of
// 512 / 768 / 1024 workgroups: a prompt of 4096 tokens 114 / 101 / 105, 4 prompts of 500 to 2000 107 / 93 / 91, the last 512 of 16384 tokens 90 / 90 / 98; one / two / four tiles:
// a prompt of 300 tokens 16 / 21 / 32, d = 256, 64 of 4000 tokens 47 / 39 / 39.
enum WeighRowsKind { kWeighOne, kWeighFew, kWeighMany, kWeighAny };
constexpr int64_t kWeighGroups = 2048;
constexpr int64_t kWeighParts = 768, kWeighLeast = 2;
struct WeighPlan {
    WeighRowsKind kind;
    int blocks, chunk, parts;  // workgroups of a (sequence, key head): blocks of `chunk` keys, times parts of the rows
};
inline WeighPlan weigh_plan(bool wide, int batch, int heads, int kv_heads, int max_q, int max_len, int64_t q_stride_n, int64_t q_stride_h) {
    const int64_t group = heads / kv_heads, rows = max_q * group, bk = (int64_t)batch * kv_heads;
    const bool tiles = group <= 128 && q_stride_n < (1 << 22) && q_stride_h < (1 << 22);
    WeighPlan p = {rows <= 16 ? kWeighOne : !tiles || !wide ? kWeighAny : rows <= 128 ? kWeighFew : kWeighMany, 0, 128, 1};
    if (!wide && rows > 32) p.chunk = 32;  // (32-bit arithmetic: see weigh_plain_kernel)
    if (p.kind == kWeighMany) p.chunk = 256;
    else while (wide && p.chunk < 1024 && (max_len + p.chunk * 2 - 1) / (p.chunk * 2) * bk >= kWeighGroups) p.chunk *= 2;
    p.blocks = (max_len + p.chunk - 1) / p.chunk;
    if (p.kind == kWeighMany) {
        const int64_t of_rows = (max_q + 128 / group - 1) / (128 / group);  // tiles
        p.parts = (int)std::max<int64_t>(1, std::min(std::min<int64_t>(64, kWeighParts / std::max<int64_t>(1, p.blocks * bk)), of_rows / kWeighLeast));
    }
    return p;
}

constexpr int kEvictHere = 64;  // moves that the workgroup that chooses them makes itself
// Workgroups that move a (sequence, key head)'s kept tokens, `rows` at a time, of which there are at most `cap`.
inline int evict_blocks(int64_t bk, int64_t cap, int64_t rows) {
    return (int)std::max<int64_t>(1, std::min((cap + rows - 1) / rows, std::min<int64_t>(1024, kMostGroups / std::max<int64_t>(1, bk))));
}

// Threads that share a row of the cache, 8 values each.
inline int cache_lanes(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }
// Rows per thread of writing and reading: K and V of so many tokens or heads are on the way at a time.  us of 88 MB of prompts, 1 row of K or V / 2 / 4 / 8
// rows of both to a thread: write 37 / 22 / 25 / 38, read 27 / 17 / 18 / 21.  A call of few rows, a decoding step, has one each: 4.2 us
// against 6.5 with four for 64 tokens of 8 heads.  The line: about one workgroup of eight waves' rows for every CU.
constexpr int kManyRows = 2;
inline int cache_rows_per_thread(int kv_heads, int total_q, int d) { return (int64_t)total_q * kv_heads * cache_lanes(d) > 256 * 2 * 256 ? kManyRows : 1; }

}  // namespace attn
