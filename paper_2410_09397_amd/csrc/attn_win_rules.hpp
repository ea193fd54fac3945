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

// Threads that share a row of the cache, 8 values each.
inline int cache_lanes(int d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }
// Rows per thread of writing and reading: K and V of so many tokens or heads are on the way at a time.  us of 88 MB of prompts, 1 row of K or V / 2 / 4 / 8
// rows of both to a thread: write 37 / 22 / 25 / 38, read 27 / 17 / 18 / 21.  A call of few rows, a decoding step, has one each: 4.2 us
// against 6.5 with four for 64 tokens of 8 heads.  The line: about one workgroup of eight waves' rows for every CU.
constexpr int kManyRows = 2;
inline int cache_rows_per_thread(int kv_heads, int total_q, int d) { return (int64_t)total_q * kv_heads * cache_lanes(d) > 256 * 2 * 256 ? kManyRows : 1; }

}  // namespace attn
