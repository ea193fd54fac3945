// C ABI of windowed attention and the paged cache: host-side validation and dispatch.  No device memory is allocated here and
// nothing is launched before every argument has been checked.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "../../include/attn_mi355x.h"
#include "attn_internal.hpp"
#include "attn_win_rules.hpp"
#include "attn_window.hpp"

namespace {

using attn::kMostGroups;
using attn::WinParams;

constexpr int64_t kMostTokens = 1 << 29;    // positions, rows of a (sequence, key head), and sums of two of them in 32 bits

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

attn_status check_heads(int32_t heads, int32_t kv_heads, int32_t d, float scale, int32_t window, int32_t sinks, int32_t dtype) {
    if (heads < 0 || kv_heads < 0 || d < 1 || window < 0 || sinks < 0 || !std::isfinite(scale)) return ATTN_ERR_INVALID_ARG;
    if (heads > 0 && (kv_heads == 0 || heads % kv_heads)) return ATTN_ERR_INVALID_ARG;
    if (dtype != ATTN_F32 && dtype != ATTN_BF16) return ATTN_ERR_UNSUPPORTED;
    if (d > 256 || (dtype == ATTN_BF16 && d % 8)) return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

// rows of d values: `unit` elements are the alignment that the kernels' loads need
bool good_stride(int64_t stride, int64_t count, int32_t d, int unit) {
    return stride >= 0 && stride % unit == 0 && (count <= 1 || stride >= d);
}

attn_status check_win(const attn_win_desc* d) {
    if (!d) return ATTN_ERR_INVALID_ARG;
    if (d->batch < 0 || d->n < 0 || d->reserved != 0) return ATTN_ERR_INVALID_ARG;
    const attn_status st = check_heads(d->heads, d->kv_heads, d->d, d->scale, d->window, d->sinks, d->dtype);
    if (st != ATTN_OK) return st;
    if (d->heads == 0 || d->batch == 0 || d->n == 0) return ATTN_OK;
    const int unit = d->dtype == ATTN_BF16 ? 8 : 1;
    if (d->q_stride_n < d->d || d->kv_stride_n < d->d) return ATTN_ERR_INVALID_ARG;
    if (!good_stride(d->q_stride_n, d->n, d->d, unit) || !good_stride(d->q_stride_h, d->heads, d->d, unit) ||
        !good_stride(d->q_stride_b, d->batch, d->d, unit) || !good_stride(d->kv_stride_n, d->n, d->d, unit) ||
        !good_stride(d->kv_stride_h, d->kv_heads, d->d, unit) || !good_stride(d->kv_stride_b, d->batch, d->d, unit))
        return ATTN_ERR_INVALID_ARG;
    // the tile copies address a tile's rows with 32-bit byte offsets from its first row
    if (d->q_stride_n >= (int64_t)1 << 22 || d->kv_stride_n >= (int64_t)1 << 22) return ATTN_ERR_UNSUPPORTED;
    const int64_t group = d->heads / d->kv_heads, rows = d->n * group, bk = (int64_t)d->batch * d->kv_heads;
    if (rows > kMostTokens || bk > kMostGroups || ((rows + 31) / 32 + 320) * bk > kMostGroups ||
        (int64_t)d->batch * d->heads > kMostGroups || (int64_t)d->batch * d->heads * d->n > kMostGroups * 32)
        return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

bool is_empty(const attn_win_desc* d) { return d->batch == 0 || d->heads == 0 || d->n == 0; }

void set_window(WinParams& p, int32_t window, int32_t sinks, int32_t longest) {
    const attn::WinReach r = attn::win_reach(window, sinks, longest);
    p.window = r.window;
    p.sinks = r.sinks;
}

bool is_wide(const attn_win_desc* d) { return attn::win_is_wide(d->dtype == ATTN_BF16, d->d); }
bool is_wide(const attn_paged_desc* d) { return attn::win_is_wide(d->dtype == ATTN_BF16, d->d, d->kind == ATTN_CACHE_FP8); }
int win_rows(const attn_win_desc* d) { return attn::win_rows(d->batch, d->heads, d->kv_heads, d->n); }
int key_tile(const attn_win_desc* d) { return attn::win_key_tile(is_wide(d)); }

void set_heads(WinParams& p, int32_t heads, int32_t kv_heads) {
    p.heads = heads;
    p.kv_heads = kv_heads;
    p.group = heads / kv_heads;
    p.group_inv = p.group > 1 ? (unsigned)((((uint64_t)1 << 32) + p.group - 1) / p.group) : 0;
}

WinParams win_params(const attn_win_desc* d) {
    WinParams p;
    std::memset(&p, 0, sizeof(p));
    p.q_b = d->q_stride_b;
    p.q_h = d->q_stride_h;
    p.q_n = d->q_stride_n;
    p.k_b = d->kv_stride_b;
    p.k_h = d->kv_stride_h;
    p.k_n = d->kv_stride_n;
    p.batch = d->batch;
    set_heads(p, d->heads, d->kv_heads);
    p.n = d->n;
    p.d = d->d;
    p.scale = d->scale;
    set_window(p, d->window, d->sinks, d->n);
    const attn::WinParts parts = attn::win_parts(is_wide(d), d->batch, d->heads, d->kv_heads, d->n, d->d, p.window, p.sinks);
    p.sink_tiles = parts.sink_tiles;
    p.parts = parts.parts;
    p.rest_parts = parts.rest_parts;
    p.slots = parts.slots;
    p.splits = 1;
    p.chunk = 0x7fffffff;
    return p;
}

size_t rows_bytes(const attn_win_desc* d) { return round_up((size_t)d->batch * d->heads * d->n * sizeof(float), 256); }
size_t parts_bytes(const WinParams& p, int tile) { return (size_t)p.batch * p.kv_heads * p.slots * 2 * tile * p.d * sizeof(float); }

attn_status check_paged(const attn_paged_desc* d) {
    if (!d) return ATTN_ERR_INVALID_ARG;
    if (d->batch < 0 || d->total_q < 0 || d->max_q < 0 || d->max_len < 0 || d->num_pages < 0 || d->max_pages < 0 || d->reserved != 0)
        return ATTN_ERR_INVALID_ARG;
    const attn_status st = check_heads(d->heads, d->kv_heads, d->d, d->scale, d->window, d->sinks, d->dtype);
    if (st != ATTN_OK) return st;
    if (d->kind != ATTN_CACHE_PLAIN && d->kind != ATTN_CACHE_FP8) return ATTN_ERR_UNSUPPORTED;
    const bool fp8 = d->kind == ATTN_CACHE_FP8;
    if (fp8 && d->d % 8) return ATTN_ERR_UNSUPPORTED;
    if (d->page_size < 8 || d->page_size > 4096 || (d->page_size & (d->page_size - 1))) return ATTN_ERR_UNSUPPORTED;
    if ((int64_t)d->max_len > (int64_t)d->max_pages * d->page_size || d->table_stride < d->max_pages) return ATTN_ERR_INVALID_ARG;
    const int unit = d->dtype == ATTN_BF16 ? 8 : 1, page_unit = fp8 ? (d->d % 64 == 0 ? 16 : 8) : unit;
    if (!good_stride(d->q_stride_n, d->total_q, d->d, unit) || !good_stride(d->q_stride_h, d->heads, d->d, unit) ||
        !good_stride(d->kv_stride_n, d->total_q, d->d, unit) || !good_stride(d->kv_stride_h, d->kv_heads, d->d, unit) ||
        !good_stride(d->page_stride_p, d->num_pages, d->d, page_unit) || !good_stride(d->page_stride_h, d->kv_heads, d->d, page_unit) ||
        !good_stride(d->page_stride_n, d->page_size, d->d, page_unit))
        return ATTN_ERR_INVALID_ARG;
    if (d->batch > 65535 || d->max_len > kMostTokens || d->total_q > kMostTokens) return ATTN_ERR_UNSUPPORTED;
    if (d->heads == 0) return ATTN_OK;
    // (every factor is bounded before it is multiplied further)
    const int64_t rows = (int64_t)d->max_q * (d->heads / d->kv_heads), bh = (int64_t)d->batch * d->heads, bk = (int64_t)d->batch * d->kv_heads;
    if (rows > kMostTokens || (d->max_q > 0 && (bk > kMostGroups || bh > 4 * kMostGroups)) || (rows + 15) / 16 * bk > kMostGroups ||
        ((int64_t)d->max_q * d->heads + 3) / 4 * d->batch > kMostGroups || (int64_t)d->max_q * d->kv_heads / 4 * d->batch > kMostGroups)
        return ATTN_ERR_UNSUPPORTED;
    return ATTN_OK;
}

bool is_empty(const attn_paged_desc* d) { return d->batch == 0 || d->heads == 0 || d->total_q == 0 || d->max_q == 0; }

attn_status check_cache(const attn_paged_desc* d, const attn_cache* c) {
    if (!c || !c->K || !c->V || !c->table || !c->lens) return ATTN_ERR_INVALID_ARG;
    if (d->num_pages < 1) return ATTN_ERR_INVALID_ARG;
    if (!c->q_ptr && (int64_t)d->batch * d->max_q > d->total_q) return ATTN_ERR_INVALID_ARG;
    if ((d->dtype == ATTN_BF16 || d->kind == ATTN_CACHE_FP8) && !(aligned16(c->K) && aligned16(c->V))) return ATTN_ERR_INVALID_ARG;
    if (d->kind == ATTN_CACHE_FP8 && (!c->K_exp || !c->V_exp)) return ATTN_ERR_INVALID_ARG;
    return ATTN_OK;
}

int paged_rows(const attn_paged_desc* d) { return attn::paged_rows(is_wide(d), d->batch, d->heads, d->kv_heads, d->total_q, d->max_q); }

WinParams paged_params(const attn_paged_desc* d, const attn_cache* c) {
    WinParams p;
    std::memset(&p, 0, sizeof(p));
    p.q_h = d->q_stride_h;
    p.q_n = d->q_stride_n;
    p.k_b = d->page_stride_p;
    p.k_h = d->page_stride_h;
    p.k_n = d->page_stride_n;
    if (c) {
        p.K = c->K;
        p.V = c->V;
        p.K_exp = c->K_exp;
        p.V_exp = c->V_exp;
        p.table = c->table;
        p.lens = c->lens;
        p.q_ptr = c->q_ptr;
    }
    p.table_stride = d->table_stride;
    p.batch = d->batch;
    set_heads(p, d->heads, d->kv_heads);
    p.n = d->max_q;
    p.d = d->d;
    while ((1 << p.page_shift) < d->page_size) ++p.page_shift;
    p.num_pages = d->num_pages;
    p.total_q = d->total_q;
    p.max_len = d->max_len;
    p.scale = d->scale;
    set_window(p, d->window, d->sinks, d->max_len);
    p.parts = p.rest_parts = 1;
    const attn::PagedSplits splits = attn::paged_splits(is_wide(d), d->batch, d->heads, d->kv_heads, d->d, d->total_q, d->max_q, d->max_len, p.window, p.sinks);
    p.row_blocks = splits.row_blocks;
    p.blocks = splits.blocks;
    p.splits = splits.splits;
    p.chunk = splits.chunk;
    return p;
}

size_t part_ml_bytes(const attn_paged_desc* d, const WinParams& p) {
    return p.splits > 1 ? round_up((size_t)d->total_q * d->heads * p.splits * 2 * sizeof(float), 256) : 0;
}
size_t part_o_bytes(const attn_paged_desc* d, const WinParams& p) {
    return p.splits > 1 ? (size_t)d->total_q * d->heads * p.splits * d->d * sizeof(float) : 0;
}

// Weights and eviction: no token in the cache.  (Without query heads there are no rows, but tokens all the same.)
bool no_cache(const attn_paged_desc* d) { return d->batch == 0 || d->kv_heads == 0 || d->max_len == 0; }

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}

// Pages' rows move in units of 16, 8 or 4 bytes, whatever all of them are a multiple of and aligned to.
int value_bytes(const attn_paged_desc* d) { return d->kind == ATTN_CACHE_FP8 ? 1 : d->dtype == ATTN_BF16 ? 2 : 4; }
int page_unit(const attn_paged_desc* d, const attn_cache* c) {
    const uint64_t es = value_bytes(d);
    const uint64_t all = (es * d->d) | (es * d->page_stride_p) | (es * d->page_stride_h) | (es * d->page_stride_n) |
                         reinterpret_cast<uintptr_t>(c->K) | reinterpret_cast<uintptr_t>(c->V);
    return all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : 4;
}

// Arrays [batch][kv_heads][slots]
bool good_slots(const attn_paged_desc* d, int64_t stride_b, int64_t stride_h, int64_t slots) {
    return stride_b >= 0 && stride_h >= 0 && (d->kv_heads <= 1 || stride_h >= slots) && (d->batch <= 1 || stride_b >= slots);
}

attn_status check_tree(const attn_paged_desc* d, const uint32_t* mask, int64_t mask_stride) {
    if (!mask || mask_stride < 0 || (d->total_q > 1 && mask_stride < ((int64_t)d->max_q + 31) / 32)) return ATTN_ERR_INVALID_ARG;
    return d->max_q > attn::kMostDrafted ? ATTN_ERR_UNSUPPORTED : ATTN_OK;
}

int tree_rows(const attn_paged_desc* d) { return attn::tree_rows(is_wide(d), d->batch, d->heads, d->kv_heads, d->total_q, d->max_q); }
// The parameters of a call on trees, and the workgroups of its launch.
WinParams tree_params(const attn_paged_desc* d, const attn_cache* c, int64_t* grid) {
    WinParams p = paged_params(d, c);
    const attn::TreeShares shares = attn::tree_shares(is_wide(d), d->batch, d->heads, d->kv_heads, d->d, d->total_q, d->max_q, d->max_len, p.window, p.sinks);
    p.row_blocks = shares.row_blocks;
    p.blocks = shares.blocks;
    p.places = shares.places;
    p.least = shares.least;
    p.fold = shares.fold;
    p.splits = 1;
    p.chunk = 0x7fffffff;
    *grid = shares.grid;
    return p;
}
size_t tree_ml_bytes(const attn_paged_desc* d, const WinParams& p, int64_t grid) {
    return p.places > 0 ? round_up((size_t)grid * tree_rows(d) * 2 * sizeof(float), 256) : 0;
}
size_t tree_o_bytes(const attn_paged_desc* d, const WinParams& p, int64_t grid) {
    return p.places > 0 ? (size_t)grid * tree_rows(d) * d->d * sizeof(float) : 0;
}

attn_status check_weigh(const attn_paged_desc* d) {
    const attn_status st = check_paged(d);
    if (st != ATTN_OK || no_cache(d)) return st;
    const int64_t bk = (int64_t)d->batch * d->kv_heads;
    return bk > kMostGroups || ((int64_t)d->max_len + 31) / 32 * bk > kMostGroups ? ATTN_ERR_UNSUPPORTED : ATTN_OK;
}
attn::WeighPlan weigh_plan(const attn_paged_desc* d) {
    return attn::weigh_plan(is_wide(d), d->batch, d->heads, d->kv_heads, d->max_q, d->max_len, d->q_stride_n, d->q_stride_h);
}
size_t weigh_bytes(const attn_paged_desc* d, const attn::WeighPlan& plan) {
    return plan.parts > 1 ? sizeof(float) * plan.parts * d->batch * d->kv_heads * d->max_len : 0;
}

int evict_cap(const attn_paged_desc* d, int32_t budget) { return std::max(0, std::min(budget, d->max_len - budget)); }
attn_status check_evict(const attn_paged_desc* d, int32_t budget) {
    const attn_status st = check_paged(d);
    if (st != ATTN_OK) return st;
    if (budget < 1) return ATTN_ERR_INVALID_ARG;
    return no_cache(d) || (int64_t)d->batch * d->kv_heads <= attn::kMostGroups ? ATTN_OK : ATTN_ERR_UNSUPPORTED;
}

attn_status status_of(hipError_t e) { return e == hipSuccess ? ATTN_OK : ATTN_ERR_DEVICE; }

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t attn_win_workspace_bytes(const attn_win_desc* desc) {
    if (check_win(desc) != ATTN_OK) return 0;
    if (is_empty(desc)) return 256;
    return rows_bytes(desc) + parts_bytes(win_params(desc), key_tile(desc));
}

attn_status attn_win_fwd(const attn_win_desc* desc, const int32_t* lens, const void* Q, const void* K, const void* V, void* O,
                         float* LSE, void* stream) {
    const attn_status st = check_win(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    if (!Q || !K || !V || !O || !LSE) return ATTN_ERR_INVALID_ARG;
    const bool bf16 = desc->dtype == ATTN_BF16;
    if (bf16 && !(aligned16(Q) && aligned16(K) && aligned16(V) && aligned16(O))) return ATTN_ERR_INVALID_ARG;
    WinParams p = win_params(desc);
    p.lens = lens;
    p.Q = Q;
    p.K = K;
    p.V = V;
    p.O = O;
    p.LSE = LSE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return status_of(is_wide(desc) ? attn::launch_win_fwd(false, win_rows(desc), p, s) : attn::launch_win_plain_fwd(bf16, false, p, s));
}

attn_status attn_win_bwd(const attn_win_desc* desc, const int32_t* lens, const void* Q, const void* K, const void* V, const void* O,
                         const void* dO, const float* LSE, void* dQ, void* dK, void* dV, void* workspace, size_t workspace_bytes,
                         void* stream) {
    const attn_status st = check_win(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    if (!Q || !K || !V || !O || !dO || !LSE || !dQ || !dK || !dV) return ATTN_ERR_INVALID_ARG;
    const bool bf16 = desc->dtype == ATTN_BF16;
    if (bf16 && !(aligned16(Q) && aligned16(K) && aligned16(V) && aligned16(O) && aligned16(dO) && aligned16(dQ) && aligned16(dK) && aligned16(dV)))
        return ATTN_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < attn_win_workspace_bytes(desc) || !aligned16(workspace)) return ATTN_ERR_WORKSPACE;
    WinParams p = win_params(desc);
    p.lens = lens;
    p.Q = Q;
    p.K = K;
    p.V = V;
    p.O_in = O;
    p.dO = dO;
    p.LSE_in = LSE;
    p.dQ = dQ;
    p.dK = dK;
    p.dV = dV;
    p.delta = static_cast<float*>(workspace);
    p.part_kv = reinterpret_cast<float*>(static_cast<char*>(workspace) + rows_bytes(desc));
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (bf16) {
        e = attn::launch_win_bwd(win_rows(desc), p, s);
    } else {
        e = attn::launch_win_rows(p, s);
        if (e == hipSuccess) e = attn::launch_win_plain_bwd(p, s);
    }
    if (e == hipSuccess && p.slots > 0) e = attn::launch_win_keys(bf16, key_tile(desc), p, s);
    return status_of(e);
}

attn_status attn_cache_write(const attn_paged_desc* desc, const attn_cache* cache, const void* K, const void* V, void* stream) {
    attn_status st = check_paged(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st != ATTN_OK) return st;
    if (!K || !V || (desc->dtype == ATTN_BF16 && !(aligned16(K) && aligned16(V)))) return ATTN_ERR_INVALID_ARG;
    return status_of(attn::launch_cache_write(desc->dtype == ATTN_BF16, desc->kind == ATTN_CACHE_FP8, paged_params(desc, cache), K, V,
                                              desc->kv_stride_n, desc->kv_stride_h, static_cast<hipStream_t>(stream)));
}

attn_status attn_cache_read(const attn_paged_desc* desc, const attn_cache* cache, void* K, void* V, void* stream) {
    attn_status st = check_paged(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st != ATTN_OK) return st;
    if (!K || !V || (desc->dtype == ATTN_BF16 && !(aligned16(K) && aligned16(V)))) return ATTN_ERR_INVALID_ARG;
    return status_of(attn::launch_cache_read(desc->dtype == ATTN_BF16, desc->kind == ATTN_CACHE_FP8, paged_params(desc, cache), K, V,
                                             desc->kv_stride_n, desc->kv_stride_h, static_cast<hipStream_t>(stream)));
}

size_t attn_paged_workspace_bytes(const attn_paged_desc* desc) {
    if (check_paged(desc) != ATTN_OK) return 0;
    if (is_empty(desc)) return 256;
    const WinParams p = paged_params(desc, nullptr);
    return std::max<size_t>(256, part_ml_bytes(desc, p) + part_o_bytes(desc, p));
}

attn_status attn_paged_fwd(const attn_paged_desc* desc, const attn_cache* cache, const void* Q, void* O, float* LSE, void* workspace,
                           size_t workspace_bytes, void* stream) {
    attn_status st = check_paged(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st != ATTN_OK) return st;
    const bool bf16 = desc->dtype == ATTN_BF16;
    if (!Q || !O || !LSE || (bf16 && !(aligned16(Q) && aligned16(O)))) return ATTN_ERR_INVALID_ARG;
    WinParams p = paged_params(desc, cache);
    if (p.splits > 1 && (!workspace || workspace_bytes < part_ml_bytes(desc, p) + part_o_bytes(desc, p) || !aligned16(workspace)))
        return ATTN_ERR_WORKSPACE;
    p.Q = Q;
    p.O = O;
    p.LSE = LSE;
    p.part_ml = static_cast<float*>(workspace);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + part_ml_bytes(desc, p));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool fp8 = desc->kind == ATTN_CACHE_FP8;
    hipError_t e = is_wide(desc) ? attn::launch_win_fwd(fp8, paged_rows(desc), p, s) : attn::launch_win_plain_fwd(bf16, fp8, p, s);
    if (e == hipSuccess && p.splits > 1) e = attn::launch_win_join(bf16, p, s);
    return status_of(e);
}

attn_status attn_tree_mask(int32_t batch, int32_t total_q, int32_t max_q, const int32_t* q_ptr, const int32_t* parents, uint32_t* mask,
                           int64_t mask_stride, void* stream) {
    if (batch < 0 || total_q < 0 || max_q < 0 || mask_stride < 0) return ATTN_ERR_INVALID_ARG;
    if (batch == 0 || total_q == 0 || max_q == 0) return ATTN_OK;
    if (!parents || !mask || (total_q > 1 && mask_stride < ((int64_t)max_q + 31) / 32) || (!q_ptr && (int64_t)batch * max_q > total_q))
        return ATTN_ERR_INVALID_ARG;
    if (batch > 65535 || max_q > attn::kMostDrafted || total_q > kMostTokens) return ATTN_ERR_UNSUPPORTED;
    WinParams p;
    std::memset(&p, 0, sizeof(p));
    p.batch = batch;
    p.total_q = total_q;
    p.n = max_q;
    p.q_ptr = q_ptr;
    p.tree_stride = mask_stride;
    return status_of(attn::launch_tree_mask(p, parents, mask, static_cast<hipStream_t>(stream)));
}

size_t attn_tree_workspace_bytes(const attn_paged_desc* desc) {
    if (check_paged(desc) != ATTN_OK || desc->max_q > attn::kMostDrafted) return 0;
    if (is_empty(desc)) return 256;
    int64_t grid;
    const WinParams p = tree_params(desc, nullptr, &grid);
    return std::max<size_t>(256, tree_ml_bytes(desc, p, grid) + tree_o_bytes(desc, p, grid));
}

attn_status attn_tree_fwd(const attn_paged_desc* desc, const attn_cache* cache, const uint32_t* mask, int64_t mask_stride, const void* Q, void* O,
                          float* LSE, void* workspace, size_t workspace_bytes, void* stream) {
    attn_status st = check_paged(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st == ATTN_OK) st = check_tree(desc, mask, mask_stride);
    if (st != ATTN_OK) return st;
    const bool bf16 = desc->dtype == ATTN_BF16, fp8 = desc->kind == ATTN_CACHE_FP8;
    if (!Q || !O || !LSE || (bf16 && !(aligned16(Q) && aligned16(O)))) return ATTN_ERR_INVALID_ARG;
    int64_t grid;
    WinParams p = tree_params(desc, cache, &grid);
    const bool joins = p.places > 0;
    if (joins && (!workspace || workspace_bytes < tree_ml_bytes(desc, p, grid) + tree_o_bytes(desc, p, grid) || !aligned16(workspace)))
        return ATTN_ERR_WORKSPACE;
    p.tree = mask;
    p.tree_stride = mask_stride;
    p.Q = Q;
    p.O = O;
    p.LSE = LSE;
    p.part_ml = static_cast<float*>(workspace);
    p.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + tree_ml_bytes(desc, p, grid));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const int rows = tree_rows(desc);
    hipError_t e = is_wide(desc) ? attn::launch_tree_fwd(fp8, rows, grid, p, s) : attn::launch_tree_plain_fwd(bf16, fp8, grid, p, s);
    if (e == hipSuccess && joins) e = attn::launch_tree_join(bf16, rows, p, s);
    return status_of(e);
}

attn_status attn_tree_commit(const attn_paged_desc* desc, const attn_cache* cache, const uint32_t* mask, int64_t mask_stride, const int32_t* leaf,
                             int32_t* new_lens, void* stream) {
    attn_status st = check_paged(desc);
    if (st != ATTN_OK) return st;
    if (is_empty(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st == ATTN_OK) st = check_tree(desc, mask, mask_stride);
    if (st != ATTN_OK) return st;
    const size_t lens_bytes = sizeof(int32_t) * (size_t)desc->batch;
    if (!leaf || !new_lens || overlap(new_lens, lens_bytes, cache->lens, lens_bytes) || overlap(new_lens, lens_bytes, leaf, lens_bytes))
        return ATTN_ERR_INVALID_ARG;
    if ((int64_t)desc->kv_heads * 2 > attn::kMostGroups / desc->batch) return ATTN_ERR_UNSUPPORTED;
    WinParams p = paged_params(desc, cache);
    p.tree = mask;
    p.tree_stride = mask_stride;
    return status_of(attn::launch_tree_commit(value_bytes(desc) * desc->d, page_unit(desc, cache), p, leaf, new_lens, static_cast<hipStream_t>(stream)));
}

size_t attn_weigh_workspace_bytes(const attn_paged_desc* desc) {
    if (check_weigh(desc) != ATTN_OK) return 0;
    if (no_cache(desc)) return 256;
    const attn::WeighPlan plan = weigh_plan(desc);
    return plan.parts > 1 ? std::max<size_t>(512, weigh_bytes(desc, plan)) : 256;  // (256: nothing is kept there, and there may be none)
}

attn_status attn_cache_weigh(const attn_paged_desc* desc, const attn_cache* cache, const void* Q, const float* LSE, const attn_weights* weights,
                             void* workspace, size_t workspace_bytes, void* stream) {
    attn_status st = check_weigh(desc);
    if (st != ATTN_OK) return st;
    if (!weights || weights->reserved != 0 || !std::isfinite(weights->decay)) return ATTN_ERR_INVALID_ARG;
    if (no_cache(desc)) return ATTN_OK;
    st = check_cache(desc, cache);
    if (st != ATTN_OK) return st;
    const bool bf16 = desc->dtype == ATTN_BF16, fp8 = desc->kind == ATTN_CACHE_FP8;
    if (!is_empty(desc) && (!Q || !LSE)) return ATTN_ERR_INVALID_ARG;
    if (!weights->out || (bf16 && !aligned16(Q))) return ATTN_ERR_INVALID_ARG;
    if (!good_slots(desc, weights->out_stride_b, weights->out_stride_h, desc->max_len)) return ATTN_ERR_INVALID_ARG;
    if (weights->in && (!good_slots(desc, weights->in_stride_b, weights->in_stride_h, desc->max_len) ||
                        (weights->in == weights->out && (weights->in_stride_b != weights->out_stride_b || weights->in_stride_h != weights->out_stride_h))))
        return ATTN_ERR_INVALID_ARG;
    attn::WeighParams w;
    std::memset(&w, 0, sizeof(w));
    w.p = paged_params(desc, cache);
    w.p.Q = Q;
    w.p.LSE_in = LSE;
    w.in = weights->in;
    w.out = weights->out;
    w.in_b = weights->in_stride_b;
    w.in_h = weights->in_stride_h;
    w.out_b = weights->out_stride_b;
    w.out_h = weights->out_stride_h;
    w.decay = weights->decay;
    const attn::WeighPlan plan = weigh_plan(desc);
    if (plan.parts > 1 && (!workspace || workspace_bytes < weigh_bytes(desc, plan) || !aligned16(workspace))) return ATTN_ERR_WORKSPACE;
    w.chunk = plan.chunk;
    w.blocks = plan.blocks;
    w.parts = plan.parts;
    w.sums = static_cast<float*>(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return status_of(is_wide(desc) ? attn::launch_weigh(fp8, plan.kind, w, s) : attn::launch_weigh_plain(bf16, fp8, w, s));
}

size_t attn_evict_workspace_bytes(const attn_paged_desc* desc, int32_t budget) {
    if (check_evict(desc, budget) != ATTN_OK) return 0;
    if (no_cache(desc)) return 256;
    const size_t bk = (size_t)desc->batch * desc->kv_heads;
    const size_t cap = (size_t)evict_cap(desc, budget);
    return cap <= attn::kEvictHere ? 256 : sizeof(int32_t) * bk * (1 + 2 * cap);
}

attn_status attn_cache_evict(const attn_paged_desc* desc, const attn_cache* cache, const attn_eviction* eviction, void* workspace,
                             size_t workspace_bytes, void* stream) {
    if (!eviction) return desc ? ATTN_ERR_INVALID_ARG : check_paged(desc);
    const attn_eviction& v = *eviction;
    attn_status st = check_evict(desc, v.budget);
    if (st != ATTN_OK) return st;
    if (v.first < 0 || v.recent < 0 || (int64_t)v.first + v.recent > v.budget || v.reserved != 0) return ATTN_ERR_INVALID_ARG;
    if (no_cache(desc)) return ATTN_OK;
    if (!cache || !cache->K || !cache->V) return ATTN_ERR_INVALID_ARG;
    attn_paged_desc rest = *desc;  // (there are no rows to check)
    rest.max_q = 0;
    st = check_cache(&rest, cache);
    if (st != ATTN_OK) return st;
    if (!v.weight || !v.weight_out || !v.new_lens || (v.pos && !v.pos_out)) return ATTN_ERR_INVALID_ARG;
    if (!good_slots(desc, v.stride_b, v.stride_h, desc->max_len) || !good_slots(desc, v.out_stride_b, v.out_stride_h, std::min(desc->max_len, v.budget)))
        return ATTN_ERR_INVALID_ARG;
    const bool same = v.stride_b == v.out_stride_b && v.stride_h == v.out_stride_h;
    if (!same && (v.weight == v.weight_out || (v.pos && v.pos == v.pos_out))) return ATTN_ERR_INVALID_ARG;
    const size_t lens_bytes = sizeof(int32_t) * (size_t)desc->batch;
    for (const int32_t* in : {cache->lens, v.kept, v.seen})
        if (in && overlap(v.new_lens, lens_bytes, in, lens_bytes)) return ATTN_ERR_INVALID_ARG;
    const bool here = evict_cap(desc, v.budget) <= attn::kEvictHere;
    if (!here && (!workspace || workspace_bytes < attn_evict_workspace_bytes(desc, v.budget) || !aligned16(workspace))) return ATTN_ERR_WORKSPACE;
    attn::EvictParams e;
    std::memset(&e, 0, sizeof(e));
    e.p = paged_params(&rest, cache);
    e.budget = v.budget;
    e.first = v.first;
    e.recent = v.recent;
    e.cap = evict_cap(desc, v.budget);
    e.here = here;
    e.weight = v.weight;
    e.pos = v.pos;
    e.kept = v.kept;
    e.seen = v.seen;
    e.weight_out = v.weight_out;
    e.pos_out = v.pos_out;
    e.new_lens = v.new_lens;
    e.in_b = v.stride_b;
    e.in_h = v.stride_h;
    e.out_b = v.out_stride_b;
    e.out_h = v.out_stride_h;
    const size_t bk = (size_t)desc->batch * desc->kv_heads;
    e.count = static_cast<int32_t*>(workspace);
    e.from = e.count + bk;
    e.to = e.from + bk * e.cap;
    return status_of(attn::launch_evict(value_bytes(desc) * desc->d, page_unit(desc, cache), e, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
#pragma GCC visibility pop
