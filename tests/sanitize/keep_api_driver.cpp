// Exercises the host-side validation of trees, weights and eviction (no GPU needed: every call is a pure host function or is rejected before anything is
// launched).  Built by tests/test_keep_sanitizers.py with the host pass of attn_win_api.hip under AddressSanitizer and UBSan.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../include/attn_mi355x.h"

static int fails = 0;
#define EXPECT(cond)                                            \
    do {                                                        \
        if (!(cond)) {                                          \
            std::printf("FAILED line %d: %s\n", __LINE__, #cond); \
            ++fails;                                            \
        }                                                       \
    } while (0)

static uint64_t state = 7;
static uint32_t next() {
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return (uint32_t)(state >> 33);
}
static int32_t any_int(int32_t ordinary) {
    const uint32_t kind = next() % 8;
    if (kind < 5) return (int32_t)(next() % (uint32_t)(ordinary + 1));
    if (kind == 7) return next() % 2 ? INT32_MAX : INT32_MIN;
    const int64_t v = ((int64_t)1 << (next() % 32)) + (int64_t)(next() % 3) - 1;
    return v > INT32_MAX ? INT32_MAX : (int32_t)v;
}
static int64_t any_stride(int64_t ordinary) {
    const uint32_t kind = next() % 8;
    if (kind < 6) return ordinary;
    return kind == 6 ? ((int64_t)1 << (next() % 63)) : INT64_MAX;
}
template <typename T>
static T pick(std::initializer_list<T> of) {
    return of.begin()[next() % of.size()];
}

int main() {
    void* P = reinterpret_cast<void*>(0x1000);
    float* W = reinterpret_cast<float*>(0x2000);
    int32_t* I = reinterpret_cast<int32_t*>(0x3000);
    const uint32_t* M = reinterpret_cast<const uint32_t*>(0x4000);
    long taken = 0, refused = 0;
    for (int i = 0; i < 400000; ++i) {
        attn_paged_desc p;
        std::memset(&p, 0, sizeof(p));
        p.batch = any_int(70);
        p.kv_heads = any_int(8);
        p.heads = next() % 4 ? (int32_t)((uint32_t)p.kv_heads * (1 + next() % 8) & INT32_MAX) : any_int(64);
        p.d = next() % 4 ? pick({64, 128, 256, 96, 8}) : any_int(300);
        p.total_q = any_int(5000);
        p.max_q = any_int(500);
        p.page_size = pick({8, 16, 64, 4096, 24});
        p.num_pages = any_int(10000);
        p.max_pages = any_int(1000);
        p.max_len = any_int(9000);
        p.scale = 0.1f;
        p.window = any_int(4000);
        p.sinks = any_int(100);
        p.dtype = pick({(int)ATTN_F32, (int)ATTN_BF16});
        p.kind = pick({(int)ATTN_CACHE_PLAIN, (int)ATTN_CACHE_FP8});
        p.q_stride_h = any_stride(p.d);
        p.q_stride_n = any_stride((int64_t)p.d * p.heads);
        p.kv_stride_h = any_stride(p.d);
        p.kv_stride_n = any_stride((int64_t)p.d * p.kv_heads);
        p.page_stride_n = any_stride(p.d);
        p.page_stride_h = any_stride((int64_t)p.d * p.page_size);
        p.page_stride_p = any_stride((int64_t)p.d * p.page_size * 8);
        p.table_stride = any_stride(p.max_pages);
        const int32_t budget = any_int(4000);
        const size_t tree = attn_tree_workspace_bytes(&p), scratch = attn_evict_workspace_bytes(&p, budget);
        tree ? ++taken : ++refused;
        scratch ? ++taken : ++refused;
        EXPECT(tree < (1ull << 50) && scratch < (1ull << 56) && attn_weigh_workspace_bytes(&p) < (1ull << 50));
        // of every sequence and key head: what moves, from and to
        const int64_t cap = std::fmax(0, std::fmin(budget, (double)p.max_len - budget));
        if (scratch && p.batch > 0 && p.heads > 0 && p.max_len > 0) EXPECT(cap <= 64 ? scratch == 256 : scratch >= 8ull * p.batch * p.kv_heads * cap);
        // without pages a call of any size is turned down or has nothing to do
        attn_cache c;
        std::memset(&c, 0, sizeof(c));
        attn_weights w = {W, W, any_stride(p.max_len), any_stride(p.max_len), any_stride(p.max_len), any_stride(p.max_len), 1.f, 0};
        attn_eviction e;
        std::memset(&e, 0, sizeof(e));
        e.budget = budget;
        e.first = any_int(10);
        e.recent = any_int(100);
        e.weight = e.weight_out = W;
        e.new_lens = I;
        e.stride_b = e.stride_h = any_stride(p.max_len);
        e.out_stride_b = e.out_stride_h = any_stride(p.max_len);
        const bool none = p.batch == 0 || p.heads == 0, no_rows = none || p.total_q == 0 || p.max_q == 0;
        EXPECT(attn_tree_fwd(&p, &c, M, any_stride(20), P, P, W, nullptr, 0, nullptr) != ATTN_OK || no_rows);
        EXPECT(attn_tree_commit(&p, &c, M, any_stride(20), I, I + 70000, nullptr) != ATTN_OK || no_rows);
        EXPECT(attn_cache_weigh(&p, &c, P, W, &w, P, ~(size_t)0, nullptr) != ATTN_OK || none || p.max_len == 0);
        EXPECT(attn_cache_evict(&p, &c, &e, P, ~(size_t)0, nullptr) != ATTN_OK || none || p.max_len == 0);
        // with them and without a workspace, or without a place for the lengths
        c.K = c.V = P;
        c.K_exp = c.V_exp = static_cast<uint8_t*>(P);
        c.table = c.lens = c.q_ptr = I;
        EXPECT(attn_tree_commit(&p, &c, M, any_stride(20), I + 70000, I, nullptr) != ATTN_OK || no_rows);
        e.new_lens = I + 70000;
        if (cap > 64) EXPECT(attn_cache_evict(&p, &c, &e, nullptr, 0, nullptr) != ATTN_OK || none || p.max_len == 0);
        w.out = nullptr;
        EXPECT(attn_cache_weigh(&p, &c, P, W, &w, P, ~(size_t)0, nullptr) != ATTN_OK || none || p.max_len == 0);
        const int32_t batch = any_int(70), total = any_int(5000), most = any_int(500);
        EXPECT(attn_tree_mask(batch, total, most, I, nullptr, nullptr, any_stride(16), nullptr) != ATTN_OK || batch == 0 || total == 0 || most == 0);
    }
    EXPECT(taken > 10000 && refused > 10000);
    std::printf("keep api driver: %ld taken, %ld refused, %d failed\n", taken, refused, fails);
    return fails ? 1 : 0;
}
