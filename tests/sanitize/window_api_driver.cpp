// Exercises the host-side validation of windowed attention and the paged cache (no GPU needed: every call is a pure host function or is
// rejected before anything is launched).  Built by tests/test_window_sanitizers.py with the host pass of attn_win_api.hip under
// AddressSanitizer and UBSan.
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

static uint64_t state = 1;
static uint32_t next() {
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    return (uint32_t)(state >> 33);
}
// ordinary sizes, powers of two and their neighbours up to the ends of the type
static int32_t any_int(int32_t ordinary) {
    const uint32_t kind = next() % 8;
    if (kind < 4) return (int32_t)(next() % (uint32_t)(ordinary + 1));
    if (kind == 7) return next() % 2 ? INT32_MAX : INT32_MIN;
    const int64_t v = ((int64_t)1 << (next() % 32)) + (int64_t)(next() % 3) - 1;
    return v > INT32_MAX ? INT32_MAX : (int32_t)v;
}
static int64_t any_stride(int64_t ordinary) {
    const uint32_t kind = next() % 8;
    if (kind < 6) return ordinary;
    return kind == 6 ? ((int64_t)1 << (next() % 63)) : INT64_MAX;
}
static int64_t product(int64_t a, int64_t b, int64_t c = 1) {  // (of sizes that may be anything)
    const __int128 v = (__int128)a * b * c;
    return v > INT64_MAX ? INT64_MAX : v < INT64_MIN ? INT64_MIN : (int64_t)v;
}
template <typename T>
static T pick(std::initializer_list<T> of) {
    return of.begin()[next() % of.size()];
}

int main() {
    void* P = reinterpret_cast<void*>(0x1000);
    const float* L = reinterpret_cast<const float*>(0x2000);
    long taken = 0, refused = 0;
    for (int i = 0; i < 400000; ++i) {
        attn_win_desc w;
        std::memset(&w, 0, sizeof(w));
        w.batch = any_int(70);
        w.kv_heads = any_int(8);
        w.heads = next() % 4 ? (int32_t)product(w.kv_heads, 1 + next() % 8) : any_int(64);
        w.n = any_int(9000);
        w.d = next() % 4 ? pick({64, 128, 256, 96, 8}) : any_int(300);
        w.scale = pick({0.125f, -1.f, 0.f, INFINITY});
        w.window = any_int(4000);
        w.sinks = any_int(100);
        w.dtype = pick({(int)ATTN_F32, (int)ATTN_BF16, 7});
        w.q_stride_n = any_stride(w.d);
        w.q_stride_h = any_stride(product(w.n, w.d));
        w.q_stride_b = any_stride(product(w.n, w.d, 64));
        w.kv_stride_n = any_stride(w.d);
        w.kv_stride_h = any_stride(product(w.n, w.d));
        w.kv_stride_b = any_stride(product(w.n, w.d, 64));
        const size_t need = attn_win_workspace_bytes(&w);
        need ? ++taken : ++refused;
        // row sums are part of it, and no call that a card could hold asks for more than this
        EXPECT(need == 0 || (need >= 4ull * w.batch * w.heads * w.n && need < (1ull << 50)));
        // without its workspace a call of any size is turned down or has nothing to do
        const attn_status st = attn_win_bwd(&w, nullptr, P, P, P, P, P, L, P, P, P, nullptr, 0, nullptr);
        EXPECT(st == ATTN_OK ? w.batch == 0 || w.heads == 0 || w.n == 0 : need == 0 || st == ATTN_ERR_WORKSPACE);

        attn_paged_desc p;
        std::memset(&p, 0, sizeof(p));
        p.batch = any_int(70);
        p.kv_heads = any_int(8);
        p.heads = next() % 4 ? (int32_t)product(p.kv_heads, 1 + next() % 8) : any_int(64);
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
        p.q_stride_n = any_stride(product(p.d, p.heads));
        p.kv_stride_h = any_stride(p.d);
        p.kv_stride_n = any_stride(product(p.d, p.kv_heads));
        p.page_stride_n = any_stride(p.d);
        p.page_stride_h = any_stride(product(p.d, p.page_size));
        p.page_stride_p = any_stride(product(p.d, p.page_size, 8));
        p.table_stride = any_stride(p.max_pages);
        const size_t scratch = attn_paged_workspace_bytes(&p);
        scratch ? ++taken : ++refused;
        EXPECT(scratch < (1ull << 50));
        // launches of what was taken: grids of at most 2^24 workgroups of 256 threads
        if (scratch && p.heads > 0 && p.batch > 0 && p.max_q > 0) {
            const long double rows = (long double)p.batch * p.heads * p.max_q, most = (long double)(1 << 24);
            EXPECT(rows <= 4 * most);
        }
    }
    EXPECT(taken > 10000 && refused > 10000);
    EXPECT(attn_win_workspace_bytes(nullptr) == 0 && attn_paged_workspace_bytes(nullptr) == 0);
    std::printf("window api driver: %ld taken, %ld refused, %d failed\n", taken, refused, fails);
    return fails ? 1 : 0;
}
