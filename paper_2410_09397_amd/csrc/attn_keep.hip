// Which tokens stay in the paged cache: the accepted ones of a tree of drafted tokens, or those with the most attention weight.
//
// Rows move whole, codes with their exponents, and no value is computed.  All of it is bound by memory or, at the size of a decoding step, by the chain of
// reads that depend on one another (length, choice, page, row).
#include "attn_internal.hpp"
#include "attn_win_rules.hpp"
#include "attn_window.hpp"

namespace attn {
namespace {

// The place of a token in the pages: of its row (bytes), and of its exponent.  A page outside the cache: none.
struct Place {
    bool there;
    long at, exp;
};
__device__ __forceinline__ Place place_of(const WinParams& p, int b, int kvh, int slot, int value_bytes) {
    Place r = {false, 0, 0};
    const int page = p.table[(long)b * p.table_stride + (slot >> p.page_shift)];
    if ((unsigned)page < (unsigned)p.num_pages) {
        const PageRow row = win_page_row(p, page, kvh, slot);
        r = {true, row.at * value_bytes, row.exp};
    }
    return r;
}

// ---------------------------------------------------------------------------------------------------- accepted tokens
// A workgroup takes K or V of a (sequence, key head).  The x-th of the tokens that stay, drafted token u_x, moves to place x behind the context.
// u_x ascends, so a row is overwritten only by a row that is read with it or later: a chunk of rows is in registers before any of it is written, and
// chunks ascend.
constexpr int kChunkRows = 4;  // rows of a thread on the way

template <typename U>
__global__ void __launch_bounds__(kThreads) tree_commit_kernel(WinParams p, const int32_t* leaf, int32_t* new_lens, int units, int lanes, int value_bytes) {
    __shared__ int stay[kMostDrafted];
    __shared__ int total;
    const int b = blockIdx.y, kvh = (int)(blockIdx.x >> 1), which = (int)(blockIdx.x & 1), tid = threadIdx.x;
    const WinSeq s = win_sequence(p, b);
    const int context = max(0, s.first), t = leaf[b];
    if (tid < 64) {  // a lane for every word of the mask
        uint32_t v = 0;
        if (t >= 0 && t < s.nq && 32 * tid < s.nq) {
            v = p.tree[(s.row0 + t) * p.tree_stride + tid];
            for (int x = 0; x < 32; ++x)
                if (32 * tid + x >= s.nq || s.first + 32 * tid + x < 0) v &= ~(1u << x);
        }
        int upto = __popc(v);
        const int own = upto;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int before = __shfl_up(upto, x, 64);
            upto += tid >= x ? before : 0;
        }
        int at = upto - own;
        for (; v; v &= v - 1) stay[at++] = 32 * tid + __builtin_ctz(v);
        if (tid == 63) total = upto;
    }
    __syncthreads();
    const int count = total;
    if (blockIdx.x == 0 && tid == 0) new_lens[b] = context + count;
    char* pages = static_cast<char*>(const_cast<void*>(which ? p.V : p.K));
    uint8_t* exps = const_cast<uint8_t*>(which ? p.V_exp : p.K_exp);
    const int per = kThreads / lanes, c = tid & (lanes - 1);
    for (int x0 = 0; x0 < count; x0 += per * kChunkRows) {  // (the same for all threads)
        U v[kChunkRows];
        uint8_t e[kChunkRows];
        Place to[kChunkRows];
#pragma unroll
        for (int k = 0; k < kChunkRows; ++k) {
            const int x = x0 + k * per + tid / lanes;
            to[k].there = false;
            if (x < count && c < units && s.first + stay[x] != context + x) {
                const Place from = place_of(p, b, kvh, s.first + stay[x], value_bytes);
                to[k] = place_of(p, b, kvh, context + x, value_bytes);
                to[k].there = to[k].there && from.there;
                if (to[k].there) {
                    v[k] = *reinterpret_cast<const U*>(pages + from.at + (long)c * sizeof(U));
                    if (exps && c == 0) e[k] = exps[from.exp];
                }
            }
        }
        // every row of the chunk is in registers before one of them is written
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kChunkRows; ++k) {
            if (!to[k].there) continue;
            *reinterpret_cast<U*>(pages + to[k].at + (long)c * sizeof(U)) = v[k];
            if (exps && c == 0) exps[to[k].exp] = e[k];
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ eviction
// What tokens are ordered by: weights as whole numbers in the same order, NaN the lowest, tokens that stay in any case the highest.
__device__ __forceinline__ uint32_t weight_key(float w) {
    const uint32_t u = __builtin_bit_cast(uint32_t, w);
    if ((u << 1) > 0xff000000u) return 0u;
    if ((u << 1) == 0u) return 0x80000000u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// Places of set flags of all threads, in the order of the threads; `total`: how many there are.
__device__ __forceinline__ int block_rank(bool flag, int* waves, int& total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const unsigned long set = __builtin_amdgcn_ballot_w64(flag);
    __syncthreads();
    if (lane == 0) waves[w] = __builtin_popcountl(set);
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int x = 0; x < kSelectWaves; ++x) {
        before += x < w ? waves[x] : 0;
        total += waves[x];
    }
    return before + __builtin_popcountl(set & ((1ul << lane) - 1ul));
}

// One workgroup per (sequence, key head): of its len tokens, len - n leave, n = min(len, budget).  The key of the last one that leaves is found 8 bits at
// a time from the top: a histogram of the keys that agree in the bits found so far says in which of 256 bins it lies.  Of tokens with this very key
// those in the highest slots leave.  Free slots below n and tokens that stay above it are as many as one another; both are listed in ascending order.
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(EvictParams e) {
    const WinParams& p = e.p;
    __shared__ int bins[256], waves[kSelectWaves], found[2];
    const int bk = blockIdx.x, b = bk / p.kv_heads, h = bk % p.kv_heads, tid = threadIdx.x;
    const int len = min(max(p.lens[b], 0), p.max_len), n = min(len, e.budget), leave = len - n;
    const long seen = e.seen ? e.seen[b] : len;
    const int kept = e.pos ? (e.kept ? min(max(e.kept[b], 0), len) : 0) : 0;
    const float* weight = e.weight + (long)b * e.in_b + (long)h * e.in_h;
    const int32_t* pos = e.pos ? e.pos + (long)b * e.in_b + (long)h * e.in_h : nullptr;
    float* weight_out = e.weight_out + (long)b * e.out_b + (long)h * e.out_h;
    int32_t* pos_out = e.pos_out ? e.pos_out + (long)b * e.out_b + (long)h * e.out_h : nullptr;
    auto position = [&](int slot) -> long { return slot < kept ? (long)pos[slot] : seen - len + slot; };
    auto key_of = [&](int slot) -> uint32_t {
        const long at = position(slot);
        return at < e.first || at >= seen - e.recent ? 0xffffffffu : weight_key(weight[slot]);
    };
    if (h == 0 && tid == 0) e.new_lens[b] = n;

    uint32_t last = 0;  // the key of the last token that leaves
    int equal = 0;      // how many with this key leave
    if (leave > 0) {
        int rank = leave - 1;  // among the keys that agree with `last` in the bits found
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int x = tid; x < 256; x += kSelectThreads) bins[x] = 0;
            __syncthreads();
            for (int slot = tid; slot < len; slot += kSelectThreads) {
                const uint32_t k = key_of(slot);
                if (shift == 24 || (k >> (shift + 8)) == (last >> (shift + 8))) atomicAdd(&bins[(k >> shift) & 255u], 1);
            }
            __syncthreads();
            if (tid < 64) {  // four bins to a lane
                int c[4], sum = 0;
#pragma unroll
                for (int x = 0; x < 4; ++x) sum += c[x] = bins[4 * tid + x];
                int upto = sum;
#pragma unroll
                for (int x = 1; x < 64; x <<= 1) {
                    const int before = __shfl_up(upto, x, 64);
                    upto += tid >= x ? before : 0;
                }
                int below = upto - sum;
                if (rank >= below && rank < upto) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        if (rank >= below && rank < below + c[x]) {
                            found[0] = 4 * tid + x;
                            found[1] = rank - below;
                        }
                        below += c[x];
                    }
                }
            }
            __syncthreads();
            last |= (uint32_t)found[0] << shift;
            rank = found[1];
        }
        equal = rank + 1;
    }
    // of the tokens with the last key, those behind the first `stay_equal` leave
    int stay_equal = 0;
    if (leave > 0) {
        int all_equal = 0;
        for (int s0 = 0; s0 < len; s0 += kSelectThreads) {
            int here;
            block_rank(s0 + tid < len && key_of(s0 + tid) == last, waves, here);
            all_equal += here;
        }
        stay_equal = all_equal - equal;
    }
    int equals = 0, free = 0, come = 0;
    for (int s0 = 0; s0 < len; s0 += kSelectThreads) {
        const int slot = s0 + tid;
        const bool inside = slot < len;
        const uint32_t k = inside ? key_of(slot) : 0xffffffffu;
        int here;
        const int rank = leave > 0 ? block_rank(inside && k == last, waves, here) : 0;
        const bool goes = leave > 0 && inside && (k < last || (k == last && equals + rank >= stay_equal));
        if (leave > 0) equals += here;
        if (inside && slot < n && !goes) {
            weight_out[slot] = weight[slot];
            if (pos_out) pos_out[slot] = (int32_t)position(slot);
        }
        if (leave > 0) {
            const int f = block_rank(inside && slot < n && goes, waves, here);
            if (inside && slot < n && goes && free + f < e.cap) e.to[(long)bk * e.cap + free + f] = slot;
            free += here;
            const int c = block_rank(inside && slot >= n && !goes, waves, here);
            if (inside && slot >= n && !goes && come + c < e.cap) e.from[(long)bk * e.cap + come + c] = slot;
            come += here;
        }
    }
    if (tid == 0) e.count[bk] = min(min(free, come), e.cap);
}

// Rows, weights and positions of the tokens that move.  What is read lies at slots of at least n, what is written below.
constexpr int kMoveRows = 4;  // rows of K and V of a thread on the way
template <typename U>
__global__ void __launch_bounds__(kThreads) evict_move_kernel(EvictParams e, int blocks, int units, int lanes, int value_bytes) {
    const WinParams& p = e.p;
    const int bk = blockIdx.x / blocks, b = bk / p.kv_heads, h = bk % p.kv_heads, tid = threadIdx.x;
    const int count = e.count[bk], per = kThreads / lanes, c = tid & (lanes - 1);
    char *K = static_cast<char*>(const_cast<void*>(p.K)), *V = static_cast<char*>(const_cast<void*>(p.V));
    uint8_t *K_exp = const_cast<uint8_t*>(p.K_exp), *V_exp = const_cast<uint8_t*>(p.V_exp);
    const int len = min(max(p.lens[b], 0), p.max_len);
    const long seen = e.seen ? e.seen[b] : len;
    const int kept = e.pos ? (e.kept ? min(max(e.kept[b], 0), len) : 0) : 0;
    for (int x0 = (blockIdx.x % blocks) * per * kMoveRows; x0 < count; x0 += blocks * per * kMoveRows) {
        U k[kMoveRows], v[kMoveRows];
        uint8_t ke[kMoveRows], ve[kMoveRows];
        Place to[kMoveRows];
#pragma unroll
        for (int r = 0; r < kMoveRows; ++r) {
            const int x = x0 + r * per + tid / lanes;
            to[r].there = false;
            if (x >= count || c >= units) continue;
            const int source = e.from[(long)bk * e.cap + x], target = e.to[(long)bk * e.cap + x];
            const Place from = place_of(p, b, h, source, value_bytes);
            to[r] = place_of(p, b, h, target, value_bytes);
            to[r].there = to[r].there && from.there;
            if (to[r].there) {
                k[r] = *reinterpret_cast<const U*>(K + from.at + (long)c * sizeof(U));
                v[r] = *reinterpret_cast<const U*>(V + from.at + (long)c * sizeof(U));
                if (K_exp && c == 0) {
                    ke[r] = K_exp[from.exp];
                    ve[r] = V_exp[from.exp];
                }
            }
            if (c == 0) {
                e.weight_out[(long)b * e.out_b + (long)h * e.out_h + target] = e.weight[(long)b * e.in_b + (long)h * e.in_h + source];
                if (e.pos_out)
                    e.pos_out[(long)b * e.out_b + (long)h * e.out_h + target] =
                        source < kept ? e.pos[(long)b * e.in_b + (long)h * e.in_h + source] : (int32_t)(seen - len + source);
            }
        }
#pragma unroll
        for (int r = 0; r < kMoveRows; ++r) {
            if (!to[r].there) continue;
            *reinterpret_cast<U*>(K + to[r].at + (long)c * sizeof(U)) = k[r];
            *reinterpret_cast<U*>(V + to[r].at + (long)c * sizeof(U)) = v[r];
            if (K_exp && c == 0) {
                K_exp[to[r].exp] = ke[r];
                V_exp[to[r].exp] = ve[r];
            }
        }
    }
}

// f(a value of the unit's type)
template <typename F>
void with_unit(int unit, F f) {
    if (unit == 16) f(u32x4{});
    else if (unit == 8) f(u32x2{});
    else f(uint32_t{});
}
int lanes_of(int units) {
    int lanes = 1;
    while (lanes < units) lanes *= 2;
    return lanes;
}

}  // namespace

hipError_t launch_tree_commit(int row_bytes, int unit, const WinParams& p, const int32_t* leaf, int32_t* new_lens, hipStream_t stream) {
    const int units = row_bytes / unit, lanes = lanes_of(units);
    if (p.n > kMostDrafted || row_bytes % unit || lanes > kThreads) return hipErrorInvalidValue;
    with_unit(unit, [&](auto u) {
        hipLaunchKernelGGL(tree_commit_kernel<decltype(u)>, dim3((unsigned)p.kv_heads * 2, (unsigned)p.batch), dim3(kThreads), 0, stream, p, leaf, new_lens, units,
                           lanes, row_bytes / p.d);
    });
    return hipGetLastError();
}
hipError_t launch_evict(int row_bytes, int unit, const EvictParams& e, hipStream_t stream) {
    const int units = row_bytes / unit, lanes = lanes_of(units), bk = e.p.batch * e.p.kv_heads;
    if (row_bytes % unit || lanes > kThreads) return hipErrorInvalidValue;
    hipLaunchKernelGGL(evict_select_kernel, dim3((unsigned)bk), dim3(kSelectThreads), 0, stream, e);
    if (e.cap > 0) {
        const int blocks = evict_blocks(bk, e.cap, kThreads / lanes * kMoveRows);
        with_unit(unit, [&](auto u) {
            hipLaunchKernelGGL(evict_move_kernel<decltype(u)>, dim3((unsigned)(bk * blocks)), dim3(kThreads), 0, stream, e, blocks, units, lanes, row_bytes / e.p.d);
        });
    }
    return hipGetLastError();
}

}  // namespace attn
