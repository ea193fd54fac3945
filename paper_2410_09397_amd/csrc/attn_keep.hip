// Which tokens stay in the paged cache: the accepted ones of a tree of drafted tokens, or those with the most attention weight.
//
// Rows move whole, codes with their exponents, and no value is computed.  All of it is bound by memory or, at the size of a decoding step, by the chain of
// reads that depend on one another (length, choice, page, row).
#include <type_traits>

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

// Sums of a wave's values up to and including each lane's, by moves between lanes that are part of the additions (an exchange through LDS takes some 100 cycles, and the next of
// the six waits for it: a scan of the bins in evict_select_kernel took 0.8 us).
__device__ __forceinline__ int wave_sums(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);  // from the lane before in a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);  // two before
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // the last lane of a row to the next row, rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2 and 3
    return v;
}

// ---------------------------------------------------------------------------------------------------- accepted tokens
// A workgroup takes K or V of a (sequence, key head).  The x-th of the tokens that stay, drafted token u_x, moves to place x behind the context.
// u_x ascends, so a row is overwritten only by a row that is read with it or later: a chunk of rows is in registers before any of it is written, and
// chunks ascend.  The chain of reads bounds it: 64 sequences with 64 drafted tokens each, k8 d = 128, quantised, 5.9 us, 15 tokens of 4 heads 4.6.
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
        const int own = __popc(v), upto = wave_sums(own);
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

constexpr uint32_t kStays = 0xfffffffeu;  // above the key of every weight, and below ~0
// The tokens of a (sequence, key head).
struct EvictSequence {
    int len, n, kept;  // n stay; slots below `kept` have their positions in an array
    long seen;
    const float* weight;
    const int32_t* pos;
    float* weight_out;
    int32_t* pos_out;
    __device__ __forceinline__ void init(const EvictParams& e, int b, int h) {
        len = min(max(e.p.lens[b], 0), e.p.max_len);
        n = min(len, e.budget);
        seen = e.seen ? e.seen[b] : len;
        kept = e.pos ? (e.kept ? min(max(e.kept[b], 0), len) : 0) : 0;
        weight = e.weight + (long)b * e.in_b + (long)h * e.in_h;
        pos = e.pos ? e.pos + (long)b * e.in_b + (long)h * e.in_h : nullptr;
        weight_out = e.weight_out + (long)b * e.out_b + (long)h * e.out_h;
        pos_out = e.pos_out ? e.pos_out + (long)b * e.out_b + (long)h * e.out_h : nullptr;
    }
    __device__ __forceinline__ long position(int slot) const { return slot < kept ? (long)pos[slot] : seen - len + slot; }
    __device__ __forceinline__ uint32_t key(const EvictParams& e, float w, long at) const { return at < e.first || at >= seen - e.recent ? kStays : weight_key(w); }
};

// Rows, weights and positions of the tokens that move, by kThreads-sized steps: lists of `count` slots, this workgroup's first row and the distance to its next ones.  What is read
// lies in slots of at least n, what is written below.
constexpr int kMoveRows = 4;  // rows of K and V of a thread on the way
template <typename U>
__device__ __forceinline__ void evict_rows(const EvictParams& e, const EvictSequence& q, int b, int h, const int* from, const int* to, int count, int row0, int step, int threads,
                                           int units, int lanes, int value_bytes) {
    const WinParams& p = e.p;
    const int tid = threadIdx.x, per = threads / lanes, c = tid & (lanes - 1);
    char *K = static_cast<char*>(const_cast<void*>(p.K)), *V = static_cast<char*>(const_cast<void*>(p.V));
    uint8_t *K_exp = const_cast<uint8_t*>(p.K_exp), *V_exp = const_cast<uint8_t*>(p.V_exp);
    for (int x0 = row0; x0 < count; x0 += step) {
        U k[kMoveRows], v[kMoveRows];
        uint8_t ke[kMoveRows], ve[kMoveRows];
        Place place[kMoveRows];
#pragma unroll
        for (int r = 0; r < kMoveRows; ++r) {
            const int x = x0 + r * per + tid / lanes;
            place[r].there = false;
            if (x >= count || c >= units) continue;
            const int source = from[x], target = to[x];
            const Place at = place_of(p, b, h, source, value_bytes);
            place[r] = place_of(p, b, h, target, value_bytes);
            place[r].there = place[r].there && at.there;
            if (place[r].there) {
                k[r] = *reinterpret_cast<const U*>(K + at.at + (long)c * sizeof(U));
                v[r] = *reinterpret_cast<const U*>(V + at.at + (long)c * sizeof(U));
                if (K_exp && c == 0) {
                    ke[r] = K_exp[at.exp];
                    ve[r] = V_exp[at.exp];
                }
            }
            if (c == 0) {
                q.weight_out[target] = q.weight[source];
                if (q.pos_out) q.pos_out[target] = (int32_t)q.position(source);
            }
        }
#pragma unroll
        for (int r = 0; r < kMoveRows; ++r) {
            if (!place[r].there) continue;
            *reinterpret_cast<U*>(K + place[r].at + (long)c * sizeof(U)) = k[r];
            *reinterpret_cast<U*>(V + place[r].at + (long)c * sizeof(U)) = v[r];
            if (K_exp && c == 0) {
                K_exp[place[r].exp] = ke[r];
                V_exp[place[r].exp] = ve[r];
            }
        }
    }
}

// One workgroup per (sequence, key head): of its len tokens, len - n leave.  The key of the last one that leaves is found 11, 11 and 10 bits at a time from the top: a histogram of
// the keys that agree in the bits found so far says in which bin it lies, and every wave reads it for itself (11 bits are the exponent and two more: with 8, most weights of a
// wave fall into a few bins, and their additions wait for one another).  Of tokens with this very key those in the highest slots leave.
// Free slots below n and tokens that stay above it are as many as one another; both are listed in ascending order, at places that come from a table of how many
// each 64 slots have.  Keys are in LDS, 16 to a thread (longer sequences are gone through again for every step).  What bounds it at the size of a decoding step is how many
// instructions are fetched for the first time: with the keys in registers, and every loop over them written out, 1040 tokens took 19 us.
// Beyond 16384 tokens each of the five sweeps (three histograms, places, what stays) reads the weights from memory again, and one CU does it: one sequence of 65536 cut down to 8192, k8
// d = 128, 122 us a call, of 131072 221 (what has to be read and written takes 12 and 14).
// Few moves (e.here) are made by the same workgroup.  64 sequences of 1040 tokens, k8 d = 128, quantised, 16 leave: 13 us with the moves; 8 prompts of 500 to 16384 cut down to 2048: 25 us and 13 of
// evict_move_kernel (3.9 TB/s).
constexpr int kSelectItems = 16, kSelectPasses = 3, kSelectBins = 2048;
__device__ __forceinline__ int select_bin(uint32_t digit) { return (int)(digit + (digit >> 5)); }
template <int THREADS>
struct SelectLds {
    uint32_t key[kSelectItems * THREADS];
    int bins[kSelectPasses][kSelectBins + kSelectBins / 32];  // (a lane reads 32 in a row: a word of padding behind them keeps the lanes on different banks)
    int table[kSelectItems * THREADS / 64 + 1];  // places, and behind them how many there are
    int from[kEvictHere], to[kEvictHere];
};
template <typename U, int THREADS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(EvictParams e, int units, int lanes, int value_bytes) {
    constexpr int W = THREADS / 64, kEntries = kSelectItems * W, kChunk = kSelectItems * THREADS;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    SelectLds<THREADS>& lds = *reinterpret_cast<SelectLds<THREADS>*>(smem);
    const int bk = blockIdx.x, b = bk / e.p.kv_heads, h = bk % e.p.kv_heads, tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    EvictSequence q;
    q.init(e, b, h);
    const int leave = q.len - q.n;
    if (h == 0 && tid == 0) e.new_lens[b] = q.n;
    // weights and positions of slots s0 .. end - 1, four of a thread on the way together (so none behind a condition): use(slot, weight, position)
    auto each = [&](int s0, int end, auto use) {
#pragma unroll 1
        for (int s = s0 + tid; s < end; s += 4 * THREADS) {
            float weight[4];
            int32_t pos[4] = {0, 0, 0, 0};
#pragma unroll
            for (int y = 0; y < 4; ++y) weight[y] = q.weight[min(s + y * THREADS, end - 1)];
            if (q.kept > 0) {
#pragma unroll
                for (int y = 0; y < 4; ++y) pos[y] = q.pos[min(s + y * THREADS, q.kept - 1)];
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int slot = s + y * THREADS;
                if (slot < end) use(slot, weight[y], slot < q.kept ? (long)pos[y] : q.seen - q.len + slot);
            }
        }
    };
    auto load = [&](int s0, int end) { each(s0, end, [&](int slot, float weight, long at) { lds.key[slot - s0] = q.key(e, weight, at); }); };
    // places of flags of slots s0 .. end - 1 (up to 16 bits each of two kinds): count(slot) says which of them a slot has
    auto places = [&](int s0, int end, auto count) {
        __syncthreads();  // (the table may still be read)
        for (int x = 0; s0 + x * THREADS < end; ++x) {
            const int slot = s0 + x * THREADS + tid, c = slot < end ? count(slot) : 0;
            const int own = __builtin_popcountl(__builtin_amdgcn_ballot_w64(c & 1)) | __builtin_popcountl(__builtin_amdgcn_ballot_w64(c & 0x10000)) << 16;
            if (lane == 0) lds.table[x * W + w] = own;
        }
        __syncthreads();
        if (w == 0) {
            const int entries = (end - s0 + THREADS - 1) / THREADS * W;
            int before = 0;
            for (int x = lane; x - lane < entries; x += 64) {
                const int own = x < entries ? lds.table[x] : 0;
                const int upto = wave_sums(own);
                if (x < entries) lds.table[x] = before + upto - own;
                before += __builtin_amdgcn_readlane(upto, 63);
            }
            if (lane == 0) lds.table[kEntries] = before;
        }
        __syncthreads();
    };
    const unsigned long lower = (1ul << lane) - 1ul;

    uint32_t last = 0;                // the key of the last token that leaves
    int rank = leave - 1, equal = 0;  // its place among the keys that agree in the bits found; how many tokens have this key
    if (leave > 0) {
        for (int x = tid; x < (int)(sizeof(lds.bins) / sizeof(int)); x += THREADS) lds.bins[0][x] = 0;
        if (q.len <= kChunk) load(0, q.len);
        __syncthreads();
#pragma unroll 1
        for (int pass = 0; pass < kSelectPasses; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t found = pass == 0 ? 0u : pass == 1 ? ~0u << 21 : ~0u << 10, digits = pass == 2 ? 1023u : 2047u;
            int* bins = lds.bins[pass];
            for (int s0 = 0; s0 < q.len; s0 += kChunk) {
                const int end = min(q.len, s0 + kChunk);
                if (q.len > kChunk) load(s0, end);  // (every thread reads back its own)
                for (int slot = s0 + tid; slot < end; slot += THREADS) {
                    const uint32_t k = lds.key[slot - s0];
                    if (((k ^ last) & found) == 0) atomicAdd(&bins[select_bin((k >> shift) & digits)], 1);
                }
            }
            __syncthreads();
            int sum = 0;
#pragma unroll 8
            for (int x = 0; x < 32; ++x) sum += bins[33 * lane + x];
            const int upto = wave_sums(sum), who = __builtin_ctzl(__builtin_amdgcn_ballot_w64(upto > rank));  // (all keys together are more than `rank`)
            rank -= __builtin_amdgcn_readlane(upto - sum, who);
            // the 32 bins of that lane, one to a lane
            const int own = lane < 32 ? bins[33 * who + lane] : 0, within = wave_sums(own);
            const int at = __builtin_ctzl(__builtin_amdgcn_ballot_w64(within > rank));
            last |= (uint32_t)(32 * who + at) << shift;
            rank -= __builtin_amdgcn_readlane(within - own, at);
            equal = __builtin_amdgcn_readlane(own, at);
        }
    }
    const int stay_equal = leave > 0 ? equal - (rank + 1) : 0;  // of the tokens with the last key so many stay, in the lowest slots
    // what stays where it is, is written out; in place, positions of the tokens that had none
    const bool in_place = q.weight_out == q.weight && q.pos_out == q.pos;
    const int copied = !in_place ? 0 : q.pos_out ? q.kept : q.n;
    int equals = 0, free = 0, come = 0;
    for (int s0 = 0; s0 < q.len; s0 += kChunk) {
        const int end = min(q.len, s0 + kChunk);
        if (leave > 0) {
            if (q.len > kChunk) load(s0, end);
            if (stay_equal > 0) {  // tokens with the last key that stay get one above all others
                places(s0, end, [&](int slot) { return lds.key[slot - s0] == last ? 1 : 0; });
                for (int x = 0; s0 + x * THREADS < end; ++x) {
                    const int slot = s0 + x * THREADS + tid;
                    const bool is = slot < end && lds.key[slot - s0] == last;
                    const int at = equals + lds.table[x * W + w] + __builtin_popcountl(__builtin_amdgcn_ballot_w64(is) & lower);
                    if (is && at < stay_equal) lds.key[slot - s0] = ~0u;
                }
                equals += lds.table[kEntries];
            }
            auto goes = [&](int slot) { return lds.key[slot - s0] <= last; };
            places(s0, end, [&](int slot) { return slot < q.n ? (goes(slot) ? 1 : 0) : goes(slot) ? 0 : 0x10000; });
            for (int x = 0; s0 + x * THREADS < end; ++x) {
                const int slot = s0 + x * THREADS + tid;
                const bool g = slot < end && goes(slot), f = g && slot < q.n, m = slot < end && slot >= q.n && !g;
                const int at = lds.table[x * W + w];
                const int fi = free + (at & 0xffff) + __builtin_popcountl(__builtin_amdgcn_ballot_w64(f) & lower);
                const int mi = come + (at >> 16) + __builtin_popcountl(__builtin_amdgcn_ballot_w64(m) & lower);
                if (f && fi < e.cap) (e.here ? lds.to : e.to + (long)bk * e.cap)[fi] = slot;
                if (m && mi < e.cap) (e.here ? lds.from : e.from + (long)bk * e.cap)[mi] = slot;
            }
            const int all = lds.table[kEntries];
            free += all & 0xffff;
            come += all >> 16;
        }
        if (max(s0, copied) < min(end, q.n))
            each(max(s0, copied), min(end, q.n), [&](int slot, float weight, long at) {
                if (leave > 0 && lds.key[slot - s0] <= last) return;
                q.weight_out[slot] = weight;
                if (q.pos_out) q.pos_out[slot] = (int32_t)at;
            });
        if (q.len > kChunk) __syncthreads();  // (the keys of the next slots come)
    }
    const int count = min(min(free, come), e.cap);
    if (e.here) {
        __syncthreads();
        evict_rows<U>(e, q, b, h, lds.from, lds.to, count, 0, THREADS / lanes * kMoveRows, THREADS, units, lanes, value_bytes);
    } else if (tid == 0) {
        e.count[bk] = count;
    }
}

template <typename U>
__global__ void __launch_bounds__(kThreads) evict_move_kernel(EvictParams e, int blocks, int units, int lanes, int value_bytes) {
    const int bk = blockIdx.x / blocks, b = bk / e.p.kv_heads, h = bk % e.p.kv_heads, count = e.count[bk], rows = kThreads / lanes * kMoveRows;
    EvictSequence q;
    q.init(e, b, h);
    evict_rows<U>(e, q, b, h, e.from + (long)bk * e.cap, e.to + (long)bk * e.cap, count, blockIdx.x % blocks * rows, blocks * rows, kThreads, units, lanes, value_bytes);
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
    hipError_t error = hipSuccess;
    with_unit(unit, [&](auto u) {
        typedef decltype(u) U;
        auto select = [&](auto threads) {
            constexpr int T = decltype(threads)::value;
            error = allow_lds(evict_select_kernel<U, T>, sizeof(SelectLds<T>));
            if (error == hipSuccess)
                hipLaunchKernelGGL((evict_select_kernel<U, T>), dim3((unsigned)bk), dim3(T), sizeof(SelectLds<T>), stream, e, units, lanes, row_bytes / e.p.d);
        };
        if (e.p.max_len <= kSelectItems * 256) select(std::integral_constant<int, 256>{});
        else select(std::integral_constant<int, 1024>{});
        if (error != hipSuccess) return;
        if (e.cap > 0 && !e.here) {
            const int blocks = evict_blocks(bk, e.cap, kThreads / lanes * kMoveRows);
            hipLaunchKernelGGL(evict_move_kernel<U>, dim3((unsigned)(bk * blocks)), dim3(kThreads), 0, stream, e, blocks, units, lanes, row_bytes / e.p.d);
        }
    });
    return error != hipSuccess ? error : hipGetLastError();
}

}  // namespace attn
