// Trees of drafted tokens: which of them each sees, from the token that each follows; and their attention in 32-bit arithmetic (the kernels of
// attn_win_plain.hpp with the tiles and masks of a tree).
#include "attn_win_plain.hpp"

namespace attn {
namespace {

template <typename T, typename E, int DP>
__global__ void __launch_bounds__(kThreads, DP <= 96 ? 2 : 1) tree_plain_out_kernel(WinParams p) {
    win_plain_out<T, E, DP, true, true>(p, p.row_blocks);
}

// One workgroup per sequence.  A token's row of words is written from the last word down, as the way up its branch passes the tokens of each: the steps are
// reads of LDS that wait for one another, as many as the branch is long, and every word is written once, without a word of LDS for it.  A
// token that does not follow an earlier one of its sequence follows the context, so the way up always ends.
__global__ void __launch_bounds__(kThreads) tree_mask_kernel(WinParams p, const int32_t* parents, uint32_t* mask) {
    __shared__ int up[kMostDrafted];
    const int b = blockIdx.x;
    const int row0 = p.q_ptr ? min(max(p.q_ptr[b], 0), p.total_q) : b * p.n;
    const int count = min(p.q_ptr ? min(max(p.q_ptr[b + 1] - row0, 0), p.total_q - row0) : p.n, p.n), words = (p.n + 31) >> 5;
    for (int t = threadIdx.x; t < count; t += kThreads) {
        const int v = parents[row0 + t];
        up[t] = v < t ? max(v, -1) : -1;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < count; t += kThreads) {
        uint32_t* row = mask + (long)(row0 + t) * p.tree_stride;
        int at = t;
        for (int w = words - 1; w >= 0; --w) {
            uint32_t bits = 0;
            while (at >= 32 * w) {  // (at < 0: the context, below every word)
                bits |= 1u << (at & 31);
                at = up[at];
            }
            row[w] = bits;
        }
    }
}

template <typename T, typename E>
hipError_t fwd(const WinParams& p, hipStream_t stream) {
    return with_width(p.d, [&](auto width) {
        constexpr int DP = decltype(width)::value;
        hipLaunchKernelGGL((tree_plain_out_kernel<T, E, DP>), dim3((unsigned)((long)p.blocks * p.kv_heads), (unsigned)p.splits), dim3(kThreads), DP * 128 + 1024,
                           stream, p);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_tree_plain_fwd(bool is_bf16, bool fp8, const WinParams& p, hipStream_t stream) {
    if (!p.table || !p.tree) return hipErrorInvalidValue;
    if (fp8) return is_bf16 ? fwd<__bf16, uint8_t>(p, stream) : fwd<float, uint8_t>(p, stream);
    return fwd<float, float>(p, stream);
}
hipError_t launch_tree_mask(const WinParams& p, const int32_t* parents, uint32_t* mask, hipStream_t stream) {
    if (p.n > kMostDrafted) return hipErrorInvalidValue;
    hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)p.batch), dim3(kThreads), 0, stream, p, parents, mask);
    return hipGetLastError();
}

}  // namespace attn
