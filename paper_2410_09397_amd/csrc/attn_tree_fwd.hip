// Attention of a tree of drafted tokens over the paged cache, bf16: the kernels of attn_win_fwd.hpp with the tiles and masks of a tree (Sight<BC, true>).
//
// The last tokens of a sequence are alternatives for what comes next: each sees the context and those in front of it on its own branch, so that
// one pass answers all branches.  The context is read as for any new tokens, once for a block of rows (tokens times heads of a group).  Behind it
// the drafted tokens are tiles of their own that start with the first of them: a tile of the context needs one comparison of positions for all of a
// wave's rows, and in a tile of drafted tokens 32 bits of a row's mask are 32 keys, read where the tile is (a tree has one or two such tiles).
//
// As in attn_win_fwd.hip the weights are rounded to bf16 for the product with V, so that it runs on the bf16 matrix pipe straight from the accumulators of the first product; scores,
// maxima, sums and O are 32 bits wide.  With the rounding of O itself that is 2.2e-3 to 2.4e-3 of the norm from 64 bits, of which O's own is 1.65e-3.
#include "attn_win_fwd.hpp"

namespace attn {
namespace {

// More than 64 rows (tree_rows says why 128 of them).  As without a tree the softmax and the waits of a tile bound it, not memory: 64 drafted tokens, h32 k8 d = 128, of one sequence of
// 65536 85 us (3.2 TB/s, 810 TFLOP/s), of 16 of 100 to 8192, quantised, 64 us (512 workgroups, the longest 22 tiles and the mean 16; 72 us where the caches are cold).  A window of 1024
// with 4 sinks leaves 11 of their 32 GFLOP: 49 us a call for 77.
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) tree_out_kernel(WinParams p) {
    win_out<D, SRC, 1, PAD, true>(p, p.row_blocks);
}
// 17 to 64 rows.  The latency of a launch and of few tiles: 15 drafted tokens of 333, h16 k4 d = 64, 9 us.  8 drafted tokens of 16 sequences of 100 to 8192, h32 k8 d = 128: a call
// takes 34 us quantised (68 MB), 48 not (133 MB, 2.8 TB/s).
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__((64 * kFewWaves<D, SRC>), (D == 256 ? 1 : 2)) tree_few_kernel(WinParams p) {
    win_few<D, SRC, PAD, true>(p);
}
// At most 16 rows.  (Padded rows of 65 to 127 columns: the masks' registers do not fit beside the tile's with three workgroups on a CU)
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads, (D == 128 && PAD ? 2 : kOnePerCu<D, SRC>)) tree_one_kernel(WinParams p) {
    win_one<D, SRC, PAD, true>(p);
}

template <int D, int SRC, bool PAD>
hipError_t launch_from(int rows, long groups, const WinParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)groups);
    auto run = [&](auto kernel, int lds, int threads) {
        const hipError_t e = allow_lds(kernel, lds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, stream, p);
        return hipGetLastError();
    };
    if (rows == 16) return run(tree_one_kernel<D, SRC, PAD>, kOneLds<D, SRC>, kThreads);
    if (rows == 32) return run(tree_few_kernel<D, SRC, PAD>, kFewLds<D, SRC>, 64 * kFewWaves<D, SRC>);
    return run(tree_out_kernel<D, SRC, PAD>, 4 * 64 * D * 2, kThreads);
}
template <int D>
hipError_t launch(bool fp8, int rows, long grid, const WinParams& p, hipStream_t stream) {
    if (fp8) return launch_from<D, kCodes, false>(rows, grid, p, stream);
    return p.d < D ? launch_from<D, kPages, true>(rows, grid, p, stream) : launch_from<D, kPages, false>(rows, grid, p, stream);
}

}  // namespace

hipError_t launch_tree_fwd(bool fp8, int rows, long grid, const WinParams& p, hipStream_t stream) {
    if (!tree_rows_exist(true, rows) || !p.table || !p.tree || (fp8 && p.d != 64 && p.d != 128 && p.d != 256)) return hipErrorInvalidValue;
    return p.d <= 64 ? launch<64>(fp8, rows, grid, p, stream) : p.d <= 128 ? launch<128>(fp8, rows, grid, p, stream) : launch<256>(fp8, rows, grid, p, stream);
}

}  // namespace attn
