// Windowed attention, forward, bf16: over tensors, bf16 pages or (d in {64, 128, 256}) quantised pages.  Kernels have widths of 64, 128 and 256
// columns; rows of another d are padded with zeros on their way into LDS and registers (PAD).
//
//   win_out_kernel  128 rows per workgroup (rows r = t * group + head of the group: see attn_window.hpp), 64-key tiles shared by its
//                   four waves.  Many rows: a prompt, a chunk, training.  SPLIT = 2: 64 rows, two waves for 32 of them with a key half
//                   of every tile each, where blocks of 128 would leave the chip half idle
//   win_few_kernel  32 rows per workgroup, whose waves take 32-key tiles in turn, each with LDS and softmax state of its own, and meet at
//                   the end.  A few tokens of a sequence
//   win_one_kernel  the same with 16 rows.  Single tokens, where the time is that of the keys' way from memory
// Each can share the keys of a row block out over workgroups (p.splits), whose sums win_join_kernel brings together.
//
// Per tile: S^T = K Q^T (lane <-> query), P^T = exp2(S^T - m) with a running reference m, O^T += V^T P^T, with V^T from transposing LDS
// reads and P^T straight from the accumulators.  P is rounded to bf16 for the second product (2^-9 of each weight; O is rounded as far
// when it is stored); scores, m, l and O are fp32.  At the head dimensions that are padded this is a choice: the forward without a window keeps P in
// 32 bits there (attn_stream.hip).  Distance from 64 bits over the norm at d = 24 to 248: O 2.0e-3 against 1.6e-3, gradients 2.4e-3 against 1.7e-3.  Windowed
// kernels of 32-bit arithmetic, which the padded ones replaced, took 156 us for a step of b2 h16 at d = 96 where these take 55 to 80.  us without
// a window, b2 h16 n1000 causal, 32-bit weights / here, forward and backward: d = 40 18 / 20, 60 / 44; d = 96 26 / 28, 74 / 67; d = 200 95 / 79, 272 / 178.
#include "attn_win_fwd.hpp"

namespace attn {
namespace {

template <int D, int SRC, int SPLIT, bool PAD>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 2 : 1) win_out_kernel(WinParams p, int row_blocks) {
    win_out<D, SRC, SPLIT, PAD, false>(p, row_blocks);
}
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__((64 * kFewWaves<D, SRC>), (D == 256 ? 1 : 2)) win_few_kernel(WinParams p) {
    win_few<D, SRC, PAD, false>(p);
}
template <int D, int SRC, bool PAD>
__global__ void __launch_bounds__(kThreads, (kOnePerCu<D, SRC>)) win_one_kernel(WinParams p) {
    win_one<D, SRC, PAD, false>(p);
}

template <int D, int SRC, int SPLIT, bool PAD>
hipError_t out(const WinParams& p, hipStream_t stream) {
    constexpr int lds = 4 * 64 * D * 2, BR = 128 / SPLIT;
    const hipError_t e = allow_lds(win_out_kernel<D, SRC, SPLIT, PAD>, lds);
    if (e != hipSuccess) return e;
    const int row_blocks = (int)(((long)p.n * p.group + BR - 1) / BR);
    const long blocks = SRC == kTensors ? (long)row_blocks * p.batch : p.blocks;
    hipLaunchKernelGGL((win_out_kernel<D, SRC, SPLIT, PAD>), dim3((unsigned)(blocks * p.kv_heads), (unsigned)p.splits), dim3(kThreads), lds, stream, p,
                       row_blocks);
    return hipGetLastError();
}
template <int D, int SRC, bool PAD>
hipError_t few(const WinParams& p, hipStream_t stream) {
    constexpr int lds = kFewLds<D, SRC>;
    const hipError_t e = allow_lds(win_few_kernel<D, SRC, PAD>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((win_few_kernel<D, SRC, PAD>), dim3((unsigned)((long)p.blocks * p.kv_heads), (unsigned)p.splits), dim3(64 * kFewWaves<D, SRC>), lds,
                       stream, p);
    return hipGetLastError();
}
template <int D, int SRC, bool PAD>
hipError_t one(const WinParams& p, hipStream_t stream) {
    constexpr int lds = kOneLds<D, SRC>;
    const hipError_t e = allow_lds(win_one_kernel<D, SRC, PAD>, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((win_one_kernel<D, SRC, PAD>), dim3((unsigned)((long)p.blocks * p.kv_heads), (unsigned)p.splits), dim3(kThreads), lds, stream, p);
    return hipGetLastError();
}
template <int D, int SRC, bool PAD>
hipError_t launch_from(int rows, const WinParams& p, hipStream_t stream) {
    if constexpr (SRC != kTensors) {
        if (rows == 16) return one<D, SRC, PAD>(p, stream);
        if (rows == 32) return few<D, SRC, PAD>(p, stream);
    }
    return rows == 64 ? out<D, SRC, 2, PAD>(p, stream) : out<D, SRC, 1, PAD>(p, stream);
}
template <int D>
hipError_t launch(bool fp8, int rows, const WinParams& p, hipStream_t stream) {
    if (fp8) return launch_from<D, kCodes, false>(rows, p, stream);
    if (p.d < D) return p.table ? launch_from<D, kPages, true>(rows, p, stream) : launch_from<D, kTensors, true>(rows, p, stream);
    return p.table ? launch_from<D, kPages, false>(rows, p, stream) : launch_from<D, kTensors, false>(rows, p, stream);
}

}  // namespace

hipError_t launch_win_fwd(bool fp8, int rows, const WinParams& p, hipStream_t stream) {
    if (fp8 && p.d != 64 && p.d != 128 && p.d != 256) return hipErrorInvalidValue;
    return p.d <= 64 ? launch<64>(fp8, rows, p, stream) : p.d <= 128 ? launch<128>(fp8, rows, p, stream) : launch<256>(fp8, rows, p, stream);
}

}  // namespace attn
