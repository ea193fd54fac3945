"""ctypes binding of libattn_mi355x.so: argument marshalling only.

Every function here has the name and meaning of the C entry point it wraps (see
include/attn_mi355x.h).  PyTorch supplies device memory and the current HIP stream; all
arithmetic runs in the library's kernels.  There is no CPU fallback: if the shared library
is missing, loading raises.
"""
import ctypes
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libattn_mi355x.so")

ATTN_OK, ATTN_ERR_INVALID_ARG, ATTN_ERR_UNSUPPORTED, ATTN_ERR_WORKSPACE, ATTN_ERR_DEVICE = range(5)
ATTN_F32, ATTN_BF16 = 0, 1
ATTN_CACHE_PLAIN, ATTN_CACHE_FP8 = 0, 1
(ATTN_BWD_AUTO, ATTN_BWD_TWO_KERNEL, ATTN_BWD_ONEPASS_K64, ATTN_BWD_ONEPASS_K128, ATTN_BWD_PART_DQ,
 ATTN_BWD_PART_DKDV, ATTN_BWD_FOUR_PHASE, ATTN_BWD_SPLIT_D) = range(8)

EXPORTS = ("attn_workspace_bytes", "attn_fwd", "attn_bwd", "attn_bwd_noalloc", "attn_bwd_blocksparse",
           "attn_wgrad_workspace_bytes", "attn_bwd_wgrad", "attn_blockmask_validate", "attn_mfma_ceiling",
           "attn_win_workspace_bytes", "attn_win_fwd", "attn_win_bwd", "attn_cache_write", "attn_cache_read",
           "attn_paged_workspace_bytes", "attn_paged_fwd", "attn_tree_mask", "attn_tree_workspace_bytes", "attn_tree_fwd", "attn_tree_commit",
           "attn_weigh_workspace_bytes", "attn_cache_weigh", "attn_evict_workspace_bytes", "attn_cache_evict", "attn_status_str")


class attn_desc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int32), ("heads", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("scale", ctypes.c_float), ("causal", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("bwd_tiling", ctypes.c_int32), ("stride_b", ctypes.c_int64),
                ("stride_h", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class attn_blockmask(ctypes.Structure):
    _fields_ = [("block", ctypes.c_int32), ("nblk", ctypes.c_int32),
                ("row_ptr", ctypes.c_void_p), ("col_idx", ctypes.c_void_p),
                ("col_ptr", ctypes.c_void_p), ("row_idx", ctypes.c_void_p), ("nmasks", ctypes.c_int32)]


class attn_win_desc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("batch", "heads", "kv_heads", "n", "d")] + [("scale", ctypes.c_float)] + \
               [(f, ctypes.c_int32) for f in ("window", "sinks", "dtype", "reserved")] + \
               [(f, ctypes.c_int64) for f in ("q_stride_b", "q_stride_h", "q_stride_n", "kv_stride_b", "kv_stride_h", "kv_stride_n")]


class attn_paged_desc(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("batch", "heads", "kv_heads", "d", "total_q", "max_q", "max_len", "page_size", "num_pages",
                                              "max_pages")] + [("scale", ctypes.c_float)] + \
               [(f, ctypes.c_int32) for f in ("window", "sinks", "dtype", "kind", "reserved")] + \
               [(f, ctypes.c_int64) for f in ("q_stride_n", "q_stride_h", "kv_stride_n", "kv_stride_h", "page_stride_p", "page_stride_h",
                                              "page_stride_n", "table_stride")]


class attn_cache(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("K", "V", "K_exp", "V_exp", "table", "lens", "q_ptr")]


class attn_weights(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("in_", "out")] + \
               [(f, ctypes.c_int64) for f in ("in_stride_b", "in_stride_h", "out_stride_b", "out_stride_h")] + \
               [("decay", ctypes.c_float), ("reserved", ctypes.c_int32)]


class attn_eviction(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("budget", "first", "recent", "reserved")] + \
               [(f, ctypes.c_void_p) for f in ("weight", "pos", "kept", "seen", "weight_out", "pos_out", "new_lens")] + \
               [(f, ctypes.c_int64) for f in ("stride_b", "stride_h", "out_stride_b", "out_stride_h")]


class AttnError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s" % (where, status_str(status)))


_lib = None


def lib():
    """The loaded shared library (raises OSError if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise OSError("libattn_mi355x.so is not built: run `python -m paper_2410_09397_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, dp, mp = ctypes.c_void_p, ctypes.POINTER(attn_desc), ctypes.POINTER(attn_blockmask)
        i32p = ctypes.POINTER(ctypes.c_int32)
        L.attn_workspace_bytes.restype = ctypes.c_size_t
        L.attn_workspace_bytes.argtypes = [dp, mp]
        L.attn_fwd.restype = ctypes.c_int
        L.attn_fwd.argtypes = [dp, mp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.attn_bwd.restype = ctypes.c_int
        L.attn_bwd.argtypes = [dp] + [vp] * 9 + [vp, ctypes.c_size_t, vp]
        L.attn_bwd_noalloc.restype = ctypes.c_int
        L.attn_bwd_noalloc.argtypes = [dp] + [vp] * 9 + [vp]
        L.attn_bwd_blocksparse.restype = ctypes.c_int
        L.attn_bwd_blocksparse.argtypes = [dp, mp] + [vp] * 9 + [vp, ctypes.c_size_t, vp]
        L.attn_wgrad_workspace_bytes.restype = ctypes.c_size_t
        L.attn_wgrad_workspace_bytes.argtypes = [dp]
        L.attn_bwd_wgrad.restype = ctypes.c_int
        L.attn_bwd_wgrad.argtypes = [dp] + [vp] * 7 + [vp, ctypes.c_size_t, vp]
        L.attn_blockmask_validate.restype = ctypes.c_int
        L.attn_blockmask_validate.argtypes = [ctypes.c_int32] * 4 + [i32p] * 4
        L.attn_mfma_ceiling.restype = ctypes.c_int
        L.attn_mfma_ceiling.argtypes = [ctypes.c_int32, ctypes.c_int32, vp, ctypes.POINTER(ctypes.c_double), vp]
        wp = pp = cp = vp  # descriptors as packed bytes or as the structures above
        L.attn_win_workspace_bytes.restype = L.attn_paged_workspace_bytes.restype = ctypes.c_size_t
        L.attn_win_workspace_bytes.argtypes = [wp]
        L.attn_paged_workspace_bytes.argtypes = [pp]
        L.attn_win_fwd.restype = L.attn_win_bwd.restype = ctypes.c_int
        L.attn_win_fwd.argtypes = [wp] + [vp] * 7
        L.attn_win_bwd.argtypes = [wp] + [vp] * 11 + [ctypes.c_size_t, vp]
        L.attn_cache_write.restype = L.attn_cache_read.restype = L.attn_paged_fwd.restype = ctypes.c_int
        L.attn_cache_write.argtypes = L.attn_cache_read.argtypes = [pp, cp, vp, vp, vp]
        L.attn_paged_fwd.argtypes = [pp, cp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.attn_tree_workspace_bytes.restype = L.attn_weigh_workspace_bytes.restype = L.attn_evict_workspace_bytes.restype = size
        L.attn_tree_workspace_bytes.argtypes = L.attn_weigh_workspace_bytes.argtypes = [pp]
        L.attn_evict_workspace_bytes.argtypes = [pp, i32]
        for fn in (L.attn_tree_mask, L.attn_tree_fwd, L.attn_tree_commit, L.attn_cache_weigh, L.attn_cache_evict):
            fn.restype = ctypes.c_int
        L.attn_tree_mask.argtypes = [i32, i32, i32, vp, vp, vp, i64, vp]
        L.attn_tree_fwd.argtypes = [pp, cp, vp, i64, vp, vp, vp, vp, size, vp]
        L.attn_tree_commit.argtypes = [pp, cp, vp, i64, vp, vp, vp]
        L.attn_cache_weigh.argtypes = [pp, cp, vp, vp, vp, vp, size, vp]
        L.attn_cache_evict.argtypes = [pp, cp, vp, vp, size, vp]
        L.attn_status_str.restype = ctypes.c_char_p
        L.attn_status_str.argtypes = [ctypes.c_int]
        _lib = L
    return _lib


def status_str(status):
    return lib().attn_status_str(int(status)).decode()


def csr_csc_from_dense(keep):
    """Host int32 arrays (row_ptr, col_idx, col_ptr, row_idx) of an [nblk, nblk] 0/1 matrix, or of a stack
    [nmasks, nblk, nblk] of them in the concatenated form of include/attn_mi355x.h (pointer arrays of
    nblk + 1 entries per mask that index the concatenated index arrays)."""
    keep = np.asarray(keep) != 0
    stack = keep[None] if keep.ndim == 2 else keep
    nblk = stack.shape[1]
    row_ptr, col_idx, col_ptr, row_idx = [], [], [], []
    start = 0
    for k in stack:
        rp = np.zeros(nblk + 1, np.int64)
        rp[1:] = np.cumsum(k.sum(1))
        cp = np.zeros(nblk + 1, np.int64)
        cp[1:] = np.cumsum(k.sum(0))
        row_ptr.append(rp + start)
        col_ptr.append(cp + start)
        col_idx.append(np.nonzero(k)[1])
        row_idx.append(np.nonzero(k.T)[1])
        start += int(rp[-1])
    cat = lambda parts: np.concatenate(parts).astype(np.int32)
    return cat(row_ptr), cat(col_idx), cat(col_ptr), cat(row_idx)


def attn_blockmask_validate(block, nblk, n, row_ptr, col_idx, col_ptr, row_idx, nmasks=1):
    """Status code of the host-side structural check of a block mask (numpy int32 arrays)."""
    i32p = ctypes.POINTER(ctypes.c_int32)
    arrs = [np.ascontiguousarray(a, dtype=np.int32) if a is not None else None
            for a in (row_ptr, col_idx, col_ptr, row_idx)]
    ptrs = [a.ctypes.data_as(i32p) if a is not None else None for a in arrs]
    return lib().attn_blockmask_validate(int(block), int(nblk), int(n), int(nmasks), *ptrs)


class BlockMask:
    """Device copies of a block mask in both compressed orientations.  `keep` is [nblk, nblk] (one
    pattern for all batches and heads) or [batch * heads, nblk, nblk] (one per pair)."""

    def __init__(self, keep, block, n, device="cuda"):
        import torch
        keep = np.asarray(keep)
        self.block, self.n = int(block), int(n)
        self.nblk = int(keep.shape[-1])
        self.nmasks = 1 if keep.ndim == 2 else int(keep.shape[0])
        self.host = csr_csc_from_dense(keep)
        st = attn_blockmask_validate(self.block, self.nblk, self.n, *self.host, nmasks=self.nmasks)
        if st != ATTN_OK:
            raise AttnError(st, "attn_blockmask_validate")
        self.dev = [torch.from_numpy(a).to(device) for a in self.host]
        self.c = attn_blockmask(self.block, self.nblk, *[t.data_ptr() for t in self.dev], self.nmasks)


def _desc(x, scale, causal, tiling=ATTN_BWD_AUTO):
    import torch
    if x.dim() != 4 or x.stride(3) != 1:
        raise ValueError("expected a [batch, heads, n, d] tensor with unit stride along d")
    dtype = x.dtype
    dt = ATTN_BF16 if dtype is torch.bfloat16 else {torch.float32: ATTN_F32}[dtype]
    b, h, n, d = x.shape
    sb, sh, sn, _ = x.stride()
    return attn_desc(b, h, n, d, float(scale), 1 if causal else 0, dt, int(tiling), sb, sh, sn)


# The smallest calls take about as long on the GPU as their marshalling here, so what is asked of torch is asked once per
# call: us of host time per call, before -> now (forward / backward / without allocation): 10.8 / 16.3 / 15.7 -> 7.0 / 11.5 / 11.4,
# of which a launch is about 2.5, with one in the forward and two in the backward.
def _same_layout(ref, *others):
    shape, strides, dtype, device = ref.shape, ref.stride(), ref.dtype, ref.device
    for t in others:
        if t.shape != shape or t.stride() != strides or t.dtype != dtype or t.device != device:
            raise ValueError("all [batch, heads, n, d] tensors must share shape, strides, dtype and device")


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    # the handle of torch.cuda.current_stream() without the object around it (3 us); the name is not a public one, and where
    # torch does not have it the object gives the handle
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(torch.cuda.current_device()) if raw is not None else torch.cuda.current_stream().cuda_stream


def attn_workspace_bytes(desc, mask=None):
    return lib().attn_workspace_bytes(ctypes.byref(desc), ctypes.byref(mask.c) if mask is not None else None)


def _workspace(desc, mask, workspace, device, stream=None):
    """The caller's workspace, or a fresh one.  A fresh one is allocated on the stream the kernels will
    run on: torch's allocator may hand a freed block to later work of the allocating stream only, so the
    block cannot be reused while these kernels still read it."""
    import torch
    if workspace is None:
        nbytes = max(attn_workspace_bytes(desc, mask), 256)
        if stream is not None:
            with torch.cuda.stream(stream):
                workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        else:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return workspace


def attn_fwd(Q, K, V, scale, causal=False, mask=None, stream=None, out=None, workspace=None):
    """O, LSE = forward(Q, K, V) on the GPU.  Q, K, V: cuda tensors [batch, heads, n, d]."""
    if out is None:
        import torch
        _same_layout(Q, K, V)
        out = torch.empty_like(Q), torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device)
    O, LSE = out[0], out[1]
    _same_layout(Q, K, V, O)
    desc = _desc(Q, scale, causal)
    if workspace is None:
        workspace = _workspace(desc, mask, None, Q.device, stream)
    st = lib().attn_fwd(ctypes.byref(desc), ctypes.byref(mask.c) if mask is not None else None,
                        Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), LSE.data_ptr(),
                        workspace.data_ptr(), workspace.numel(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_fwd")
    return O, LSE


def _bwd(name, Q, K, V, O, dO, LSE, scale, causal, mask, stream, out, workspace, tiling):
    import torch
    if out is None:
        _same_layout(Q, K, V, O, dO)
        out = torch.empty_like(Q), torch.empty_like(Q), torch.empty_like(Q)
    dQ, dK, dV = out
    _same_layout(Q, K, V, O, dO, dQ, dK, dV)
    desc = _desc(Q, scale, causal, tiling)
    if LSE.dtype != torch.float32 or not LSE.is_contiguous() or LSE.shape != Q.shape[:3]:
        raise ValueError("LSE must be a contiguous float32 [batch, heads, n] tensor")
    if workspace is None:
        workspace = _workspace(desc, mask, None, Q.device, stream)
    args = [Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), dO.data_ptr(), LSE.data_ptr(),
            dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(), workspace.numel(), _stream(stream)]
    if name == "attn_bwd":
        st = lib().attn_bwd(ctypes.byref(desc), *args)
    else:
        st = lib().attn_bwd_blocksparse(ctypes.byref(desc), ctypes.byref(mask.c), *args)
    if st != ATTN_OK:
        raise AttnError(st, name)
    return dQ, dK, dV


def attn_bwd(Q, K, V, O, dO, LSE, scale, causal=False, stream=None, out=None, workspace=None,
             tiling=ATTN_BWD_AUTO):
    """dQ, dK, dV from the forward's O and LSE (no block mask)."""
    return _bwd("attn_bwd", Q, K, V, O, dO, LSE, scale, causal, None, stream, out, workspace, tiling)


def attn_bwd_noalloc(Q, K, V, O, dO, LSE, scale, out, causal=False, stream=None, tiling=ATTN_BWD_AUTO):
    """attn_bwd with the library's fixed device scratch: the caller passes inputs and the outputs
    out = (dQ, dK, dV); nothing is allocated here or in the library."""
    import torch
    _same_layout(Q, K, V, O, dO, *out)
    desc = _desc(Q, scale, causal, tiling)
    if LSE.dtype != torch.float32 or not LSE.is_contiguous() or LSE.shape != Q.shape[:3]:
        raise ValueError("LSE must be a contiguous float32 [batch, heads, n] tensor")
    st = lib().attn_bwd_noalloc(ctypes.byref(desc), Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                                dO.data_ptr(), LSE.data_ptr(), out[0].data_ptr(), out[1].data_ptr(),
                                out[2].data_ptr(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_noalloc")
    return out


def attn_bwd_blocksparse(Q, K, V, O, dO, LSE, scale, mask, causal=False, stream=None, out=None, workspace=None,
                         tiling=ATTN_BWD_AUTO):
    """dQ, dK, dV under a BlockMask."""
    return _bwd("attn_bwd_blocksparse", Q, K, V, O, dO, LSE, scale, causal, mask, stream, out, workspace, tiling)


def attn_wgrad_workspace_bytes(desc):
    return lib().attn_wgrad_workspace_bytes(ctypes.byref(desc))


def attn_bwd_wgrad(A1, A2, A3, X, Y, dO, scale=1.0, causal=False, stream=None, out=None, workspace=None):
    """g = dL/dX [batch, heads, d, d] (float32) of the paper's loss: queries A1 X, keys A2, values A3 Y."""
    import torch
    _same_layout(A1, A2, A3, dO)
    _same_layout(X, Y)
    desc = _desc(A1, scale, causal)
    b, h, n, d = A1.shape
    if tuple(X.shape) != (b, h, d, d) or not X.is_contiguous() or not Y.is_contiguous() or X.dtype != A1.dtype:
        raise ValueError("X and Y must be contiguous [batch, heads, d, d] tensors of the inputs' dtype")
    g = out if out is not None else torch.empty((b, h, d, d), dtype=torch.float32, device=A1.device)
    if workspace is None:
        nbytes = max(attn_wgrad_workspace_bytes(desc), 256)
        if stream is not None:  # see _workspace
            with torch.cuda.stream(stream):
                workspace = torch.empty(nbytes, dtype=torch.uint8, device=A1.device)
        else:
            workspace = torch.empty(nbytes, dtype=torch.uint8, device=A1.device)
    st = lib().attn_bwd_wgrad(ctypes.byref(desc), A1.data_ptr(), A2.data_ptr(), A3.data_ptr(), X.data_ptr(),
                              Y.data_ptr(), dO.data_ptr(), g.data_ptr(), workspace.data_ptr(), workspace.numel(),
                              _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_bwd_wgrad")
    return g


def attn_mfma_ceiling(iters, operands=0, stream=None):
    """Launches the register-only MFMA loop (include/attn_mi355x.h).  Returns (clock, flops): a
    device float tensor that holds the shader clock in GHz once the stream is synchronised, and
    the number of floating-point operations of the launch."""
    import torch
    clock = torch.zeros(1, dtype=torch.float32, device="cuda")
    flops = ctypes.c_double(0.0)
    st = lib().attn_mfma_ceiling(int(iters), int(operands), clock.data_ptr(), ctypes.byref(flops),
                                 _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_mfma_ceiling")
    return clock, flops.value


# ------------------------------------------------------------------------- windowed attention with shared heads
# A call of a few tokens takes 6 us on the GPU, so its marshalling is kept short as well: descriptors are packed as bytes (the layouts of attn_win_desc,
# attn_paged_desc and attn_cache; half the time of filling the structures), and every tensor is asked once for its shape, strides and device.
_WIN_DESC = struct.Struct("@5if4i6q")
_PAGED_DESC = struct.Struct("@10if5i8q")
_CACHE = struct.Struct("@7P")
_WEIGHTS = struct.Struct("@2P4qfi")
_EVICTION = struct.Struct("@4i7P4q")


def _dtype(dtype):
    import torch
    if dtype is torch.bfloat16:
        return ATTN_BF16
    if dtype is torch.float32:
        return ATTN_F32
    raise ValueError("expected bfloat16 or float32 tensors, got %s" % dtype)


def _int32(name, t, count, device):
    """Device address of an int32 vector that the kernels index."""
    if t is None:
        return None
    import torch
    if t.dtype is not torch.int32 or t.shape != (count,) or not t.is_contiguous() or t.device != device:
        raise ValueError("%s must be a contiguous int32 tensor of %d entries on the device of the other tensors" % (name, count))
    return t.data_ptr()


def _made_on(stream, make):
    """make()'s tensors, allocated on the stream that the kernels will run on: memory that was freed on another one may still be in use there
    when they write to it, and theirs may be handed out there while they do."""
    if stream is None:
        return make()
    import torch
    with torch.cuda.stream(stream):
        return make()


def _empty_as(x):
    """An uninitialised tensor of x's shape and strides.  A view of a wider tensor (the queries of a fused projection) has gaps between its
    rows, and so has its image; views whose entries share memory have none."""
    import torch
    y = torch.empty_like(x)
    if y.stride() == x.stride():
        return y
    reach = 0  # of the axes with smaller strides
    for stride, size in sorted((a, n) for a, n in zip(x.stride(), x.shape) if n > 1):
        if stride <= reach:
            raise ValueError("expected a tensor whose entries do not share memory, got strides %s of shape %s" % (x.stride(), tuple(x.shape)))
        reach += stride * (size - 1)
    return torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device)


def _scratch(nbytes, device, stream):
    import torch
    return _made_on(stream, lambda: torch.empty(nbytes, dtype=torch.uint8, device=device))


def _on_gpu(x):
    if not x.is_cuda:  # (the kernels would be given a host address)
        raise ValueError("expected tensors on a GPU, got %s" % x.device)


def _check_workspace(workspace, device):
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError("the workspace must be a contiguous tensor on the device of the other tensors")


def _win_desc(Q, K, scale, window, sinks):
    if Q.dim() != 4 or K.dim() != 4:
        raise ValueError("expected [batch, heads, n, d] tensors")
    (b, h, n, d), (kb, kh, kn, kd), dtype = Q.shape, K.shape, Q.dtype
    (qsb, qsh, qsn, qsd), (ksb, ksh, ksn, ksd) = Q.stride(), K.stride()
    if qsd != 1 or ksd != 1:
        raise ValueError("expected unit stride along d")
    if (kb, kn, kd) != (b, n, d) or K.dtype != dtype or K.device != Q.device:
        raise ValueError("Q and K must share batch, n, d, dtype and device")
    _on_gpu(Q)
    return _WIN_DESC.pack(b, h, kh, n, d, scale, window, sinks, _dtype(dtype), 0, qsb, qsh, qsn, ksb, ksh, ksn)


def _as_argument(desc):
    return desc if isinstance(desc, bytes) else ctypes.byref(desc)


def attn_win_workspace_bytes(desc):
    return lib().attn_win_workspace_bytes(_as_argument(desc))


def attn_win_fwd(Q, K, V, scale, window=0, sinks=0, lens=None, stream=None, out=None):
    """O, LSE of causal attention in which a query sees itself, the window - 1 keys in front of it (window = 0: all of them) and the
    first `sinks` keys.  Q: [batch, heads, n, d]; K, V: [batch, kv_heads, n, d], heads a multiple of kv_heads; lens: the
    sequences' lengths (int32 [batch]), rows from there on are padding.  Q, K and V may be views of one wider tensor; O has Q's strides."""
    desc = _win_desc(Q, K, scale, window, sinks)
    _same_layout(K, V)
    if out is None:
        import torch
        O, LSE = _made_on(stream, lambda: (_empty_as(Q), torch.empty(Q.shape[:3], dtype=torch.float32, device=Q.device)))
    else:
        O, LSE = out
        _same_layout(Q, O)
        _check_lse(LSE, Q)
    st = lib().attn_win_fwd(desc, _int32("lens", lens, Q.shape[0], Q.device), Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                            LSE.data_ptr(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_win_fwd")
    return O, LSE


def _check_lse(LSE, Q):
    import torch
    if LSE.dtype != torch.float32 or not LSE.is_contiguous() or LSE.shape != Q.shape[:-1] or LSE.device != Q.device:
        raise ValueError("LSE must be a contiguous float32 tensor of the queries' shape without d")


def attn_win_bwd(Q, K, V, O, dO, LSE, scale, window=0, sinks=0, lens=None, stream=None, out=None, workspace=None):
    """dQ, dK, dV of attn_win_fwd from its O and LSE; dK and dV are sums over the query heads that share a key head.  O, dO and dQ have Q's
    strides, V, dK and dV those of K."""
    desc = _win_desc(Q, K, scale, window, sinks)
    if out is None:
        out = _made_on(stream, lambda: (_empty_as(Q), _empty_as(K), _empty_as(K)))
    dQ, dK, dV = out
    _same_layout(Q, O, dO, dQ)
    _same_layout(K, V, dK, dV)
    _check_lse(LSE, Q)
    if workspace is None:
        workspace = _scratch(max(attn_win_workspace_bytes(desc), 256), Q.device, stream)
    else:
        _check_workspace(workspace, Q.device)
    st = lib().attn_win_bwd(desc, _int32("lens", lens, Q.shape[0], Q.device), Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(),
                            dO.data_ptr(), LSE.data_ptr(), dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), workspace.data_ptr(),
                            workspace.numel(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_win_bwd")
    if Q.shape[1] == 0:  # nothing is launched: keys that no head reads
        _made_on(stream, lambda: (dK.zero_(), dV.zero_()))
    return dQ, dK, dV


# ----------------------------------------------------------------------------------------------- the paged cache
def attn_cache_pages(num_pages, kv_heads, page_size, d, dtype, device="cuda"):
    """K_pages, V_pages, K_exp, V_exp of an empty cache [num_pages, kv_heads, page_size, d]; dtype torch.float8_e4m3fn: quantised, else the
    type of the keys and values, and no exponents (None)."""
    import torch
    K, V = (torch.zeros(num_pages, kv_heads, page_size, d, dtype=dtype, device=device) for _ in range(2))
    if dtype is not torch.float8_e4m3fn:
        return K, V, None, None
    return K, V, *(torch.full((num_pages, kv_heads, page_size), 127, dtype=torch.uint8, device=device) for _ in range(2))


def _paged(name, x, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, kv_rows, scale=1.0, window=0, sinks=0):
    """The descriptor and the cache structure of a call whose rows are x: [total, heads, d]; kv_rows: x has the pages' heads."""
    if x.dim() != 3 or K_pages.dim() != 4:
        raise ValueError("%s: expected rows [total, heads, d], pages [num_pages, kv_heads, page_size, d] and a table [batch, pages]" % name)
    (total, h, dx), (sn, sh, sd) = x.shape, x.stride()
    if sd != 1:
        raise ValueError("%s: expected unit stride along d" % name)
    if dx != K_pages.shape[3] or (kv_rows and h != K_pages.shape[1]):
        raise ValueError("%s: rows and pages must agree in d and in their heads" % name)
    return _on_pages(name, total, h, sn, sh, x.dtype, x.device, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, scale, window, sinks)


def _on_pages(name, total, h, sn, sh, dtype, device, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, scale=1.0, window=0, sinks=0):
    """The same for rows [total, h, d] with strides sn, sh, or for none (total 0 or strides of the pages' width)."""
    import torch
    if K_pages.dim() != 4 or table.dim() != 2:
        raise ValueError("%s: expected pages [num_pages, kv_heads, page_size, d] and a table [batch, pages]" % name)
    shape, strides, kind = K_pages.shape, K_pages.stride(), K_pages.dtype
    (num, kvh, page, d), (psp, psh, psn, psd) = shape, strides
    if psd != 1:
        raise ValueError("%s: expected unit stride along d" % name)
    if V_pages.shape != shape or V_pages.stride() != strides or V_pages.dtype != kind or V_pages.device != device or K_pages.device != device:
        raise ValueError("%s: K_pages and V_pages must share shape, strides, dtype and the rows' device" % name)
    fp8 = kind is torch.float8_e4m3fn
    if fp8:
        for e in (K_exp, V_exp):
            if e is None or e.dtype is not torch.uint8 or e.shape != shape[:3] or not e.is_contiguous() or e.device != device:
                raise ValueError("%s: quantised pages need contiguous uint8 exponents [num_pages, kv_heads, page_size]" % name)
    elif kind is not dtype:
        raise ValueError("%s: pages hold the rows' type, or float8_e4m3fn with exponents" % name)
    batch, width = table.shape
    ts, t1 = table.stride()
    if table.dtype is not torch.int32 or t1 != 1 or table.device != device:
        raise ValueError("%s: the table must be an int32 tensor with unit stride along the pages" % name)
    if max_q is None:
        if q_ptr is not None:
            raise ValueError("%s: q_ptr needs max_q, the largest number of new tokens of a sequence" % name)
        if batch and total % batch:
            raise ValueError("%s: without q_ptr every sequence has the same number of rows" % name)
        max_q = total // batch if batch else 0
    _on_gpu(K_pages)
    desc = _PAGED_DESC.pack(batch, h, kvh, d, total, max_q, width * page if max_len is None else max_len, page, num, width, scale, window, sinks,
                            _dtype(dtype), ATTN_CACHE_FP8 if fp8 else ATTN_CACHE_PLAIN, 0, sn, sh, sn, sh, psp, psh, psn, ts)
    cache = _CACHE.pack(K_pages.data_ptr(), V_pages.data_ptr(), K_exp.data_ptr() if fp8 else 0, V_exp.data_ptr() if fp8 else 0,
                        table.data_ptr(), _int32("lens", lens, batch, device) or 0, _int32("q_ptr", q_ptr, batch + 1, device) or 0)
    return desc, cache


def attn_cache_write(K, V, K_pages, V_pages, table, lens, q_ptr=None, max_q=None, K_exp=None, V_exp=None, stream=None):
    """The new tokens' K and V ([total, kv_heads, d]) into the pages of their sequences, quantised where the pages are float8_e4m3fn.
    lens (int32 [batch]) counts the new tokens already; rows q_ptr[b] .. q_ptr[b + 1] - 1 belong to sequence b (None: the same number each)."""
    _same_layout(K, V)
    desc, cache = _paged("attn_cache_write", K, K_pages, V_pages, table, lens, q_ptr, max_q, None, K_exp, V_exp, True)
    st = lib().attn_cache_write(desc, cache, K.data_ptr(), V.data_ptr(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_cache_write")


def attn_cache_read(K_pages, V_pages, table, lens, dtype, total, q_ptr=None, max_q=None, K_exp=None, V_exp=None, stream=None, out=None):
    """K, V ([total, kv_heads, d]): the last tokens of every sequence, as many as q_ptr says (None: total / batch each)."""
    if K_pages.dim() != 4:
        raise ValueError("attn_cache_read: expected pages [num_pages, kv_heads, page_size, d]")
    shape = (total, K_pages.shape[1], K_pages.shape[3])
    if out is None:
        import torch
        device = K_pages.device
        out = _made_on(stream, lambda: (torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device)))
    K, V = out
    if K.shape != shape or K.dtype != dtype:
        raise ValueError("attn_cache_read: out must hold tensors [total, kv_heads, d] of the given type")
    _same_layout(K, V)
    desc, cache = _paged("attn_cache_read", K, K_pages, V_pages, table, lens, q_ptr, max_q, None, K_exp, V_exp, True)
    st = lib().attn_cache_read(desc, cache, K.data_ptr(), V.data_ptr(), _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_cache_read")
    return K, V


def attn_paged_workspace_bytes(desc):
    return lib().attn_paged_workspace_bytes(_as_argument(desc))


def attn_paged_fwd(Q, K_pages, V_pages, table, lens, scale, q_ptr=None, max_q=None, max_len=None, window=0, sinks=0, K_exp=None,
                   V_exp=None, stream=None, out=None, workspace=None):
    """O [total, heads, d], LSE [total, heads] of the new tokens Q [total, heads, d] over the paged cache that their keys and values have
    been written to.  max_len bounds the lengths (None: what the table can hold; a tighter bound gives better launches).  Q may be a view of a
    wider tensor; O has its strides."""
    desc, cache = _paged("attn_paged_fwd", Q, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, False, scale, window, sinks)
    if out is None:
        import torch
        O, LSE = _made_on(stream, lambda: (_empty_as(Q), torch.empty(Q.shape[:2], dtype=torch.float32, device=Q.device)))
    else:
        O, LSE = out
        _same_layout(Q, O)
        _check_lse(LSE, Q)
    where = size = 0
    if workspace is None:
        size = attn_paged_workspace_bytes(desc)
        if size > 256:  # (256: nothing is kept there)
            workspace = _scratch(size, Q.device, stream)
    else:
        _check_workspace(workspace, Q.device)
    if workspace is not None:
        where, size = workspace.data_ptr(), workspace.numel()
    st = lib().attn_paged_fwd(desc, cache, Q.data_ptr(), O.data_ptr(), LSE.data_ptr(), where, size, _stream(stream))
    if st != ATTN_OK:
        raise AttnError(st, "attn_paged_fwd")
    return O, LSE


# ------------------------------------------------------------------------- what stays in the cache: trees, eviction
def _stream_on(device, stream):
    """The handle of the stream to launch on: the current one of the tensors' device, which has to be the current device (launches and allocations are
    that one's), or the one that is given, of the same device."""
    import torch
    if device.type != "cuda":
        raise ValueError("expected tensors on a GPU, got %s" % device)
    here = torch.cuda.current_device()
    if device.index != here or (stream is not None and stream.device_index != here):
        raise ValueError("expected tensors, and a stream, of the current GPU (%d), got tensors on %s" % (here, device))
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # (as _stream)
    return raw(here) if raw is not None else torch.cuda.current_stream().cuda_stream


def _cache_only(name, total, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp):
    """The descriptor and the cache structure of a call on the pages alone."""
    import torch
    if K_pages.dim() != 4:
        raise ValueError("%s: expected pages [num_pages, kv_heads, page_size, d] and a table [batch, pages]" % name)
    kvh, d = K_pages.shape[1], K_pages.shape[3]
    dtype = torch.bfloat16 if K_pages.dtype is torch.float8_e4m3fn else K_pages.dtype
    return _on_pages(name, total, kvh, kvh * d, d, dtype, K_pages.device, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp)


def _check_mask(name, mask, total, max_q, device):
    import torch
    if mask.dtype is torch.int32 and mask.dim() == 2 and mask.device == device:
        (rows, words), (stride, unit) = mask.shape, mask.stride()
        if rows == total and words * 32 >= max_q and (unit == 1 or rows * words == 0):
            return mask.data_ptr(), stride
    raise ValueError("%s: the mask must be an int32 tensor [total, words] on the rows' device, 32 new tokens to a word, with unit stride along them" % name)


def _max_q(name, total, batch, q_ptr, max_q):
    if max_q is not None:
        return max_q
    if q_ptr is not None:
        raise ValueError("%s: q_ptr needs max_q, the largest number of new tokens of a sequence" % name)
    if batch and total % batch:
        raise ValueError("%s: without q_ptr every sequence has the same number of rows" % name)
    return total // batch if batch else 0


def attn_tree_mask(parents, max_q, q_ptr=None, stream=None, out=None):
    """int32 words [total, (max_q + 31) // 32]: bit u % 32 of word u // 32 of a row says that it is drafted token u of its sequence, or follows it.
    parents (int32 [total]): the number, among the drafted tokens of its sequence, of the one that a row follows; -1: it follows the context.  Rows
    q_ptr[b] .. q_ptr[b + 1] - 1 belong to sequence b (None: max_q rows each).  Rows of no sequence are not written."""
    import torch
    if parents.dim() != 1 or max_q < 0 or (q_ptr is not None and (q_ptr.dim() != 1 or q_ptr.shape[0] < 1)):
        raise ValueError("attn_tree_mask: expected parents [total], q_ptr [batch + 1] and max_q, the largest number of drafted tokens of a sequence")
    total, device, words = parents.shape[0], parents.device, -(-max_q // 32)
    if q_ptr is None and (total % max_q if max_q else total):
        raise ValueError("attn_tree_mask: without q_ptr every sequence has max_q rows")
    batch = q_ptr.shape[0] - 1 if q_ptr is not None else total // max_q if max_q else 0
    on = _stream_on(device, stream)
    parents_at, q_ptr_at = _int32("parents", parents, total, device), _int32("q_ptr", q_ptr, batch + 1, device)
    if out is None:
        out = _made_on(stream, lambda: torch.empty((total, words), dtype=torch.int32, device=device))
    st = lib().attn_tree_mask(batch, total, max_q, q_ptr_at, parents_at, *_check_mask("attn_tree_mask", out, total, max_q, device), on)
    if st != ATTN_OK:
        raise AttnError(st, "attn_tree_mask")
    return out


def attn_tree_workspace_bytes(desc):
    return lib().attn_tree_workspace_bytes(_as_argument(desc))


def attn_tree_fwd(Q, mask, K_pages, V_pages, table, lens, scale, q_ptr=None, max_q=None, max_len=None, window=0, sinks=0, K_exp=None,
                  V_exp=None, stream=None, out=None, workspace=None):
    """attn_paged_fwd for new tokens that are a tree of drafted ones: each sees the context and the new tokens of its row of the mask
    (attn_tree_mask's, or any bits).  O [total, heads, d], LSE [total, heads]."""
    desc, cache = _paged("attn_tree_fwd", Q, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, False, scale, window, sinks)
    on = _stream_on(Q.device, stream)
    bits = _check_mask("attn_tree_fwd", mask, Q.shape[0], _max_q("attn_tree_fwd", Q.shape[0], table.shape[0], q_ptr, max_q), Q.device)
    if out is None:
        import torch
        O, LSE = _made_on(stream, lambda: (_empty_as(Q), torch.empty(Q.shape[:2], dtype=torch.float32, device=Q.device)))
    else:
        O, LSE = out
        _same_layout(Q, O)
        _check_lse(LSE, Q)
    where = size = 0
    if workspace is None:
        size = attn_tree_workspace_bytes(desc)
        if size > 256:  # (256: nothing is kept there)
            workspace = _scratch(size, Q.device, stream)
    else:
        _check_workspace(workspace, Q.device)
    if workspace is not None:
        where, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    st = lib().attn_tree_fwd(desc, cache, *bits, Q.data_ptr(), O.data_ptr(), LSE.data_ptr(), where, size, on)
    if st != ATTN_OK:
        raise AttnError(st, "attn_tree_fwd")
    return O, LSE


def attn_tree_commit(mask, leaf, K_pages, V_pages, table, lens, q_ptr=None, max_q=None, K_exp=None, V_exp=None, stream=None, out=None):
    """Of the drafted tokens (the last of every sequence in the cache) those that row leaf[b] of the mask sees stay, moved up behind the context in
    their order.  leaf (int32 [batch]): a drafted token's number in its sequence, anything else: none stays.  Returns the lengths that are left."""
    import torch
    total, device, batch = mask.shape[0], K_pages.device, table.shape[0]
    desc, cache = _cache_only("attn_tree_commit", total, K_pages, V_pages, table, lens, q_ptr, max_q, None, K_exp, V_exp)
    on = _stream_on(device, stream)
    bits = _check_mask("attn_tree_commit", mask, total, _max_q("attn_tree_commit", total, batch, q_ptr, max_q), device)
    leaf_at = _int32("leaf", leaf, batch, device)
    if leaf_at is None:
        raise ValueError("attn_tree_commit: expected leaf, int32 [batch]")
    nothing = total == 0 or max_q == 0 or K_pages.shape[1] == 0  # nothing is launched: no drafted token, all of the context stays
    if out is None:
        out = _made_on(stream, lambda: lens.clone() if nothing else torch.empty_like(lens))
    elif nothing:
        _made_on(stream, lambda: out.copy_(lens))
    st = lib().attn_tree_commit(desc, cache, *bits, leaf_at, _int32("out", out, batch, device), on)
    if st != ATTN_OK:
        raise AttnError(st, "attn_tree_commit")
    return out


def _slots(name, what, x, dtype, batch, kv_heads, slots, device):
    """Address and strides of an array [batch, kv_heads, at least `slots`]."""
    if x.dtype is dtype and x.dim() == 3 and x.device == device:
        (b, h, n), (stride_b, stride_h, unit) = x.shape, x.stride()
        if b == batch and h == kv_heads and n >= slots and (unit == 1 or b * h * n == 0):
            return x.data_ptr(), stride_b, stride_h
    raise ValueError("%s: %s must be a %s tensor [batch, kv_heads, at least %d] on the pages' device with unit stride along the slots"
                     % (name, what, str(dtype).split(".")[-1], slots))


def attn_cache_weigh(Q, LSE, K_pages, V_pages, table, lens, scale, weight=None, decay=1.0, q_ptr=None, max_q=None, max_len=None, window=0, sinks=0,
                     K_exp=None, V_exp=None, stream=None, out=None, workspace=None):
    """Attention that the new tokens pay to every token of the cache: out[b, h, j] = decay * weight[b, h, j] + the sum of exp(scale q.k - LSE) over the
    new tokens that see slot j and the query heads of key head h; Q, LSE and the rest as attn_paged_fwd had or gave them.  New tokens start at zero,
    weight=None: all do.  weight, out: float32 [batch, kv_heads, at least max_len]; slots from a sequence's length on are left as they are.  out=None:
    `weight` itself is updated, or without one a new array is made, with zeros in those slots."""
    import torch
    desc, cache = _paged("attn_cache_weigh", Q, K_pages, V_pages, table, lens, q_ptr, max_q, max_len, K_exp, V_exp, False, scale, window, sinks)
    device, batch, kvh = Q.device, table.shape[0], K_pages.shape[1]
    on = _stream_on(device, stream)
    _check_lse(LSE, Q)
    slots = table.shape[1] * K_pages.shape[2] if max_len is None else max_len
    if out is None:
        out = weight if weight is not None else _made_on(stream, lambda: torch.zeros((batch, kvh, slots), dtype=torch.float32, device=device))
    to, to_b, to_h = _slots("attn_cache_weigh", "out", out, torch.float32, batch, kvh, slots, device)
    at, at_b, at_h = (0, 0, 0) if weight is None else _slots("attn_cache_weigh", "weight", weight, torch.float32, batch, kvh, slots, device)
    where = size = 0
    if workspace is None:
        size = attn_weigh_workspace_bytes(desc)
        if size > 256:  # (256: nothing is kept there)
            workspace = _scratch(size, device, stream)
    else:
        _check_workspace(workspace, device)
    if workspace is not None:
        where, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    st = lib().attn_cache_weigh(desc, cache, Q.data_ptr(), LSE.data_ptr(), _WEIGHTS.pack(at, to, at_b, at_h, to_b, to_h, decay, 0), where, size, on)
    if st != ATTN_OK:
        raise AttnError(st, "attn_cache_weigh")
    return out


def attn_weigh_workspace_bytes(desc):
    return lib().attn_weigh_workspace_bytes(_as_argument(desc))


def attn_evict_workspace_bytes(desc, budget):
    return lib().attn_evict_workspace_bytes(_as_argument(desc), budget)


def attn_cache_evict(weight, K_pages, V_pages, table, lens, budget, first=0, recent=0, pos=None, kept=None, seen=None, max_len=None, K_exp=None,
                     V_exp=None, stream=None, out=None, workspace=None):
    """Every key head of a sequence of more than `budget` tokens keeps `budget` of them: those at positions below `first`, the `recent` latest, and those
    with the largest weights.  Kept tokens in slots from `budget` on move into the free ones below (so a
    page of a sequence that is cut down belongs to it alone).  max_len: a bound on the lengths (None: all of the table's pages); one at most 64
    above the budget makes a call twice as fast, as few moves need one launch.  weight: float32 [batch, kv_heads, at least max_len];
    pos: the same in int32, positions of the tokens in slots below kept[b] (int32 [batch], the lengths of the last eviction); later slots hold the latest
    tokens of seen[b] (int32 [batch]; None: lens).  Returns weight, pos, the new lengths; out: where to put them (None: weight and pos
    themselves).  Without pos, slots are positions, as they are until the first eviction, and pos comes back as None unless `out` has one."""
    import torch
    name, device, batch, kvh = "attn_cache_evict", K_pages.device, table.shape[0], K_pages.shape[1]
    desc, cache = _cache_only(name, 0, K_pages, V_pages, table, lens, None, 0, max_len, K_exp, V_exp)
    on = _stream_on(device, stream)
    slots = table.shape[1] * K_pages.shape[2] if max_len is None else max_len
    if out is None:
        out = weight, pos, _made_on(stream, lambda: torch.empty_like(lens))
    weight_out, pos_out, new_lens = out
    at, at_b, at_h = _slots(name, "weight", weight, torch.float32, batch, kvh, slots, device)
    to, to_b, to_h = _slots(name, "weight's out", weight_out, torch.float32, batch, kvh, min(slots, budget), device)
    pos_at = pos_to = 0
    if pos is not None:
        pos_at, pos_b, pos_h = _slots(name, "pos", pos, torch.int32, batch, kvh, slots, device)
        if pos_b != at_b or pos_h != at_h or pos_out is None:
            raise ValueError("%s: pos must have weight's strides, and a place to go to" % name)
    if pos_out is not None:
        pos_to, pos_b, pos_h = _slots(name, "pos' out", pos_out, torch.int32, batch, kvh, min(slots, budget), device)
        if pos_b != to_b or pos_h != to_h:
            raise ValueError("%s: what weight and pos come out in must share strides" % name)
    lens_to = _int32("the new lengths", new_lens, batch, device)
    if lens_to is None:
        raise ValueError("%s: out must have a place for the new lengths" % name)
    where = size = 0
    if workspace is None:
        size = attn_evict_workspace_bytes(desc, budget)
        if size > 256:  # (256: nothing is kept there)
            workspace = _scratch(size, device, stream)
    else:
        _check_workspace(workspace, device)
    if workspace is not None:
        where, size = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    args = _EVICTION.pack(budget, first, recent, 0, at, pos_at, _int32("kept", kept, batch, device) or 0, _int32("seen", seen, batch, device) or 0,
                          to, pos_to, lens_to, at_b, at_h, to_b, to_h)
    st = lib().attn_cache_evict(desc, cache, args, where, size, on)
    if st != ATTN_OK:
        raise AttnError(st, name)
    if kvh == 0 or slots == 0:  # nothing is launched
        _made_on(stream, lambda: new_lens.copy_(lens.clamp(0, min(budget, slots))))
    return out
