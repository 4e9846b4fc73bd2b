"""ctypes binding of libcyclotron_mm.so.  Same names as the C ABI (include/cyclotron_mm.h).

PyTorch appears here only as the owner of device memory and streams.  There is no
fallback: if the shared library is missing, the first call raises ImportError.
"""
from __future__ import annotations

import ctypes
import os

CYC_BF16_F32 = 0
CYC_I8_I32 = 1
CYC_OK = 0
CYC_ERR_WORKSPACE = 6

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libcyclotron_mm.so")


class cyc_cache(ctypes.Structure):
    """A cache of keys and values in pages and the sequences of a call (include/cyclotron_mm.h)."""
    _fields_ = [(name, ctypes.c_void_p) for name in ("K", "V", "table", "lengths", "starts")] + \
        [(name, ctypes.c_int64) for name in ("seqs", "pages", "max_pages", "kv_heads", "page", "d", "table_stride",
                                             "page_stride", "head_stride", "row_stride")]


def lib_path() -> str:
    return _LIB_PATH


def _load() -> ctypes.CDLL:
    if not os.path.exists(_LIB_PATH):
        raise ImportError(f"{_LIB_PATH} is not built; run `python -m paper_2511_09987_amd.build` "
                          "(needs hipcc, cross-compiles for gfx950)")
    lib = ctypes.CDLL(_LIB_PATH)
    i64, ptr, cint = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
    lib.cyc_recurrence_matmul.argtypes = [ptr, ptr, ptr, i64, i64, i64, cint, ptr]
    lib.cyc_recurrence_matmul.restype = cint
    lib.cyc_recurrence_matmul_noalloc.argtypes = [ptr, ptr, ptr, i64, i64, i64, cint, ptr]
    lib.cyc_recurrence_matmul_noalloc.restype = cint
    lib.cyc_recurrence_matmul_batched.argtypes = [ptr, ptr, ptr, i64, i64, i64, i64, i64, i64, i64, cint, ptr]
    lib.cyc_recurrence_matmul_batched.restype = cint
    lib.cyc_recurrence_matmul_in.argtypes = [ptr, ptr, ptr, i64, i64, i64, cint, ptr, i64, ptr]
    lib.cyc_recurrence_matmul_in.restype = cint
    lib.cyc_matmul_workspace.argtypes = [ptr, ptr, ptr, i64, i64, i64, cint]
    lib.cyc_matmul_workspace.restype = i64
    lib.cyc_recurrence_trsm.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, ptr]
    lib.cyc_recurrence_trsm.restype = cint
    lib.cyc_recurrence_cholesky.argtypes = [ptr, ptr, ptr, i64, i64, ptr]
    lib.cyc_recurrence_cholesky.restype = cint
    lib.cyc_recurrence_trsm_in.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_trsm_in.restype = cint
    lib.cyc_trsm_workspace.argtypes = [ptr, ptr, ptr, i64, i64, i64]
    lib.cyc_trsm_workspace.restype = i64
    lib.cyc_recurrence_cholesky_in.argtypes = [ptr, ptr, ptr, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_cholesky_in.restype = cint
    lib.cyc_cholesky_workspace.argtypes = [ptr, ptr, ptr, i64, i64]
    lib.cyc_cholesky_workspace.restype = i64
    lib.cyc_recurrence_attention.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, i64, ptr]
    lib.cyc_recurrence_attention.restype = cint
    lib.cyc_recurrence_attention_split.argtypes = [ptr, ptr, ptr, ptr, i64, i64, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_attention_split.restype = cint
    lib.cyc_attention_workspace.argtypes = [i64, i64, i64, i64]
    lib.cyc_attention_workspace.restype = i64
    strides, cache = ctypes.POINTER(i64), ctypes.POINTER(cyc_cache)
    lib.cyc_attention_window_workspace.argtypes = [i64] * 8
    lib.cyc_attention_window_workspace.restype = i64
    lib.cyc_recurrence_attention_window.argtypes = [ptr] * 5 + [i64] * 6 + [strides, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_attention_window.restype = cint
    lib.cyc_attention_window_grad_workspace.argtypes = [i64] * 8
    lib.cyc_attention_window_grad_workspace.restype = i64
    lib.cyc_recurrence_attention_window_grad.argtypes = [ptr] * 9 + [i64] * 6 + [strides, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_attention_window_grad.restype = cint
    lib.cyc_cache_append.argtypes = [ptr, ptr, cache, i64, strides, ptr]
    lib.cyc_cache_append.restype = cint
    lib.cyc_attention_paged_workspace.argtypes = [cache, i64, i64, i64, i64, i64]
    lib.cyc_attention_paged_workspace.restype = i64
    lib.cyc_recurrence_attention_paged.argtypes = [ptr, cache, ptr, i64, i64, strides, i64, i64, i64, ptr, i64, ptr]
    lib.cyc_recurrence_attention_paged.restype = cint
    lib.cyc_status_string.argtypes = [cint]
    lib.cyc_status_string.restype = ctypes.c_char_p
    lib.cyc_version.argtypes = []
    lib.cyc_version.restype = cint
    lib.cyc_kernel_name.argtypes = [ptr, ptr, ptr, i64, i64, i64, i64, i64, i64, i64, cint]
    lib.cyc_kernel_name.restype = ctypes.c_char_p
    lib.cyc_kernel_variant.argtypes = lib.cyc_kernel_name.argtypes
    lib.cyc_kernel_variant.restype = ctypes.c_char_p
    lib.cyc_force_kernel.argtypes = [ctypes.c_char_p]
    lib.cyc_force_kernel.restype = cint
    lib.cyc_diag_mfma_ceiling.argtypes = [cint, cint, i64, ptr, ctypes.POINTER(ctypes.c_double), ptr]
    lib.cyc_diag_mfma_ceiling.restype = cint
    lib.cyc_diag_issue_mix.argtypes = [cint, cint, cint, cint, i64, ptr, ctypes.POINTER(ctypes.c_double), ptr]
    lib.cyc_diag_issue_mix.restype = cint
    lib.cyc_diag_mfma_f32_tiles.argtypes = [ptr, ptr, ptr, ptr, i64, ptr]
    lib.cyc_diag_mfma_f32_tiles.restype = cint
    lib.cyc_diag_pivots.argtypes = [cint, i64, i64, ptr, ptr]
    lib.cyc_diag_pivots.restype = cint
    lib.cyc_diag_set_wait_limit.argtypes = [i64]
    lib.cyc_diag_set_wait_limit.restype = cint
    lib.cyc_diag_clock.argtypes = [ptr, i64, ptr]
    lib.cyc_diag_clock.restype = cint
    return lib


_cached = None


def _lib() -> ctypes.CDLL:
    """The loaded library; loading is deferred to first use so that the build module can be
    imported before the library exists.  Raises ImportError if it is not built."""
    global _cached
    if _cached is None:
        _cached = _load()
    return _cached


def _stream_handle(tensor, stream) -> int:
    """The handle of `stream`, or of the current stream of the tensor's device.  torch.cuda.current_stream builds an object
    around it, which takes 1.8 us of the 9 us that a small call spends on the host; asking for the handle takes 0.1."""
    import torch
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(tensor.device.index) if raw else torch.cuda.current_stream(tensor.device).cuda_stream


def _memory(wanted: int, tensor, stream):
    """`wanted` bytes from the allocator's pool of the stream that a call runs on, or None.  They go back to that pool when the
    caller drops them: whoever gets them next is ordered after the call.  Under capture they belong to the graph."""
    import torch
    try:
        if stream is None:
            return torch.empty(wanted, dtype=torch.uint8, device=tensor.device)
        if isinstance(stream, torch.cuda.Stream) and stream.device == tensor.device:
            with torch.cuda.stream(stream):
                return torch.empty(wanted, dtype=torch.uint8, device=tensor.device)
    except torch.OutOfMemoryError:
        pass
    return None


class CycError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(cyc_status_string(status))


def cyc_status_string(status: int) -> str:
    return _lib().cyc_status_string(int(status)).decode()


def cyc_version() -> int:
    return int(_lib().cyc_version())


def cyc_recurrence_matmul(A: int, B: int, C: int, M: int, K: int, N: int, dtype: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_matmul(A, B, C, M, K, N, dtype, stream))


def cyc_recurrence_matmul_noalloc(A: int, B: int, C: int, M: int, K: int, N: int, dtype: int, stream: int = 0) -> int:
    """Raw call of the allocation-free variant: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_matmul_noalloc(A, B, C, M, K, N, dtype, stream))


def cyc_recurrence_matmul_batched(A: int, B: int, C: int, batch: int, M: int, K: int, N: int,
                                  strideA: int, strideB: int, strideC: int, dtype: int, stream: int = 0) -> int:
    return int(_lib().cyc_recurrence_matmul_batched(A, B, C, batch, M, K, N, strideA, strideB, strideC,
                                                  dtype, stream))


def cyc_matmul_workspace(A: int, B: int, C: int, M: int, K: int, N: int, dtype: int) -> int:
    """Bytes of workspace that cyc_recurrence_matmul_in wants for this problem."""
    return int(_lib().cyc_matmul_workspace(A, B, C, M, K, N, dtype))


def cyc_recurrence_matmul_in(A: int, B: int, C: int, M: int, K: int, N: int, dtype: int, workspace: int, workspace_bytes: int,
                             stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_matmul_in(A, B, C, M, K, N, dtype, workspace, workspace_bytes, stream))


def cyc_recurrence_trsm(L: int, B: int, X: int, Xh: int, n: int, nrhs: int, nb: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_trsm(L, B, X, Xh, n, nrhs, nb, stream))


def cyc_trsm_workspace(L: int, X: int, Xh: int, n: int, nrhs: int, nb: int) -> int:
    """Bytes of workspace that cyc_recurrence_trsm_in wants for this system."""
    return int(_lib().cyc_trsm_workspace(L, X, Xh, n, nrhs, nb))


def cyc_recurrence_trsm_in(L: int, B: int, X: int, Xh: int, n: int, nrhs: int, nb: int, workspace: int, workspace_bytes: int,
                           stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_trsm_in(L, B, X, Xh, n, nrhs, nb, workspace, workspace_bytes, stream))


def cyc_recurrence_attention(Q: int, K: int, V: int, O: int, batch: int, N: int, M: int, d: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_attention(Q, K, V, O, batch, N, M, d, stream))


def cyc_attention_workspace(batch: int, N: int, M: int, d: int) -> int:
    """Bytes of workspace that cyc_recurrence_attention_split wants for these extents."""
    return int(_lib().cyc_attention_workspace(batch, N, M, d))


def cyc_recurrence_attention_split(Q: int, K: int, V: int, O: int, batch: int, N: int, M: int, d: int, workspace: int,
                                   workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_attention_split(Q, K, V, O, batch, N, M, d, workspace, workspace_bytes, stream))


def cyc_kernel_name(A: int, B: int, C: int, batch: int, M: int, K: int, N: int,
                    strideA: int, strideB: int, strideC: int, dtype: int) -> str:
    return _lib().cyc_kernel_name(A, B, C, batch, M, K, N, strideA, strideB, strideC, dtype).decode()


def cyc_kernel_variant(A: int, B: int, C: int, batch: int, M: int, K: int, N: int,
                       strideA: int, strideB: int, strideC: int, dtype: int) -> str:
    """The kernel that runs, where cyc_kernel_name says whose part of the dispatch the problem falls into."""
    return _lib().cyc_kernel_variant(A, B, C, batch, M, K, N, strideA, strideB, strideC, dtype).decode()


def cyc_force_kernel(name) -> int:
    """Force a kernel by name (None or "": back to the dispatcher); returns the cyc_status."""
    return int(_lib().cyc_force_kernel((name or "").encode()))


def cyc_diag_mfma_ceiling(dtype: int, mfma_shape: int, iters: int, sink: int, stream: int = 0):
    """Raw call; returns (cyc_status, operations of the launch)."""
    ops = ctypes.c_double(0.0)
    st = int(_lib().cyc_diag_mfma_ceiling(dtype, mfma_shape, iters, sink, ctypes.byref(ops), stream))
    return st, ops.value


def cyc_diag_issue_mix(mfma_shape: int, other_kind: int, others_per_round: int, waves_per_simd: int, iters: int, sink: int,
                       stream: int = 0):
    """Raw call; returns (cyc_status, MFMA operations of the launch)."""
    ops = ctypes.c_double(0.0)
    st = int(_lib().cyc_diag_issue_mix(mfma_shape, other_kind, others_per_round, waves_per_simd, iters, sink, ctypes.byref(ops), stream))
    return st, ops.value


def cyc_diag_mfma_f32_tiles(A: int, B: int, C: int, D: int, tiles: int, stream: int = 0) -> int:
    return int(_lib().cyc_diag_mfma_f32_tiles(A, B, C, D, tiles, stream))


def cyc_diag_pivots(what: int, first: int, count: int, bad: int, stream: int = 0) -> int:
    return int(_lib().cyc_diag_pivots(what, first, count, bad, stream))


def cyc_diag_set_wait_limit(polls: int) -> int:
    return int(_lib().cyc_diag_set_wait_limit(polls))


def cyc_diag_clock(out: int, microseconds: int, stream: int = 0) -> int:
    return int(_lib().cyc_diag_clock(out, microseconds, stream))


def recurrence_matmul(A, B, out=None, stream=None):
    """Tensor-level convenience: C = weight-stationary recurrence of A against B.

    A: (M,K) or (batch,M,K); B: (K,N) or (batch,K,N); contiguous CUDA tensors, both
    torch.bfloat16 (C float32) or both torch.int8 (C int32).  Only allocates C and, under
    stream capture, memory for the partial products of a long k, and forwards pointers to the
    C ABI on the current (or given) stream.  (Where no memory is to be had for those, fewer
    slices of k or none are taken, and the fp32 sums are added in another order.)
    """
    import torch
    if not (A.is_cuda and B.is_cuda):
        raise ValueError("A and B must be device tensors; there is no CPU path")
    if A.dtype != B.dtype or A.dtype not in (torch.bfloat16, torch.int8):
        raise ValueError("A and B must both be bfloat16 or both int8")
    if A.dim() != B.dim() or A.dim() not in (2, 3) or not (A.is_contiguous() and B.is_contiguous()):
        raise ValueError("A and B must be contiguous and both 2-D or both 3-D")
    dtype = CYC_BF16_F32 if A.dtype == torch.bfloat16 else CYC_I8_I32
    batch = A.shape[0] if A.dim() == 3 else 1
    M, K = A.shape[-2:]
    K2, N = B.shape[-2:]
    if K != K2 or (A.dim() == 3 and B.shape[0] != batch):
        raise ValueError(f"shape mismatch: A {tuple(A.shape)}, B {tuple(B.shape)}")
    cshape = (batch, M, N) if A.dim() == 3 else (M, N)
    cdtype = torch.float32 if dtype == CYC_BF16_F32 else torch.int32
    if out is None:
        out = torch.empty(cshape, dtype=cdtype, device=A.device)
    elif tuple(out.shape) != cshape or out.dtype != cdtype or not out.is_contiguous() or out.device != A.device:
        raise ValueError("out has the wrong shape, dtype, layout or device")
    s = _stream_handle(A, stream)
    if batch == 1:
        args = A.data_ptr(), B.data_ptr(), out.data_ptr(), M, K, N, dtype
        st = cyc_recurrence_matmul_in(*args, 0, 0, s)
        if st == CYC_ERR_WORKSPACE:               # under capture: partial sums in memory of the graph's own
            wanted = cyc_matmul_workspace(*args)
            for size in (wanted, min(wanted, 16 << 20)):      # (what fewer slices need, where there is not all of it)
                work = _memory(size, A, stream) if size else None
                if work is not None:
                    st = cyc_recurrence_matmul_in(*args, work.data_ptr(), size, s)
                    break
            if st == CYC_ERR_WORKSPACE:
                st = cyc_recurrence_matmul(*args, s)
    else:
        st = cyc_recurrence_matmul_batched(A.data_ptr(), B.data_ptr(), out.data_ptr(), batch, M, K, N,
                                           M * K, K * N, M * N, dtype, s)
    if st != CYC_OK:
        raise CycError(st)
    return out


def cyc_recurrence_cholesky(A: int, L: int, Lh: int, n: int, nb: int, stream: int = 0) -> int:
    """Raw C-ABI call: device pointers as integers, returns the status code."""
    return int(_lib().cyc_recurrence_cholesky(A, L, Lh, n, nb, stream))


def cyc_cholesky_workspace(A: int, L: int, Lh: int, n: int, nb: int) -> int:
    """Bytes of workspace that cyc_recurrence_cholesky_in wants for this matrix."""
    return int(_lib().cyc_cholesky_workspace(A, L, Lh, n, nb))


def cyc_recurrence_cholesky_in(A: int, L: int, Lh: int, n: int, nb: int, workspace: int, workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, returns the cyc_status."""
    return int(_lib().cyc_recurrence_cholesky_in(A, L, Lh, n, nb, workspace, workspace_bytes, stream))


def recurrence_cholesky(A, nb: int = 64, out=None, out_bf16=None, stream=None):
    """Tensor-level convenience: (L, Lh) with A = L L^T factored tile by tile (tiles of nb).

    A: (n,n) torch.float32 contiguous CUDA tensor, symmetric positive definite (its lower triangle is what counts).
    Allocates L (fp32, zero above the diagonal) and Lh (bf16, both triangles filled) unless given, and memory for
    the padded copy of an unaligned matrix or under stream capture, and forwards pointers to the C ABI on the
    current (or given) stream.  (Where that memory is not to be had an unaligned matrix is factored in place, more
    slowly and with other last bits.)
    """
    import torch
    if not A.is_cuda:
        raise ValueError("A must be a device tensor; there is no CPU path")
    if A.dtype != torch.float32 or A.dim() != 2 or A.shape[0] != A.shape[1] or not A.is_contiguous():
        raise ValueError(f"A must be a contiguous square float32 matrix, got {tuple(A.shape)} {A.dtype}")
    n = A.shape[0]
    if out is None:
        out = torch.empty((n, n), dtype=torch.float32, device=A.device)
    if out_bf16 is None:
        out_bf16 = torch.empty((n, n), dtype=torch.bfloat16, device=A.device)
    for t, dt in ((out, torch.float32), (out_bf16, torch.bfloat16)):
        if tuple(t.shape) != (n, n) or t.dtype != dt or not t.is_contiguous() or t.device != A.device:
            raise ValueError("out / out_bf16 has the wrong shape, dtype, layout or device")
    s = _stream_handle(A, stream)
    args = A.data_ptr(), out.data_ptr(), out_bf16.data_ptr(), n, nb
    st = cyc_recurrence_cholesky_in(*args, 0, 0, s)
    if st == CYC_ERR_WORKSPACE:                   # unaligned, or under capture: in memory that the caller brings
        wanted = cyc_cholesky_workspace(*args)
        work = _memory(wanted, A, stream) if wanted else None
        st = cyc_recurrence_cholesky(*args, s) if work is None else cyc_recurrence_cholesky_in(*args, work.data_ptr(), wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return out, out_bf16


def recurrence_trsm(L, B, nb: int = 64, out=None, out_bf16=None, stream=None):
    """Tensor-level convenience: (X, Xh) with L X = B solved tile by tile (tiles of nb rows).

    L: (n,n) torch.bfloat16, B: (n,nrhs) torch.float32, contiguous CUDA tensors.  Allocates X (fp32)
    and Xh (bf16) unless given, and memory for the padded copy of an unaligned system or under stream
    capture, and forwards pointers to the C ABI on the current (or given) stream.  (Where that memory is
    not to be had an unaligned system is solved in place, more slowly and with other last bits.)
    """
    import torch
    if not (L.is_cuda and B.is_cuda):
        raise ValueError("L and B must be device tensors; there is no CPU path")
    if L.dtype != torch.bfloat16 or B.dtype != torch.float32:
        raise ValueError("L must be bfloat16 and B float32")
    if L.dim() != 2 or B.dim() != 2 or L.shape[0] != L.shape[1] or B.shape[0] != L.shape[0]:
        raise ValueError(f"shape mismatch: L {tuple(L.shape)}, B {tuple(B.shape)}")
    if not (L.is_contiguous() and B.is_contiguous()):
        raise ValueError("L and B must be contiguous")
    n, nrhs = B.shape
    if out is None:
        out = torch.empty((n, nrhs), dtype=torch.float32, device=L.device)
    if out_bf16 is None:
        out_bf16 = torch.empty((n, nrhs), dtype=torch.bfloat16, device=L.device)
    for t, dt in ((out, torch.float32), (out_bf16, torch.bfloat16)):
        if tuple(t.shape) != (n, nrhs) or t.dtype != dt or not t.is_contiguous() or t.device != L.device:
            raise ValueError("out / out_bf16 has the wrong shape, dtype, layout or device")
    s = _stream_handle(L, stream)
    args = L.data_ptr(), B.data_ptr(), out.data_ptr(), out_bf16.data_ptr(), n, nrhs, nb
    st = cyc_recurrence_trsm_in(*args, 0, 0, s)
    if st == CYC_ERR_WORKSPACE:                   # unaligned, or under capture: in memory that the caller brings
        wanted = cyc_trsm_workspace(args[0], *args[2:])
        work = _memory(wanted, L, stream) if wanted else None
        st = cyc_recurrence_trsm(*args, s) if work is None else cyc_recurrence_trsm_in(*args, work.data_ptr(), wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return out, out_bf16


def recurrence_attention(Q, K, V, out=None, stream=None):
    """Tensor-level convenience: O = softmax(Q K^T / sqrt(d)) V by the tile recurrence.

    Q: (N,d) or (batch,N,d); K, V: (M,d) or (batch,M,d); contiguous torch.bfloat16 CUDA tensors, d 64 or 128.
    Allocates O (float32) unless given and forwards pointers to the C ABI on the current (or given) stream.
    """
    import torch
    if not (Q.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("Q, K and V must be device tensors; there is no CPU path")
    if not (Q.dtype == K.dtype == V.dtype == torch.bfloat16):
        raise ValueError("Q, K and V must be bfloat16")
    if Q.dim() not in (2, 3) or K.dim() != Q.dim() or K.shape != V.shape or Q.shape[-1] != K.shape[-1]:
        raise ValueError(f"shape mismatch: Q {tuple(Q.shape)}, K {tuple(K.shape)}, V {tuple(V.shape)}")
    if Q.dim() == 3 and Q.shape[0] != K.shape[0]:
        raise ValueError("batch extents differ")
    if not (Q.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("Q, K and V must be contiguous")
    batch = Q.shape[0] if Q.dim() == 3 else 1
    N, d = Q.shape[-2:]
    M = K.shape[-2]
    if out is None:
        out = torch.empty(tuple(Q.shape), dtype=torch.float32, device=Q.device)
    elif tuple(out.shape) != tuple(Q.shape) or out.dtype != torch.float32 or not out.is_contiguous() or out.device != Q.device:
        raise ValueError("out has the wrong shape, dtype, layout or device")
    s = _stream_handle(Q, stream)
    # The library splits no key list below 512.  Without memory the keys are not split, which is slower and adds the fp32 sums in
    # another order.
    wanted = cyc_attention_workspace(batch, N, M, d) if M >= 512 else 0
    work = _memory(wanted, Q, stream) if wanted else None
    if work is None:
        st = cyc_recurrence_attention(Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), batch, N, M, d, s)
    else:
        st = cyc_recurrence_attention_split(Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), batch, N, M, d, work.data_ptr(),
                                            wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return out


def _numbers(strides):
    """Strides as the C ABI takes them (a sequence of ints, or None)."""
    return None if strides is None else (ctypes.c_int64 * len(strides))(*strides)


def cyc_attention_window_workspace(batch: int, heads: int, kv_heads: int, N: int, M: int, d: int, window: int, sinks: int) -> int:
    """Bytes of workspace that cyc_recurrence_attention_window wants for these extents."""
    return int(_lib().cyc_attention_window_workspace(batch, heads, kv_heads, N, M, d, window, sinks))


def cyc_recurrence_attention_window(Q: int, K: int, V: int, O: int, lse: int, batch: int, heads: int, kv_heads: int, N: int, M: int, d: int,
                                    strides, window: int, sinks: int, workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> int:
    """Raw call: device addresses as ints, strides twelve ints or None; returns the cyc_status."""
    return int(_lib().cyc_recurrence_attention_window(Q, K, V, O, lse, batch, heads, kv_heads, N, M, d, _numbers(strides), window, sinks,
                                                      workspace, workspace_bytes, stream))


def cyc_attention_window_grad_workspace(batch: int, heads: int, kv_heads: int, N: int, M: int, d: int, window: int, sinks: int) -> int:
    """Bytes of workspace that cyc_recurrence_attention_window_grad needs for these extents."""
    return int(_lib().cyc_attention_window_grad_workspace(batch, heads, kv_heads, N, M, d, window, sinks))


def cyc_recurrence_attention_window_grad(Q: int, K: int, V: int, O: int, lse: int, dO: int, dQ: int, dK: int, dV: int, batch: int, heads: int,
                                         kv_heads: int, N: int, M: int, d: int, strides, window: int, sinks: int, workspace: int,
                                         workspace_bytes: int, stream: int = 0) -> int:
    """Raw call: device addresses as ints, strides twenty-four ints or None; returns the cyc_status."""
    return int(_lib().cyc_recurrence_attention_window_grad(Q, K, V, O, lse, dO, dQ, dK, dV, batch, heads, kv_heads, N, M, d, _numbers(strides),
                                                           window, sinks, workspace, workspace_bytes, stream))


def cyc_cache_append(K: int, V: int, cache: cyc_cache, tokens: int, strides, stream: int = 0) -> int:
    """Raw call: device addresses as ints, strides four ints or None; returns the cyc_status."""
    return int(_lib().cyc_cache_append(K, V, cache, tokens, _numbers(strides), stream))


def cyc_attention_paged_workspace(cache: cyc_cache, tokens: int, heads: int, max_new: int, window: int, sinks: int) -> int:
    """Bytes of workspace that cyc_recurrence_attention_paged wants for these extents."""
    return int(_lib().cyc_attention_paged_workspace(cache, tokens, heads, max_new, window, sinks))


def cyc_recurrence_attention_paged(Q: int, cache: cyc_cache, O: int, tokens: int, heads: int, strides, max_new: int, window: int, sinks: int,
                                   workspace: int = 0, workspace_bytes: int = 0, stream: int = 0) -> int:
    """Raw call: device addresses as ints, strides four ints or None; returns the cyc_status."""
    return int(_lib().cyc_recurrence_attention_paged(Q, cache, O, tokens, heads, _numbers(strides), max_new, window, sinks, workspace,
                                                     workspace_bytes, stream))


def _elsewhere(call, tensor, stream, *args):
    """call(*args, stream) with the tensor's device as the current one and `stream`, where one is given, as its current stream: what is
    allocated inside comes from the pool of the stream that the call runs on, so that no work still pending on another stream uses it.
    A stream of another library (any object with a handle in `cuda_stream`) has a pool too, which goes by the handle."""
    import torch
    if getattr(stream, "device", tensor.device) != tensor.device:
        raise ValueError(f"the stream is on {stream.device}, the tensors are on {tensor.device}")
    with torch.cuda.device(tensor.device):
        if stream is None:
            return call(*args, None)
        if not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(stream.cuda_stream, device=tensor.device)
        with torch.cuda.stream(stream):
            return call(*args, stream)


def _mask_arguments(window, sinks):
    """window and sinks as the C ABI takes them."""
    if window is not None and window < 1:
        raise ValueError(f"window must be at least 1, or None for no window; got {window}")
    if sinks < 0:
        raise ValueError(f"sinks must not be negative; got {sinks}")
    return window or 0, sinks


def _device_of(name, t):
    """The index of the device that a tensor lies on, which decides for the whole call."""
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor; there is no CPU path")
    if t.dtype is not torch.bfloat16:
        raise ValueError(f"{name} must be bfloat16, got {t.dtype}")
    return t.get_device()


def _dense(t, shape, device, bfloat16) -> bool:
    """The usual operand: all that _check_rows asks for, and contiguous."""
    return t.is_cuda and t.dtype is bfloat16 and t.is_contiguous() and t.shape == shape and t.get_device() == device and not t.data_ptr() & 15


def _empty_like(t):
    """A dense tensor of the shape, type and device of t: empty_like, the faster call by 0.5 of 12 us, would keep other strides."""
    import torch
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _steps(t):
    """The strides that count: those of all dimensions but the last, 0 for those of one element or none, which torch leaves open."""
    return [s if n > 1 else 0 for n, s in zip(t.shape[:-1], t.stride())]


def _check_rows(name, t, shape, device):
    """A bfloat16 tensor of `shape` on `device` whose rows a kernel can read 16 bytes at a time."""
    import torch
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor; there is no CPU path")
    if t.dtype != torch.bfloat16:
        raise ValueError(f"{name} must be bfloat16, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"shape mismatch: {name} is {tuple(t.shape)}, expected {tuple(shape)}")
    if t.get_device() != device:
        raise ValueError("all tensors must be on one device")
    if t.stride(-1) != 1 and t.numel() or t.data_ptr() & 15 or any([s % 8 for s in _steps(t)]):
        raise ValueError(f"{name} needs contiguous rows at multiples of 16 bytes")


def _operands(named, device):
    """Strides of (name, tensor, shape) as the C ABI takes them, None where all are dense; raises where one will not do.  The
    usual case is looked at first: a small call is over in 8 us, of which all checks one by one would be 4."""
    import torch
    bfloat16 = torch.bfloat16
    if all([_dense(t, shape, device, bfloat16) for _, t, shape in named]):
        return None
    for name, t, shape in named:
        _check_rows(name, t, shape, device)
    return [s for _, t, _ in named for s in t.stride()[:-1]]


def _attention_shapes(Q, K):
    q, k = Q.shape, K.shape
    if len(q) != 4 or len(k) != 4 or q[0] != k[0] or q[3] != k[3]:
        raise ValueError(f"shape mismatch: Q {tuple(q)}, K {tuple(k)}")
    if q[3] not in (64, 128):
        raise ValueError(f"the head dimension must be 64 or 128, got {q[3]}")
    if k[1] == 0 or q[1] % k[1]:
        raise ValueError(f"{q[1]} query heads do not divide among {k[1]} key heads")
    return q, k


def _check_lse(lse, shape, device):
    import torch
    if not lse.is_cuda or lse.dtype != torch.float32 or lse.shape != shape or not lse.is_contiguous() or lse.get_device() != device:
        raise ValueError("lse has the wrong shape, dtype, layout or device")


def recurrence_attention_window(Q, K, V, window=None, sinks: int = 0, out=None, lse=None, stream=None):
    """Tensor-level convenience: (O, lse) of causal attention with a sliding window and sinks.

    Q: (batch, heads, N, d), K, V: (batch, kv_heads, M, d), torch.bfloat16 CUDA tensors with contiguous rows of d (64 or 128) and any
    strides otherwise that are multiples of 8 (so views of (batch, N, heads, d) will do); heads a multiple of kv_heads.  The
    queries are the last N of the M positions; position p sees the keys j <= p with p - j < window (None: all) or j < sinks.
    Allocates O (bfloat16, dense) and lse (float32, (batch, heads, N): the logarithms of the sums, for the gradient) unless given, and
    memory to split the keys of few queries over the chip, and forwards pointers to the C ABI on the current (or given) stream.
    (Where that memory is not to be had the keys are not split.  Each part of split keys rounds its weights to bfloat16 against a largest score of
    its own, so that O differs by as much as those roundings.)  Records nothing for autograd: O and lse have no graph, and
    recurrence_attention_window_grad is what a torch.autograd.Function calls in its backward.
    """
    import torch
    if Q.is_cuda and (stream is not None or Q.get_device() != torch.cuda.current_device()):
        return _elsewhere(_attention_window, Q, stream, Q, K, V, window, sinks, out, lse)
    return _attention_window(Q, K, V, window, sinks, out, lse, stream)


def _attention_window(Q, K, V, window, sinks, out, lse, stream):
    import torch
    q, k = _attention_shapes(Q, K)
    window, sinks = _mask_arguments(window, sinks)
    batch, heads, N, d = q
    kv_heads, M = k[1:3]
    device = _device_of("Q", Q)
    if out is None:
        out = _empty_like(Q)
    strides = _operands((("Q", Q, q), ("K", K, k), ("V", V, k), ("out", out, q)), device)
    if lse is None:
        lse = Q.new_empty(q[:3], dtype=torch.float32)
    else:
        _check_lse(lse, q[:3], device)
    s = _stream_handle(Q, stream)
    work, wanted = None, 0
    if M >= 512:                                  # shorter lists of keys are not worth splitting
        wanted = cyc_attention_window_workspace(batch, heads, kv_heads, N, M, d, window, sinks)
        work = _memory(wanted, Q, stream) if wanted else None
    st = cyc_recurrence_attention_window(Q.data_ptr(), K.data_ptr(), V.data_ptr(), out.data_ptr(), lse.data_ptr(), batch, heads, kv_heads, N, M, d,
                                         strides, window, sinks, 0 if work is None else work.data_ptr(), 0 if work is None else wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return out, lse


def recurrence_attention_window_grad(Q, K, V, O, lse, dO, window=None, sinks: int = 0, dQ=None, dK=None, dV=None, stream=None):
    """Tensor-level convenience: (dQ, dK, dV) of recurrence_attention_window from what it returned and the gradient of O.

    Q, K, V, window, sinks as in the forward call, O and lse what it returned, dO like O.  Allocates the gradients (bfloat16, dense, of the
    shapes of Q, K and V) unless given and the memory that the call needs (torch.OutOfMemoryError where there is none), and forwards pointers to
    the C ABI on the current (or given) stream.
    """
    import torch
    if Q.is_cuda and (stream is not None or Q.get_device() != torch.cuda.current_device()):
        return _elsewhere(_attention_window_grad, Q, stream, Q, K, V, O, lse, dO, window, sinks, dQ, dK, dV)
    return _attention_window_grad(Q, K, V, O, lse, dO, window, sinks, dQ, dK, dV, stream)


def _attention_window_grad(Q, K, V, O, lse, dO, window, sinks, dQ, dK, dV, stream):
    import torch
    q, k = _attention_shapes(Q, K)
    window, sinks = _mask_arguments(window, sinks)
    batch, heads, N, d = q
    kv_heads, M = k[1:3]
    device = _device_of("Q", Q)
    dQ = _empty_like(Q) if dQ is None else dQ
    dK = _empty_like(K) if dK is None else dK
    dV = _empty_like(V) if dV is None else dV
    strides = _operands((("Q", Q, q), ("K", K, k), ("V", V, k), ("O", O, q), ("dO", dO, q), ("dQ", dQ, q), ("dK", dK, k), ("dV", dV, k)), device)
    _check_lse(lse, q[:3], device)
    s = _stream_handle(Q, stream)
    wanted = cyc_attention_window_grad_workspace(batch, heads, kv_heads, N, M, d, window, sinks)
    work = Q.new_empty(wanted, dtype=torch.uint8) if wanted else None        # (of the stream's pool, see _elsewhere; the call cannot do without)
    st = cyc_recurrence_attention_window_grad(Q.data_ptr(), K.data_ptr(), V.data_ptr(), O.data_ptr(), lse.data_ptr(), dO.data_ptr(), dQ.data_ptr(),
                                              dK.data_ptr(), dV.data_ptr(), batch, heads, kv_heads, N, M, d, strides, window, sinks,
                                              0 if work is None else work.data_ptr(), 0 if work is None else wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return dQ, dK, dV


def _cache(K_cache, V_cache, table, lengths, starts, name, t):
    """The tensors of a cache, checked, as the C ABI takes them, and the device of the call, that of tensor `t`."""
    import torch
    shape, strides = K_cache.shape, K_cache.stride()
    if len(shape) != 4 or (strides != V_cache.stride() and (V_cache.shape != shape or _steps(K_cache) != _steps(V_cache))):
        raise ValueError("K_cache and V_cache must be (pages, kv_heads, page, d) with the same strides")
    device = _device_of(name, t)
    _operands((("K_cache", K_cache, shape), ("V_cache", V_cache, shape)), device)
    int32 = torch.int32
    for name, t, dims in (("table", table, 2), ("lengths", lengths, 1), ("starts", starts, 1)):
        if not t.is_cuda or t.dtype is not int32 or t.dim() != dims or (not t.is_contiguous() and t.stride(-1) != 1):
            raise ValueError(f"{name} must be a device tensor of int32 with {dims} dimension(s) and contiguous rows")
        if t.get_device() != device:
            raise ValueError("all tensors must be on one device")
    pages, kv_heads, page, d = shape
    seqs, max_pages = table.shape
    if lengths.shape[0] != seqs or starts.shape[0] != seqs + 1:
        raise ValueError(f"{seqs} sequences need {seqs} lengths and {seqs + 1} starts, got {lengths.shape[0]} and {starts.shape[0]}")
    if page < 1 or page & (page - 1) or page > 65536 or d not in (64, 128):
        raise ValueError(f"pages hold a power of two of keys (up to 65536) of 64 or 128 elements, got {page} of {d}")
    return cyc_cache(K_cache.data_ptr(), V_cache.data_ptr(), table.data_ptr(), lengths.data_ptr(), starts.data_ptr(), seqs, pages, max_pages,
                     kv_heads, page, d, table.stride(0), *strides[:3]), device


def cache_append(K, V, K_cache, V_cache, table, lengths, starts, stream=None):
    """Tensor-level convenience: writes the keys and values of new tokens into the pages of a cache.

    K, V: (tokens, kv_heads, d), K_cache, V_cache: (pages, kv_heads, page, d), torch.bfloat16 CUDA tensors with contiguous rows and any
    strides otherwise that are multiples of 8; table: (sequences, max_pages), lengths: (sequences,), starts: (sequences + 1,), torch.int32.
    Rows starts[b] .. starts[b+1] - 1 of K and V become the last of the lengths[b] keys of sequence b; key j lies in row j % page of
    page table[b, j // page].  Tokens without a place (no sequence, key, or page) are not written.  Allocates nothing.
    """
    import torch
    if K.is_cuda and (stream is not None or K.get_device() != torch.cuda.current_device()):
        return _elsewhere(_append, K, stream, K, V, K_cache, V_cache, table, lengths, starts)
    return _append(K, V, K_cache, V_cache, table, lengths, starts, stream)


def _append(K, V, K_cache, V_cache, table, lengths, starts, stream):
    cache, device = _cache(K_cache, V_cache, table, lengths, starts, "K", K)
    shape = (K.shape[0] if K.dim() else 0, cache.kv_heads, cache.d)
    strides = _operands((("K", K, shape), ("V", V, shape)), device)
    st = cyc_cache_append(K.data_ptr(), V.data_ptr(), cache, shape[0], strides, _stream_handle(K, stream))
    if st != CYC_OK:
        raise CycError(st)


def recurrence_attention_paged(Q, K_cache, V_cache, table, lengths, starts, window=None, sinks: int = 0, max_new=None, out=None, stream=None):
    """Tensor-level convenience: attention of new tokens over a paged cache that holds their keys and values already (cache_append).

    Q: (tokens, heads, d), torch.bfloat16; the cache, table, lengths and starts as in cache_append, heads a multiple of kv_heads; window
    and sinks as in recurrence_attention_window.  Rows starts[b] .. starts[b+1] - 1 of Q are the last positions of sequence b.  max_new: the
    most new tokens that any sequence brings, where the caller knows it: with 1, the usual step of a decoder, only the kernel for
    few rows is launched (a sequence that brings more has NaN in its rows then).  The last bits of a row depend on how its keys are split, and that on
    the lengths of all sequences of the call.  Records nothing for autograd.  Allocates O (bfloat16, dense) unless given and memory to
    split the keys over the chip, and forwards pointers to the C ABI on the current (or given) stream.
    """
    import torch
    if Q.is_cuda and (stream is not None or Q.get_device() != torch.cuda.current_device()):
        return _elsewhere(_attention_paged, Q, stream, Q, K_cache, V_cache, table, lengths, starts, window, sinks, max_new, out)
    return _attention_paged(Q, K_cache, V_cache, table, lengths, starts, window, sinks, max_new, out, stream)


def _attention_paged(Q, K_cache, V_cache, table, lengths, starts, window, sinks, max_new, out, stream):
    cache, device = _cache(K_cache, V_cache, table, lengths, starts, "Q", Q)
    q = Q.shape
    if len(q) != 3 or q[2] != cache.d:
        raise ValueError(f"shape mismatch: Q {tuple(q)}, K_cache {tuple(K_cache.shape)}")
    window, sinks = _mask_arguments(window, sinks)
    if max_new is not None and max_new < 1:
        raise ValueError(f"max_new must be at least 1, or None; got {max_new}")
    tokens, heads, _ = q
    if cache.kv_heads == 0 or heads % cache.kv_heads:
        raise ValueError(f"{heads} query heads do not divide among {cache.kv_heads} key heads")
    if out is None:
        out = _empty_like(Q)
    strides = _operands((("Q", Q, q), ("out", out, q)), device)
    s = _stream_handle(Q, stream)
    work, wanted = None, 0
    if cache.max_pages * cache.page >= 512:       # shorter lists of keys are not worth splitting
        wanted = cyc_attention_paged_workspace(cache, tokens, heads, max_new or 0, window, sinks)
        work = _memory(wanted, Q, stream) if wanted else None
    st = cyc_recurrence_attention_paged(Q.data_ptr(), cache, out.data_ptr(), tokens, heads, strides, max_new or 0, window, sinks,
                                        0 if work is None else work.data_ptr(), 0 if work is None else wanted, s)
    if st != CYC_OK:
        raise CycError(st)
    return out
