"""Python binding of libvq (MI355X / gfx950 vector-quantised GEMV library).

Argument marshalling only: every step of the path runs in the HIP kernels behind
the C ABI declared in include/vq.h.  Tensors are used for device memory and
streams, nothing else.  There is no CPU fallback: if the shared library is not
built, importing the binding's functions raises.
"""
from __future__ import annotations

import array
import ctypes
import os
import struct
from typing import Sequence

__all__ = [
    "VQDesc", "VQError", "VQ_F16", "VQ_F32", "VQ_I8", "VQ_I8_BN", "lib", "lib_path", "make_desc",
    "vq_status_string", "vq_version", "vq_canonical_bytes", "vq_layout_bytes",
    "vq_pack_layout", "vq_gemv", "vq_gemv_multi", "GemvMultiArgs", "VQLoraDesc", "vq_lora_workspace_bytes", "vq_gemv_lora",
    "vq_gemv_lora_multi", "vq_gemv_lora_multi_static", "vq_gemm_batched", "vq_decode_dense", "vq_em_assign", "vq_em_update",
    "VQ_BF16", "VQAttnDesc", "VQAttnBatch", "VQStrides", "make_attn_desc", "AttnBatch", "attn_workspace", "vq_cache_bytes",
    "vq_cache_append", "vq_cache_copy", "vq_attn_workspace_bytes", "vq_attn_decode", "vq_attn_prompt",
]

VQ_F16 = 1
VQ_F32 = 2
VQ_I8 = 3      # codebook_dtype: int8 lookup tables with one fp16 scale per group
VQ_I8_BN = 4   # the same plus blockwise normalisation (16 levels per group, a 4-bit code per 32 weights)
VQ_BF16 = 5    # attention over the paged cache only

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libvq.so")
_lib = None


class VQDesc(ctypes.Structure):
    """Mirror of `vq_desc` (include/vq.h)."""
    _fields_ = [
        ("out_features", ctypes.c_int32), ("in_features", ctypes.c_int32),
        ("group_rows", ctypes.c_int32), ("group_cols", ctypes.c_int32),
        ("d", ctypes.c_int32), ("k", ctypes.c_int32),
        ("index_bits", ctypes.c_int32), ("codebook_dtype", ctypes.c_int32),
    ]


class VQLoraDesc(ctypes.Structure):
    """Mirror of `vq_lora_desc` (include/vq.h)."""
    _fields_ = [("A_f16", ctypes.c_void_p), ("B_f16", ctypes.c_void_p),
                ("rank", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class VQAttnDesc(ctypes.Structure):
    """Mirror of `vq_attn_desc` (include/vq.h)."""
    _fields_ = [("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)]


class VQAttnBatch(ctypes.Structure):
    """Mirror of `vq_attn_batch` (include/vq.h)."""
    _fields_ = [("n_seqs", ctypes.c_int32), ("n_tokens", ctypes.c_int32), ("table_width", ctypes.c_int32),
                ("max_len", ctypes.c_int32), ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p)]


class VQStrides(ctypes.Structure):
    """Mirror of `vq_strides` (include/vq.h)."""
    _fields_ = [("token", ctypes.c_int64), ("head", ctypes.c_int64), ("dim", ctypes.c_int64)]


_LORA_STRUCT = struct.Struct("=QQii")   # the fields of VQLoraDesc


class VQError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {vq_status_string(status)} ({status})")


def lib_path() -> str:
    return _LIB_PATH


def lib() -> ctypes.CDLL:
    """Loads libvq.so (built in-tree by `python -m paper_2402_15319_amd.build`)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(
                f"{_LIB_PATH} is not built; run `python -m paper_2402_15319_amd.build` "
                "(there is no fallback path)")
        L = ctypes.CDLL(_LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(ctypes.c_size_t)
        dp = ctypes.POINTER(VQDesc)
        L.vq_status_string.restype = ctypes.c_char_p
        L.vq_status_string.argtypes = [i32]
        L.vq_version.restype = i32
        L.vq_version.argtypes = []
        for name in ("vq_canonical_bytes", "vq_layout_bytes"):
            getattr(L, name).restype = i32
            getattr(L, name).argtypes = [dp, sz, sz]
        L.vq_pack_layout.restype = i32
        L.vq_pack_layout.argtypes = [dp, vp, vp, vp, vp, vp]
        L.vq_gemv.restype = i32
        L.vq_gemv.argtypes = [dp, vp, vp, vp, vp, i32, vp]
        L.vq_gemv_multi.restype = i32
        L.vq_gemv_multi.argtypes = [i32, dp, ctypes.POINTER(vp), ctypes.POINTER(vp),
                                    ctypes.POINTER(vp), ctypes.POINTER(vp), i32, vp]
        L.vq_lora_workspace_bytes.restype = i32
        L.vq_lora_workspace_bytes.argtypes = [i32, sz]
        L.vq_gemv_lora.restype = i32
        L.vq_gemv_lora.argtypes = [dp, vp, vp, vp, vp, vp, i32, vp, ctypes.c_size_t, vp, i32, vp]
        L.vq_gemv_lora_multi.restype = i32
        L.vq_gemv_lora_multi.argtypes = [i32, dp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                         ctypes.POINTER(VQLoraDesc), vp, ctypes.c_size_t, ctypes.POINTER(vp), i32, vp]
        L.vq_gemv_lora_multi_static.restype = i32
        L.vq_gemv_lora_multi_static.argtypes = [i32, dp, ctypes.POINTER(vp), ctypes.POINTER(vp), ctypes.POINTER(vp),
                                                ctypes.POINTER(VQLoraDesc), ctypes.POINTER(vp), i32, vp]
        L.vq_gemm_batched.restype = i32
        L.vq_gemm_batched.argtypes = [dp, vp, vp, vp, i32, i32, vp, i32, i32, vp]
        L.vq_decode_dense.restype = i32
        L.vq_decode_dense.argtypes = [dp, vp, vp, vp, vp]
        L.vq_em_assign.restype = i32
        L.vq_em_assign.argtypes = [dp, vp, vp, vp, vp, vp]
        L.vq_em_update.restype = i32
        L.vq_em_update.argtypes = [dp, vp, vp, vp, vp, vp]
        ap, bp, st = ctypes.POINTER(VQAttnDesc), ctypes.POINTER(VQAttnBatch), ctypes.POINTER(VQStrides)
        L.vq_cache_bytes.restype = i32
        L.vq_cache_bytes.argtypes = [ap, sz]
        L.vq_cache_append.restype = i32
        L.vq_cache_append.argtypes = [ap, bp, vp, st, vp, st, vp, vp, vp]
        L.vq_cache_copy.restype = i32
        L.vq_cache_copy.argtypes = [ap, i32, vp, i32, vp, vp]   # two host arrays
        L.vq_attn_workspace_bytes.restype = i32
        L.vq_attn_workspace_bytes.argtypes = [ap, bp, sz]
        for name in ("vq_attn_decode", "vq_attn_prompt"):
            getattr(L, name).restype = i32
            getattr(L, name).argtypes = [ap, bp, vp, st, vp, vp, vp, st, vp, vp, ctypes.c_size_t, vp]
        _lib = L
    return _lib


def make_desc(out_features: int, in_features: int, k: int, index_bits: int,
              group_rows: int = 8, group_cols: int = 256, d: int = 2,
              codebook_dtype: int = VQ_F16) -> VQDesc:
    return VQDesc(out_features, in_features, group_rows, group_cols, d, k, index_bits,
                  codebook_dtype)


def _ptr(t) -> int:
    """Device/host address of a tensor, or an int passed through (0 = NULL)."""
    if t is None:
        return 0
    if isinstance(t, int):
        return t
    return t.data_ptr()


_torch = None


def _stream(stream) -> int:
    # The current stream's handle without building a Stream object: 0.3 us of a call's host time in place
    # of 2.8.  A torch without these two functions (they are not part of its public interface) gets the Stream object.
    if stream is None:
        global _torch
        if _torch is None:
            import torch
            _torch = torch
        if not _torch.cuda.is_initialized():
            return _torch.cuda.current_stream().cuda_stream
        try:
            return _torch._C._cuda_getCurrentRawStream(_torch._C._cuda_getDevice())
        except AttributeError:
            return _torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int, where: str) -> None:
    if status != 0:
        raise VQError(status, where)


def vq_status_string(status: int) -> str:
    return lib().vq_status_string(status).decode()


def vq_version() -> int:
    return lib().vq_version()


def vq_canonical_bytes(desc: VQDesc) -> tuple[int, int]:
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().vq_canonical_bytes(ctypes.byref(desc), ctypes.byref(a), ctypes.byref(b)),
           "vq_canonical_bytes")
    return a.value, b.value


def vq_layout_bytes(desc: VQDesc) -> tuple[int, int]:
    a, b = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().vq_layout_bytes(ctypes.byref(desc), ctypes.byref(a), ctypes.byref(b)),
           "vq_layout_bytes")
    return a.value, b.value


def vq_pack_layout(desc: VQDesc, idx_canon, cb_canon, idx_dev, cb_dev, stream=None) -> None:
    _check(lib().vq_pack_layout(ctypes.byref(desc), _ptr(idx_canon), _ptr(cb_canon),
                                _ptr(idx_dev), _ptr(cb_dev), _stream(stream)), "vq_pack_layout")


def vq_gemv(desc: VQDesc, idx_dev, cb_dev, x, y, y_dtype: int = VQ_F16, stream=None) -> None:
    _check(lib().vq_gemv(ctypes.byref(desc), _ptr(idx_dev), _ptr(cb_dev), _ptr(x), _ptr(y),
                         y_dtype, _stream(stream)), "vq_gemv")


class GemvMultiArgs:
    """Pre-marshalled argument arrays for vq_gemv_multi (build once, call many times).  Keeps a
    reference to every tensor it was given, so the device memory behind the stored addresses
    lives as long as this object."""

    def __init__(self, descs: Sequence[VQDesc], idx_dev, cb_dev, xs, ys):
        n = len(descs)
        if not (len(idx_dev) == len(cb_dev) == len(xs) == len(ys) == n):
            raise ValueError("vq_gemv_multi: argument lists differ in length")
        self.count = n
        self.descs = (VQDesc * n)(*descs)
        arr = ctypes.c_void_p * n
        self.idx = arr(*[_ptr(t) for t in idx_dev])
        self.cb = arr(*[_ptr(t) for t in cb_dev])
        self.x = arr(*[_ptr(t) for t in xs])
        self.y = arr(*[_ptr(t) for t in ys])
        self._keep = (list(idx_dev), list(cb_dev), list(xs), list(ys))


def vq_gemv_multi(args_or_descs, idx_dev=None, cb_dev=None, xs=None, ys=None,
                  y_dtype: int = VQ_F16, stream=None) -> None:
    a = args_or_descs if isinstance(args_or_descs, GemvMultiArgs) else \
        GemvMultiArgs(args_or_descs, idx_dev, cb_dev, xs, ys)
    _check(lib().vq_gemv_multi(a.count, a.descs, a.idx, a.cb, a.x, a.y, y_dtype,
                               _stream(stream)), "vq_gemv_multi")


def vq_lora_workspace_bytes(count: int) -> int:
    a = ctypes.c_size_t(0)
    _check(lib().vq_lora_workspace_bytes(count, ctypes.byref(a)), "vq_lora_workspace_bytes")
    return a.value


def vq_gemv_lora(desc: VQDesc, idx_dev, cb_dev, x, A, B, rank: int, workspace, y,
                 y_dtype: int = VQ_F16, stream=None, workspace_bytes: int | None = None) -> None:
    nb = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    _check(lib().vq_gemv_lora(ctypes.byref(desc), _ptr(idx_dev), _ptr(cb_dev), _ptr(x), _ptr(A), _ptr(B), rank,
                              _ptr(workspace), nb, _ptr(y), y_dtype, _stream(stream)), "vq_gemv_lora")


def _lora_array(As, Bs, ranks: Sequence[int]):
    """The adapters' descriptors as one array, filled from packed bytes (a structure object per adapter
    costs about 1 us)."""
    n = len(ranks)
    try:
        packed = b"".join([_LORA_STRUCT.pack(_ptr(a), _ptr(b), r, 0) for a, b, r in zip(As, Bs, ranks)])
    except struct.error:   # a value that does not fit its field: as a structure takes it, for the library to judge
        return (VQLoraDesc * n)(*[VQLoraDesc(_ptr(a), _ptr(b), r, 0) for a, b, r in zip(As, Bs, ranks)])
    return (VQLoraDesc * n).from_buffer_copy(packed)


def vq_gemv_lora_multi(args: GemvMultiArgs, As, Bs, ranks: Sequence[int], workspace,
                       y_dtype: int = VQ_F16, stream=None, workspace_bytes: int | None = None) -> None:
    """args as for vq_gemv_multi; As/Bs/ranks: one adapter per product (rank 0 = none)."""
    n = args.count
    if not (len(As) == len(Bs) == len(ranks) == n):
        raise ValueError("vq_gemv_lora_multi: argument lists differ in length")
    lora = _lora_array(As, Bs, ranks)
    nb = workspace.numel() * workspace.element_size() if workspace_bytes is None else workspace_bytes
    _check(lib().vq_gemv_lora_multi(n, args.descs, args.idx, args.cb, args.x, lora, _ptr(workspace), nb,
                                    args.y, y_dtype, _stream(stream)), "vq_gemv_lora_multi")


def vq_gemv_lora_multi_static(args: GemvMultiArgs, As, Bs, ranks: Sequence[int],
                              y_dtype: int = VQ_F16, stream=None) -> None:
    """vq_gemv_lora_multi without a workspace (at most 256 products; allocates nothing)."""
    n = args.count
    if not (len(As) == len(Bs) == len(ranks) == n):
        raise ValueError("vq_gemv_lora_multi_static: argument lists differ in length")
    lora = _lora_array(As, Bs, ranks)
    _check(lib().vq_gemv_lora_multi_static(n, args.descs, args.idx, args.cb, args.x, lora, args.y, y_dtype,
                                           _stream(stream)), "vq_gemv_lora_multi_static")


def vq_gemm_batched(desc: VQDesc, idx_dev, cb_dev, X, B: int, ldx: int, Y, ldy: int,
                    y_dtype: int = VQ_F16, stream=None) -> None:
    _check(lib().vq_gemm_batched(ctypes.byref(desc), _ptr(idx_dev), _ptr(cb_dev), _ptr(X), B, ldx,
                                 _ptr(Y), ldy, y_dtype, _stream(stream)), "vq_gemm_batched")


def vq_decode_dense(desc: VQDesc, idx_dev, cb_dev, W, stream=None) -> None:
    _check(lib().vq_decode_dense(ctypes.byref(desc), _ptr(idx_dev), _ptr(cb_dev), _ptr(W),
                                 _stream(stream)), "vq_decode_dense")


def vq_em_assign(desc: VQDesc, W_f32, hdiag_f32, cb_f32, assign_u8, stream=None) -> None:
    _check(lib().vq_em_assign(ctypes.byref(desc), _ptr(W_f32), _ptr(hdiag_f32), _ptr(cb_f32),
                              _ptr(assign_u8), _stream(stream)), "vq_em_assign")


def vq_em_update(desc: VQDesc, W_f32, hdiag_f32, assign_u8, cb_f32_out, stream=None) -> None:
    _check(lib().vq_em_update(ctypes.byref(desc), _ptr(W_f32), _ptr(hdiag_f32), _ptr(assign_u8),
                              _ptr(cb_f32_out), _stream(stream)), "vq_em_update")


def make_attn_desc(heads: int, kv_heads: int, head_dim: int, page_size: int, n_pages: int, dtype: int = VQ_F16,
                   scale: float | None = None) -> VQAttnDesc:
    """scale: of the logits; None means 1 / sqrt(head_dim)."""
    return VQAttnDesc(heads, kv_heads, head_dim, page_size, n_pages, dtype, head_dim ** -0.5 if scale is None else scale, 0)


class AttnBatch:
    """The sequences of a call (build once, call as long as the arrays and these sizes stay; what the arrays hold may change).
    Keeps references to the tensors.  kv_len: int32 [n_seqs]; page_table: int32 [n_seqs, table_width]; q_start: int32
    [n_seqs + 1], or None for one new token of every sequence; max_len: no kv_len is larger (None: what the table can list)."""

    def __init__(self, kv_len, page_table, n_tokens: int | None = None, max_len: int | None = None, q_start=None, page_size: int | None = None):
        import torch
        _kinds.update({VQ_F16: torch.float16, VQ_BF16: torch.bfloat16, VQ_F32: torch.float32})
        for what, t, dim in (("kv_len", kv_len, 1), ("page_table", page_table, 2), ("q_start", q_start, 1)):
            if t is not None and (t.dtype != torch.int32 or t.dim() != dim or not t.is_contiguous()):
                raise ValueError(f"AttnBatch: {what} is a contiguous int32 tensor of {dim} dimension(s)")
        n = kv_len.shape[0]
        if page_table.shape[0] != n or (q_start is not None and q_start.shape[0] != n + 1):
            raise ValueError("AttnBatch: arrays of different numbers of sequences")
        self.device, self.gpu = kv_len.device, kv_len.get_device()   # -1: on the host, which is enough for sizes
        if page_table.get_device() != self.gpu or (q_start is not None and q_start.get_device() != self.gpu):
            raise ValueError("AttnBatch: arrays on different devices")
        if n_tokens is None:
            if q_start is not None:
                raise ValueError("AttnBatch: n_tokens is needed with q_start")
            n_tokens = n
        if max_len is None:
            if page_size is None:
                raise ValueError("AttnBatch: max_len, or page_size to take what the table can list")
            max_len = page_table.shape[1] * page_size
        self.struct = VQAttnBatch(n, n_tokens, page_table.shape[1], max_len, _ptr(q_start) or None, _ptr(kv_len), _ptr(page_table))
        self.n_tokens = n_tokens
        self._keep = (kv_len, page_table, q_start)


_kinds: dict = {}   # VQ_F16, VQ_BF16, VQ_F32: the torch type (filled by the first AttnBatch)


def _rows(t, n: int, heads: int, dim: int, what: str, kind, gpu: int):
    """The strides of a [n, heads, dim] tensor; None where it has no gaps."""
    if t.shape != (n, heads, dim) or t.dtype is not kind or t.get_device() != gpu or gpu < 0:
        raise ValueError(f"{what}: a tensor [{n}, {heads}, {dim}] of the descriptor's type on the GPU of the batch's arrays is wanted, not {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    return None if t.is_contiguous() else VQStrides(*t.stride())


def _pages(t, size: int, what: str, kind, gpu: int) -> int:
    """The address of a K or V buffer (an address passes through)."""
    try:
        if t.dtype is kind and t.nbytes >= size and t.get_device() == gpu and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        return _ptr(t)
    raise ValueError(f"{what}: a contiguous tensor of the descriptor's type and of {size} bytes or more on the batch's GPU is wanted, not {t.dtype} "
                     f"{tuple(t.shape)} on {t.device}")


def vq_cache_bytes(desc: VQAttnDesc) -> int:
    a = ctypes.c_size_t(0)
    _check(lib().vq_cache_bytes(ctypes.byref(desc), ctypes.byref(a)), "vq_cache_bytes")
    return a.value


def vq_cache_append(desc: VQAttnDesc, batch: AttnBatch, k, v, k_pages, v_pages, stream=None) -> None:
    """k, v: [n_tokens, kv_heads, head_dim] views (strides as vq_strides allows) of the new tokens."""
    n, heads, dim, kind, gpu = batch.n_tokens, desc.kv_heads, desc.head_dim, _kinds.get(desc.dtype), batch.gpu
    size = 2 * desc.n_pages * heads * desc.page_size * dim
    _check(lib().vq_cache_append(desc, batch.struct, k.data_ptr(), _rows(k, n, heads, dim, "k", kind, gpu), v.data_ptr(),
                                 _rows(v, n, heads, dim, "v", kind, gpu), _pages(k_pages, size, "k_pages", kind, gpu),
                                 _pages(v_pages, size, "v_pages", kind, gpu), _stream(stream)), "vq_cache_append")


def vq_cache_copy(desc: VQAttnDesc, buffers, from_to, stream=None) -> None:
    """buffers: K and V buffers, whole ones (vq_cache_bytes each, on the current GPU: of so many this is not checked); from_to: (page,
    page) pairs, copied one after another in every buffer."""
    try:
        flat = array.array("i", [p for a, b in from_to for p in (a, b)])
    except (ValueError, TypeError, OverflowError) as e:
        raise ValueError("vq_cache_copy: from_to is a list of pairs of page numbers") from e
    if not isinstance(buffers, (list, tuple)):
        buffers = list(buffers)   # gone through twice where there are addresses among them
    try:
        at = array.array("Q", [b.data_ptr() for b in buffers])
    except AttributeError:
        at = array.array("Q", [_ptr(b) for b in buffers])
    _check(lib().vq_cache_copy(desc, len(at), at.buffer_info()[0], len(flat) // 2, flat.buffer_info()[0], _stream(stream)), "vq_cache_copy")


def vq_attn_workspace_bytes(desc: VQAttnDesc, batch: AttnBatch) -> int:
    a = ctypes.c_size_t(0)
    _check(lib().vq_attn_workspace_bytes(desc, batch.struct, ctypes.byref(a)), "vq_attn_workspace_bytes")
    return a.value


def attn_workspace(desc: VQAttnDesc, batch: AttnBatch, device=None):
    """A workspace for vq_attn_decode and vq_attn_prompt, ready for use: for this batch and every one of no more sequences, new tokens
    and max_len.  device: the batch's, if it is not given."""
    import torch
    return torch.zeros(vq_attn_workspace_bytes(desc, batch), dtype=torch.uint8, device=batch.device if device is None else device)


def _attn(call, name, desc, batch, q, k_pages, v_pages, out, workspace, lse, stream):
    n, heads, dim, kind, gpu = batch.n_tokens, desc.heads, desc.head_dim, _kinds.get(desc.dtype), batch.gpu
    size = 2 * desc.n_pages * desc.kv_heads * desc.page_size * dim
    if lse is not None and (lse.shape != (n, heads) or lse.dtype is not _kinds[VQ_F32] or not lse.is_contiguous() or lse.get_device() != gpu):
        raise ValueError(f"{name}: lse is a contiguous float32 tensor [n_tokens, heads] on the batch's GPU")
    if workspace.get_device() != gpu:
        raise ValueError(f"{name}: the workspace is on the batch's GPU")
    _check(call(desc, batch.struct, q.data_ptr(), _rows(q, n, heads, dim, "q", kind, gpu), _pages(k_pages, size, "k_pages", kind, gpu),
                _pages(v_pages, size, "v_pages", kind, gpu), out.data_ptr(), _rows(out, n, heads, dim, "out", kind, gpu), _ptr(lse),
                _ptr(workspace), workspace.nbytes, _stream(stream)), name)


def vq_attn_decode(desc: VQAttnDesc, batch: AttnBatch, q, k_pages, v_pages, out, workspace, lse=None, stream=None) -> None:
    """q, out: [n_seqs, heads, head_dim] views (strides as vq_strides allows); lse: float32 [n_seqs, heads] or None."""
    _attn(lib().vq_attn_decode, "vq_attn_decode", desc, batch, q, k_pages, v_pages, out, workspace, lse, stream)


def vq_attn_prompt(desc: VQAttnDesc, batch: AttnBatch, q, k_pages, v_pages, out, workspace, lse=None, stream=None) -> None:
    """q, out: [n_tokens, heads, head_dim] views (strides as vq_strides allows); lse: float32 [n_tokens, heads] or None."""
    _attn(lib().vq_attn_prompt, "vq_attn_prompt", desc, batch, q, k_pages, v_pages, out, workspace, lse, stream)
