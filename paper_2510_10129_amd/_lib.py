"""ctypes binding of include/cacheclip.h: same calls, same argument order.

torch is used for device memory and the current HIP stream only.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from array import array
from dataclasses import dataclass
from operator import index
from typing import Optional, Sequence, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_NAME = "libcacheclip.so"

CC_OK = 0
CC_ERR_NULL, CC_ERR_SHAPE, CC_ERR_IDX, CC_ERR_WORKSPACE, CC_ERR_HIP = -1, -2, -3, -4, -5
FLAG_NO_GROUPING, FLAG_CHECK_IDX = 1, 2
K_NAMES = ("colsum", "select", "gather_norm", "qkv", "attn", "oproj", "post_norm", "gate_up", "down",
           "assemble", "copy", "block_scores", "rope_append", "paged_attn", "pages", "page_copy")
ROPE_SCALINGS = ("plain", "linear", "turns", "index")

EXPORTS = (
    "cc_create", "cc_destroy", "cc_set_stream", "cc_last_error", "cc_select",
    "cc_step_column_scores", "cc_recompute_layer", "cc_step_gather_rmsnorm",
    "cc_step_qkv_rope_scatter", "cc_step_sparse_attention", "cc_step_oproj_residual",
    "cc_step_mlp", "cc_profile_enable", "cc_profile_read", "cc_calib_copy", "cc_assemble_cache",
    "cc_step_block_scores", "cc_select_blocks", "cc_debug_set_launch", "cc_select_noalloc",
    "cc_page_work_bytes", "cc_grow_pages", "cc_fork_pages", "cc_free_pages", "cc_compact_pages",
    "cc_step_rope_append", "cc_step_paged_attention",
)


class CacheClipError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"cacheclip status {status}: {msg}")
        self.status = status


class ModelDesc(C.Structure):
    _fields_ = [("d", C.c_int32), ("H_q", C.c_int32), ("H_kv", C.c_int32), ("d_h", C.c_int32),
                ("f", C.c_int32), ("rope_base", C.c_float), ("rms_eps", C.c_float),
                ("N_cap", C.c_int32), ("M_cap", C.c_int32), ("T_cap", C.c_int32)]


class _KV(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("stride_token", C.c_int64),
                ("stride_head", C.c_int64), ("N", C.c_int32)]


class _Chunk(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("len", C.c_int32)]


class _AuxBlock(C.Structure):
    _fields_ = [("attn", C.c_void_p), ("stride_head", C.c_int64), ("stride_row", C.c_int64),
                ("col0", C.c_int32), ("len", C.c_int32)]


class _Weights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("w_in_norm", "w_qkv", "b_qkv", "w_o", "w_post_norm",
                                          "w_gate", "w_up", "w_down")]


class LaunchOverride(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("gemm_tile", "gemm_staged", "gemm_mfma32", "gemm_gm",
                                         "gemm_splitk", "attn_splits")]


class _Pool(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("refs", "table", "len", "status", "work")] + [
        ("work_bytes", C.c_int64), ("stride_table", C.c_int64), ("n_pages", C.c_int32), ("page_size", C.c_int32),
        ("n_seqs", C.c_int32), ("max_pages", C.c_int32), ("refused", C.c_void_p)]


class _PagedKV(C.Structure):
    _fields_ = [("K", C.c_void_p), ("V", C.c_void_p), ("stride_page", C.c_int64), ("stride_token", C.c_int64),
                ("stride_head", C.c_int64)]


class _NewRows(C.Structure):
    _fields_ = [("start", C.c_void_p), ("seq", C.c_void_p), ("n", C.c_int32), ("rows", C.c_int32), ("max_new", C.c_int32)]


class _Rope(C.Structure):
    _fields_ = [("base", C.c_double), ("rot", C.c_int32), ("interleaved", C.c_int32), ("scaling", C.c_int32),
                ("orig_len", C.c_int32), ("factor", C.c_double), ("low", C.c_double), ("high", C.c_double),
                ("mscale", C.c_double)]


def lib_path() -> str:
    return os.path.join(_HERE, _LIB_NAME)


_lib = None


def load_library() -> C.CDLL:
    """Loads the in-tree shared library.  No fallback: a missing library is an error."""
    global _lib
    if _lib is not None:
        return _lib
    # torch first: the process must hold ONE HIP runtime, the one torch's
    # allocator and streams live in; the library binds to whichever
    # libamdhip64.so.7 is already mapped.
    import torch  # noqa: F401
    p = lib_path()
    if not os.path.exists(p):
        raise ImportError(
            f"{p} is missing: build it with `python -m paper_2510_10129_amd.build` "
            "(hipcc, gfx950). There is no CPU fallback.")
    lib = C.CDLL(p)
    vp, i32, i64, u32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32
    lib.cc_create.argtypes = [C.POINTER(vp), C.POINTER(ModelDesc), vp]
    lib.cc_destroy.argtypes = [vp]
    lib.cc_set_stream.argtypes = [vp, vp]
    lib.cc_last_error.argtypes = [vp]
    lib.cc_last_error.restype = C.c_char_p
    lib.cc_select.argtypes = [vp, vp, i32, i32, i64, u32, i32, i32, i32, i32, i32, vp, vp,
                              C.POINTER(i32)]
    lib.cc_select_noalloc.argtypes = [vp, vp, i32, i32, i64, u32, i32, i32, i32, i32, i32, vp, vp]
    lib.cc_step_column_scores.argtypes = [vp, vp, i32, i32, i64, vp]
    lib.cc_recompute_layer.argtypes = [vp, vp, i64, vp, C.POINTER(_KV), vp, i32,
                                       C.POINTER(_Weights), vp, i32]
    lib.cc_step_gather_rmsnorm.argtypes = [vp, vp, i64, vp, i32, vp, vp]
    lib.cc_step_qkv_rope_scatter.argtypes = [vp, vp, i32, vp, vp, vp, C.POINTER(_KV), vp, i32]
    lib.cc_step_sparse_attention.argtypes = [vp, vp, i32, vp, C.POINTER(_KV), vp, i32]
    lib.cc_step_oproj_residual.argtypes = [vp, vp, i32, vp, vp, i64, vp, vp]
    lib.cc_step_mlp.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
    lib.cc_calib_copy.argtypes = [vp, vp, vp, i64]
    lib.cc_assemble_cache.argtypes = [vp, C.POINTER(_Chunk), i32, i32, i64, i64, i32, C.POINTER(_KV)]
    lib.cc_step_block_scores.argtypes = [vp, C.POINTER(_AuxBlock), i32, i32, i32, vp]
    lib.cc_select_blocks.argtypes = [vp, C.POINTER(_AuxBlock), i32, i32, i32, u32, i32, i32, i32, i32, i32,
                                     vp, vp, C.POINTER(i32)]
    lib.cc_debug_set_launch.argtypes = [vp, C.POINTER(LaunchOverride)]
    lib.cc_profile_enable.argtypes = [vp, i32]
    lib.cc_profile_read.argtypes = [vp, C.POINTER(C.c_float), C.POINTER(i32)]
    lib.cc_page_work_bytes.argtypes = [i32, i32]
    lib.cc_grow_pages.argtypes = [vp, C.POINTER(_Pool), C.POINTER(_PagedKV), i32, vp, vp, i32, C.POINTER(i32)]
    lib.cc_fork_pages.argtypes = [vp, C.POINTER(_Pool), vp, vp, i32, C.POINTER(i32)]
    lib.cc_free_pages.argtypes = [vp, C.POINTER(_Pool), vp, i32, C.POINTER(i32)]
    lib.cc_compact_pages.argtypes = [vp, C.POINTER(_Pool), C.POINTER(_PagedKV), i32, C.POINTER(i32)]
    lib.cc_step_rope_append.argtypes = [vp, vp, i64, vp, i64, vp, i64, C.POINTER(_NewRows), vp, C.POINTER(_Pool),
                                        C.POINTER(_PagedKV), C.POINTER(_Rope), vp, i32]
    lib.cc_step_paged_attention.argtypes = [vp, vp, C.POINTER(_NewRows), C.POINTER(_Pool), C.POINTER(_PagedKV), i32, i32, vp,
                                            i32]
    for name in EXPORTS:
        if name != "cc_last_error":
            getattr(lib, name).restype = i32
    lib.cc_page_work_bytes.restype = i64
    _lib = lib
    return lib


def select_noalloc(attn, recomp_bp: int, window: int, tau: int, flags: int, idx_offset: int, n_tail: int,
                   idx_out, n_out, stream=None):
    """cc_select_noalloc: attn cuda fp32 [Q_a, T]; idx_out, n_out preallocated cuda int32.  Enqueues on
    `stream` (default: torch's current stream); raises CacheClipError on a non-zero status."""
    import torch
    lib = load_library()
    Q_a, T = attn.shape
    s = torch.cuda.current_stream().cuda_stream if stream is None else stream
    st = lib.cc_select_noalloc(C.c_void_p(s), attn.data_ptr(), Q_a, T, attn.stride(0), recomp_bp, window, tau,
                               flags, idx_offset, n_tail, idx_out.data_ptr(), n_out.data_ptr())
    if st != CC_OK:
        raise CacheClipError(st, (lib.cc_last_error(None) or b"").decode())


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


@dataclass
class KVLayer:
    """One layer's cache: K, V torch bf16 tensors [N, H_kv, d_h] (last dim contiguous)."""
    K: "object"
    V: "object"

    def c_struct(self) -> _KV:
        K, V = self.K, self.V
        assert K.shape == V.shape and K.stride() == V.stride() and K.stride(2) == 1
        return _KV(K.data_ptr(), V.data_ptr(), K.stride(0), K.stride(1), K.shape[0])


def _i32(t, what: str, dims: int = 1):
    """A device list as the library reads it: int32, unit stride."""
    if t.dtype is not _torch.int32 or t.dim() != dims or (t.shape[-1] > 1 and t.stride(-1) != 1):
        raise ValueError(f"{what} must be an int32 tensor of {dims} dimension(s) with unit stride")
    return t


def _int32(v: int, what: str) -> int:
    """A number as the library takes it: what does not fit would lose its upper half on the way."""
    if not -1 << 31 <= v < 1 << 31:
        raise ValueError(f"{what} must be a 32-bit integer")
    return v


def _bf16(t, what: str):
    if t.dtype is not _torch.bfloat16:
        raise ValueError(f"{what} must be a bfloat16 tensor")
    return t


def _on(pool, *tensors):
    """A host address, or one of another device, would fault the GPU."""
    device = pool.refs.get_device()
    for t in tensors:
        if t.get_device() != device:
            raise ValueError("tensors must lie on the pool's device")


class _Module:
    """torch, imported when first asked for something."""

    def __getattr__(self, name):
        import torch
        global _torch
        _torch = torch
        return getattr(torch, name)


_torch = _Module()


class _Described:
    """What a call is told of a pool, a layer's pages, a batch or a rotary rule: checked and laid out for the library when first
    used, and again after a field was assigned (the tensors themselves are described as they were then: what changes
    their strides or their memory in place is not seen)."""

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        object.__setattr__(self, "_c", None)

    def c_struct(self):
        if self._c is None:
            object.__setattr__(self, "_c", self._describe())
        return self._c


@dataclass
class PagePool(_Described):
    """Pages that sequences hold by reference: refs [n_pages], table [n_seqs, max_pages], len [n_seqs] int32 on
    the device, page_size tokens a page.  status, work and refused (int32 [n_seqs]: 0, or why the last grow that asked for tokens of
    the sequence was refused; `step_rope_append` skips its rows then) are allocated where they are not given.
    `PagePool.empty` makes one with every page free."""
    refs: "object"
    table: "object"
    len: "object"
    page_size: int
    status: "object" = None
    work: "object" = None
    refused: "object" = None

    def __post_init__(self):
        torch = _torch
        _i32(self.refs, "refs"), _i32(self.len, "len")
        if self.status is None:
            self.status = torch.zeros(1, dtype=torch.int32, device=self.refs.device)
        if self.work is None:
            size = load_library().cc_page_work_bytes(self.refs.numel(), self.len.numel())
            self.work = torch.empty(size, dtype=torch.uint8, device=self.refs.device)
        if self.refused is None:
            self.refused = torch.zeros_like(self.len)
            # a context's stream need not wait for torch's, and what the memory held before would read as refusals
            if self.len.is_cuda and not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream(self.len.device).synchronize()
        self._check()

    def _check(self):
        _i32(self.refs, "refs"), _i32(self.table, "table", 2), _i32(self.len, "len")
        if self.table.shape[0] != self.len.shape[0]:
            raise ValueError("table and len must have a row for each sequence")
        if _i32(self.status, "status").numel() < 1:
            raise ValueError("status must hold one value")
        if not self.work.is_contiguous():
            raise ValueError("work must be contiguous")
        if _i32(self.refused, "refused").numel() != self.len.numel():
            raise ValueError("refused must have an entry for each sequence")
        _on(self, self.table, self.len, self.status, self.work, self.refused)

    @classmethod
    def empty(cls, n_pages: int, page_size: int, n_seqs: int, max_pages: int, device="cuda"):
        i32 = dict(dtype=_torch.int32, device=device)
        return cls(_torch.zeros(n_pages, **i32), _torch.full((n_seqs, max_pages), -1, **i32), _torch.zeros(n_seqs, **i32), page_size)

    def _describe(self) -> _Pool:
        self._check()
        return _Pool(self.refs.data_ptr(), self.table.data_ptr(), self.len.data_ptr(), self.status.data_ptr(),
                     self.work.data_ptr(), self.work.numel() * self.work.element_size(), self.table.stride(0),
                     _int32(self.refs.numel(), "the number of pages"), _int32(self.page_size, "page_size"),
                     _int32(self.len.numel(), "the number of sequences"), _int32(self.table.shape[1], "the table's width"),
                     self.refused.data_ptr())


@dataclass
class PagedKV(_Described):
    """One layer's pages: K, V torch bf16 tensors [n_pages, page_size, H_kv, d_h] (last dim contiguous; a view of
    [n_pages, H_kv, page_size, d_h] will do)."""
    K: "object"
    V: "object"

    def _describe(self):
        K, V = _bf16(self.K, "K"), _bf16(self.V, "V")
        if K.dim() != 4 or K.shape != V.shape or K.stride() != V.stride() or K.stride(3) != 1 or K.device != V.device:
            raise ValueError("K and V must be of one shape, [n_pages, page_size, H_kv, d_h], with equal strides, the last of them 1")
        one = _PagedKV(K.data_ptr(), V.data_ptr(), *K.stride()[:3])
        return bytes(one), (*K.shape, K.get_device()), one

    @staticmethod
    def table(kvs: Sequence["PagedKV"], pool: PagePool, model) -> array:
        """A cc_paged_kv (two addresses, three strides) for each of kvs, if their pages are those of the pool and the model."""
        want = (pool.c_struct().n_pages, pool.page_size, model.H_kv, model.d_h, pool.refs.get_device())
        layers = [kv._c or kv.c_struct() for kv in kvs]
        for layer in layers:
            if layer[1] != want:
                raise ValueError(f"K and V are {layer[1][:4]} on device {layer[1][4]}; the pool and the model want {want[:4]} on {want[4]}")
        return array("q", b"".join([layer[0] for layer in layers]))

    def checked(self, pool: PagePool, model) -> _PagedKV:
        self.table((self,), pool, model)
        return self._c[2]


@dataclass
class NewRows(_Described):
    """New tokens of a batch: start int32 [n + 1] on the device, seq int32 [n] or None (sequence b is row b of the table),
    rows of the buffers, and a bound on the rows of one sequence."""
    start: "object"
    seq: "object"
    rows: int
    max_new: int

    def _describe(self) -> _NewRows:
        n = _i32(self.start, "start").numel() - 1
        if n < 0 or (self.seq is not None and _i32(self.seq, "seq").numel() != n):
            raise ValueError("start must have one entry more than seq")
        return _NewRows(self.start.data_ptr(), _ptr(self.seq), _int32(n, "the number of sequences"), _int32(self.rows, "rows"),
                        _int32(self.max_new, "max_new"))


@dataclass
class Rope(_Described):
    """A rotary rule (cc_rope): scaling is "plain", "linear", "turns" or "index"."""
    base: float
    rot: int
    interleaved: bool = False
    scaling: str = "plain"
    factor: float = 1.0
    orig_len: int = 0
    low: float = 1.0
    high: float = 4.0
    mscale: float = 1.0

    def _describe(self) -> _Rope:
        if self.scaling not in ROPE_SCALINGS:
            raise ValueError(f"scaling must be one of {ROPE_SCALINGS}")
        return _Rope(self.base, _int32(self.rot, "rot"), int(bool(self.interleaved)), ROPE_SCALINGS.index(self.scaling),
                     _int32(self.orig_len, "orig_len"), self.factor, self.low, self.high, self.mscale)


@dataclass
class LayerWeights:
    """Device bf16 tensors of one layer (b_qkv may be None)."""
    w_in_norm: "object"
    w_qkv: "object"
    b_qkv: "object"
    w_o: "object"
    w_post_norm: "object"
    w_gate: "object"
    w_up: "object"
    w_down: "object"

    def c_struct(self) -> _Weights:
        return _Weights(*[_ptr(getattr(self, n)) for n, _ in _Weights._fields_])


class Context:
    """Owns a cc_ctx.  Methods mirror the C entry points one to one."""
    _device = None                          # index of the GPU that it was created on

    def __init__(self, d, H_q, H_kv, d_h, f, rope_base, rms_eps, N_cap, M_cap, T_cap, stream=None):
        import torch
        self._lib = load_library()
        self.desc = ModelDesc(d, H_q, H_kv, d_h, f, rope_base, rms_eps, N_cap, M_cap, T_cap)
        self._h = C.c_void_p()
        s = torch.cuda.current_stream().cuda_stream if stream is None else stream
        st = self._lib.cc_create(C.byref(self._h), C.byref(self.desc), C.c_void_p(s))
        if st != CC_OK:
            raise CacheClipError(st, (self._lib.cc_last_error(None) or b"").decode())
        self._device = torch.cuda.current_device()

    @classmethod
    def for_model(cls, model, N_cap, M_cap, T_cap, stream=None):
        return cls(model.d, model.H_q, model.H_kv, model.d_h, model.f, model.rope_base,
                   model.rms_eps, N_cap, M_cap, T_cap, stream)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h.value:
            self._lib.cc_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != CC_OK:
            raise CacheClipError(st, (self._lib.cc_last_error(self._h) or b"").decode())

    def set_stream(self, stream: int):
        self._check(self._lib.cc_set_stream(self._h, C.c_void_p(stream)))

    # ---- selection ----
    def select(self, attn, recomp_bp: int, window: int, tau: int = 0, flags: int = 0,
               idx_offset: int = 0, n_tail: int = 0, idx_out=None, n_out=None,
               sync: bool = True) -> Tuple["object", Optional[int]]:
        """attn: cuda fp32 [Q_a, T].  Returns (idx_out tensor, count or None)."""
        import torch
        Q_a, T = attn.shape
        if idx_out is None:
            idx_out = torch.empty(T + n_tail, dtype=torch.int32, device=attn.device)
        if n_out is None:
            n_out = torch.empty(1, dtype=torch.int32, device=attn.device)
        host = C.c_int32(-1)
        self._check(self._lib.cc_select(self._h, attn.data_ptr(), Q_a, T, attn.stride(0), recomp_bp,
                                        window, tau, flags, idx_offset, n_tail, idx_out.data_ptr(),
                                        n_out.data_ptr(), C.byref(host) if sync else None))
        return idx_out, (host.value if sync else None)

    def step_column_scores(self, attn, score):
        Q_a, T = attn.shape
        self._check(self._lib.cc_step_column_scores(self._h, attn.data_ptr(), Q_a, T, attn.stride(0),
                                                    score.data_ptr()))

    @staticmethod
    def _aux_blocks(blocks):
        """blocks: sequence of (attn cuda fp32 [H, Q_a, W], col0, len)."""
        first = None
        flat = []
        for a, col0, ln in blocks:
            shape, st = a.shape, a.stride()
            if len(shape) != 3 or st[2] != 1:
                raise ValueError("a block must be [H, Q_a, W] with unit column stride")
            if first is None:
                first = shape
            elif shape[0] != first[0] or shape[1] != first[1]:
                raise ValueError("all blocks must have the same H and Q_a")
            if col0 + ln > shape[2]:
                raise ValueError("col0 + len exceeds the block's width")
            flat += (a.data_ptr(), st[0], st[1], col0, ln)
        if first is None:
            return (_AuxBlock * 0)(), None, None
        n = len(flat) // 5
        try:                                    # an _AuxBlock is an address, two strides and two 32-bit counts
            packed = struct.pack("Pqqii" * n, *flat)
        except struct.error as e:
            raise TypeError(f"col0 and len must be 32-bit integers: {e}") from None
        return (_AuxBlock * n).from_buffer_copy(packed), first[0], first[1]

    def step_block_scores(self, blocks, score):
        arr, H, Q_a = self._aux_blocks(blocks)
        self._check(self._lib.cc_step_block_scores(self._h, arr, len(blocks), H, Q_a, score.data_ptr()))

    def select_blocks(self, blocks, recomp_bp: int, window: int, tau: int = 0, flags: int = 0,
                      idx_offset: int = 0, n_tail: int = 0, idx_out=None, n_out=None,
                      sync: bool = True) -> Tuple["object", Optional[int]]:
        """blocks: sequence of (attn cuda fp32 [H, Q_a, W], col0, len).  Returns (idx_out, count or None)."""
        import torch
        arr, H, Q_a = self._aux_blocks(blocks)
        if idx_out is None:
            idx_out = torch.empty(sum(b[2] for b in blocks) + n_tail, dtype=torch.int32, device=blocks[0][0].device)
        if n_out is None:
            n_out = torch.empty(1, dtype=torch.int32, device=blocks[0][0].device)
        host = C.c_int32(-1)
        self._check(self._lib.cc_select_blocks(self._h, arr, len(blocks), H, Q_a, recomp_bp, window, tau,
                                               flags, idx_offset, n_tail, idx_out.data_ptr(),
                                               n_out.data_ptr(), C.byref(host) if sync else None))
        return idx_out, (host.value if sync else None)

    # ---- layer ----
    def recompute_layer(self, hidden, gather_idx, kv: KVLayer, idx, M: int, w: LayerWeights, out,
                        flags: int = 0):
        kvs, ws = kv.c_struct(), w.c_struct()
        self._check(self._lib.cc_recompute_layer(self._h, hidden.data_ptr(), hidden.shape[0],
                                                 _ptr(gather_idx), C.byref(kvs), idx.data_ptr(), M,
                                                 C.byref(ws), out.data_ptr(), flags))

    def step_gather_rmsnorm(self, hidden, gather_idx, M, w_norm, xn):
        self._check(self._lib.cc_step_gather_rmsnorm(self._h, hidden.data_ptr(), hidden.shape[0],
                                                     _ptr(gather_idx), M, w_norm.data_ptr(),
                                                     xn.data_ptr()))

    def step_qkv_rope_scatter(self, xn, M, idx, w_qkv, b_qkv, kv: KVLayer, q_out, flags: int = 0):
        kvs = kv.c_struct()
        self._check(self._lib.cc_step_qkv_rope_scatter(self._h, xn.data_ptr(), M, idx.data_ptr(),
                                                       w_qkv.data_ptr(), _ptr(b_qkv), C.byref(kvs),
                                                       q_out.data_ptr(), flags))

    def step_sparse_attention(self, q, M, idx, kv: KVLayer, o, flags: int = 0):
        kvs = kv.c_struct()
        self._check(self._lib.cc_step_sparse_attention(self._h, q.data_ptr(), M, idx.data_ptr(),
                                                       C.byref(kvs), o.data_ptr(), flags))

    def step_oproj_residual(self, o, M, w_o, hidden, gather_idx, y):
        self._check(self._lib.cc_step_oproj_residual(self._h, o.data_ptr(), M, w_o.data_ptr(),
                                                     hidden.data_ptr(), hidden.shape[0],
                                                     _ptr(gather_idx), y.data_ptr()))

    def step_mlp(self, y, M, w_post_norm, w_gate, w_up, w_down, out):
        self._check(self._lib.cc_step_mlp(self._h, y.data_ptr(), M, w_post_norm.data_ptr(),
                                          w_gate.data_ptr(), w_up.data_ptr(), w_down.data_ptr(),
                                          out.data_ptr()))

    # ---- cache assembly ----
    def assemble_cache(self, chunk_K: Sequence, chunk_V: Sequence, P: int, n_tail: int, dst: KVLayer):
        """chunk_K[c], chunk_V[c]: cuda bf16 [P + L_c, H_kv, d_h], all with the same strides."""
        n, P = len(chunk_K), index(P)
        st = chunk_K[0].stride()
        assert st[2] == 1
        flat = []                               # a _Chunk is two addresses and a length padded to 8 bytes
        for K, V in zip(chunk_K, chunk_V):
            shape = K.shape
            assert shape == V.shape and K.stride() == st and V.stride() == st
            flat += (K.data_ptr(), V.data_ptr(), (shape[0] - P) & 0xFFFFFFFF)
        arr = (_Chunk * n).from_buffer(array("Q", flat))
        kvs = dst.c_struct()
        self._check(self._lib.cc_assemble_cache(self._h, arr, n, P, st[0], st[1], n_tail, C.byref(kvs)))

    # ---- the paged cache of the answer phase ----
    def _layers(self, pool: PagePool, kvs: Sequence[PagedKV]):
        n = len(kvs)
        return (_PagedKV * n).from_buffer(PagedKV.table(kvs, pool, self.desc)) if n else None, n

    def _pool(self, pool: PagePool) -> _Pool:
        """A pool's tensors lie together, and what comes with them lies there too (_on): on the host, perhaps."""
        if pool.refs.get_device() != self._device:
            raise ValueError("the pool must lie on the context's GPU")
        return pool.c_struct()

    def _pages(self, call, pool: PagePool, sync: bool, *args):
        p, host = self._pool(pool), C.c_int32(0)
        self._check(call(self._h, C.byref(p), *args, C.byref(host) if sync else None))

    @staticmethod
    def _seqs(pool: PagePool, a, b):
        if _i32(a, "sequences").numel() != _i32(b, "their second list").numel():
            raise ValueError("the two lists must have the same length")
        _on(pool, a, b)
        return a.data_ptr(), b.data_ptr(), a.numel()

    def grow_pages(self, pool: PagePool, kvs: Sequence[PagedKV], seq, n_new, sync: bool = True):
        """Room for n_new[i] more tokens of sequence seq[i].  sync: waits for the device's status and raises on an error;
        without it pool.status says how the call ended (so for the three calls below), until the next of them, and pool.refused
        whose tokens have no room, until a grow of the sequence is made."""
        arr, n_layers = self._layers(pool, kvs)
        self._pages(self._lib.cc_grow_pages, pool, sync, arr, n_layers, *self._seqs(pool, seq, n_new))

    def fork_pages(self, pool: PagePool, src, dst, sync: bool = True):
        self._pages(self._lib.cc_fork_pages, pool, sync, *self._seqs(pool, src, dst))

    def free_pages(self, pool: PagePool, seq, sync: bool = True):
        _on(pool, _i32(seq, "seq"))
        self._pages(self._lib.cc_free_pages, pool, sync, seq.data_ptr(), seq.numel())

    def compact_pages(self, pool: PagePool, kvs: Sequence[PagedKV], sync: bool = True):
        self._pages(self._lib.cc_compact_pages, pool, sync, *self._layers(pool, kvs))

    def _row_buffer(self, t, what: str, rows: int, width: int):
        st = _bf16(t, what).stride()
        if t.shape != (rows, width) or st[1] != 1:
            raise ValueError(f"{what} must be [{rows}, {width}] with unit column stride")
        return st[0] if rows > 1 else width

    def step_rope_append(self, q, k, v, new: NewRows, pool: PagePool, kv: PagedKV, rope: Rope, q_out, pos=None, flags: int = 0):
        """q [rows, H_q*d_h], k, v [rows, H_kv*d_h] cuda bf16 (column slices of one product will do) -> q_out, pages of kv.  Rows of
        a sequence whose last grow was refused (pool.refused) are skipped."""
        m, rows, row = self.desc, new.rows, self._row_buffer
        d_h = m.d_h
        nq, nk = m.H_q * d_h, m.H_kv * d_h
        st_q, st_k, st_v = row(q, "q", rows, nq), row(k, "k", rows, nk), row(v, "v", rows, nk)
        if row(q_out, "q_out", rows, nq) != nq:
            raise ValueError("q_out must be contiguous")
        if pos is not None:
            if _i32(pos, "pos").numel() < rows:
                raise ValueError("pos must have an entry for each row")
            _on(pool, pos)
        _on(pool, q, k, v, q_out, new.start) if new.seq is None else _on(pool, q, k, v, q_out, new.start, new.seq)
        p, kvs, r, rule = self._pool(pool), kv.checked(pool, m), new.c_struct(), rope.c_struct()
        self._check(self._lib.cc_step_rope_append(self._h, q.data_ptr(), st_q, k.data_ptr(), st_k, v.data_ptr(), st_v, C.byref(r),
                                                  _ptr(pos), C.byref(p), C.byref(kvs), C.byref(rule), q_out.data_ptr(), flags))

    def step_paged_attention(self, q, new: NewRows, pool: PagePool, kv: PagedKV, o, window: int = 0, sinks: int = 0, flags: int = 0):
        """q, o cuda bf16 [rows, H_q*d_h], contiguous."""
        m = self.desc
        for t, what in ((q, "q"), (o, "o")):
            if self._row_buffer(t, what, new.rows, m.H_q * m.d_h) != m.H_q * m.d_h:
                raise ValueError(f"{what} must be contiguous")
        _int32(window, "window"), _int32(sinks, "sinks")
        _on(pool, q, o, new.start, *(() if new.seq is None else (new.seq,)))
        p, kvs, r = self._pool(pool), kv.checked(pool, m), new.c_struct()
        self._check(self._lib.cc_step_paged_attention(self._h, q.data_ptr(), C.byref(r), C.byref(p), C.byref(kvs), window, sinks,
                                                      o.data_ptr(), flags))

    # ---- measurement support ----
    def calib_copy(self, dst, src):
        self._check(self._lib.cc_calib_copy(self._h, dst.data_ptr(), src.data_ptr(),
                                            src.numel() * src.element_size()))

    # ---- test support ----
    def debug_set_launch(self, gemm_tile: str = "", gemm_staged: int = 0, gemm_mfma32: bool = False,
                         gemm_gm: int = 0, gemm_splitk: int = 0, attn_splits: int = 0):
        """Overrides the launch shapes until the next call; no arguments = the library's own choices."""
        o = LaunchOverride(ord(gemm_tile) if gemm_tile else 0, int(gemm_staged), int(gemm_mfma32), gemm_gm,
                           gemm_splitk, attn_splits)
        self._check(self._lib.cc_debug_set_launch(self._h, C.byref(o)))

    # ---- timing ----
    def profile_enable(self, on: bool):
        self._check(self._lib.cc_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        n = len(K_NAMES)
        ms = (C.c_float * n)()
        cnt = (C.c_int32 * n)()
        self._check(self._lib.cc_profile_read(self._h, ms, cnt))
        return {K_NAMES[i]: (ms[i], cnt[i]) for i in range(n)}
