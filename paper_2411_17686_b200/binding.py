"""ctypes binding of libficoco (argument marshalling only; every step runs in the library).

PyTorch is used for device memory and streams.  Function names mirror the C ABI declared in
``include/ficoco.h``.  Importing this module never loads the library; the first call does,
and raises if ``libficoco.so`` has not been built (``python -m paper_2411_17686_b200.build``).
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple, Union

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libficoco.so")

FICOCO_FP32, FICOCO_BF16 = 0, 1
FICOCO_HAS_CLS, FICOCO_LOCAL_PENALTY, FICOCO_AVERAGE_COMPRESSION, FICOCO_BACK_TO_BACK, FICOCO_CONVERGENT = 1, 2, 4, 8, 16
FICOCO_CAUSAL = 1
KCAP = 16

INSPECT = {
    "rnorm": (0, np.float32, 1), "score_raw": (1, np.float32, 1), "score": (2, np.float32, 1),
    "src_idx": (3, np.int32, 1), "tgt_idx": (4, np.int32, 1), "corr_cnt": (5, np.int32, 1),
    "corr_tgt": (6, np.int32, KCAP), "corr_w": (7, np.float32, KCAP), "corr_c": (8, np.float32, KCAP),
    "tau": (9, np.float32, 1),
}

EXPORTS = [
    "ficoco_create", "ficoco_destroy", "ficoco_strerror", "ficoco_last_cuda_error",
    "ficoco_default_params", "ficoco_v_reduce", "ficoco_l_reduce", "ficoco_v_reduce_host",
    "ficoco_l_reduce_host", "ficoco_status", "ficoco_inspect", "ficoco_last_launch_count",
    "ficoco_profile", "ficoco_profile_read", "ficoco_vision_redundancy_noalloc",
    "ficoco_equivalent_token", "ficoco_v_reduce_relation", "ficoco_debug_waits", "ficoco_v_reduce_schedule",
    "ficoco_v_plan", "ficoco_debug_barrier_wait",
    "ficoco_cache_append", "ficoco_cache_attention", "ficoco_cache_weights", "ficoco_cache_copy", "ficoco_cache_compact",
    "ficoco_pool_create", "ficoco_pool_destroy", "ficoco_pool_free_pages", "ficoco_pool_take", "ficoco_pool_give",
    "ficoco_pool_fork",
]


class ficoco_params(C.Structure):
    _fields_ = [("lambda_", C.c_double), ("beta", C.c_double), ("gamma", C.c_double),
                ("eps", C.c_double), ("penalty_coef", C.c_double), ("window", C.c_int),
                ("max_targets", C.c_int), ("flags", C.c_uint), ("reserved", C.c_int)]


class ficoco_v_args(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("seqlens", C.c_void_p), ("attn", C.c_void_p),
                ("grid_h", C.c_void_p), ("grid_w", C.c_void_p), ("pos", C.c_void_p),
                ("keep", C.c_void_p), ("out_tokens", C.c_void_p), ("kept_idx", C.c_void_p),
                ("pos_out", C.c_void_p), ("scores_out", C.c_void_p),
                ("dtype", C.c_int), ("batch", C.c_int), ("n_tokens", C.c_int), ("dim", C.c_int),
                ("heads", C.c_int), ("n_grid", C.c_int), ("n_keep", C.c_int), ("reserved", C.c_int),
                ("out_cu_seqlens", C.c_void_p)]


class ficoco_l_args(C.Structure):
    _fields_ = [("tokens", C.c_void_p), ("attn_t2v", C.c_void_p), ("keep", C.c_void_p),
                ("out_tokens", C.c_void_p), ("kept_idx", C.c_void_p), ("scores_out", C.c_void_p),
                ("dtype", C.c_int), ("batch", C.c_int), ("n_vision", C.c_int), ("n_text", C.c_int),
                ("dim", C.c_int), ("heads", C.c_int), ("n_keep", C.c_int), ("reserved", C.c_int)]


class ficoco_cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("page_table", C.c_void_p), ("lengths", C.c_void_p), ("table_stride", C.c_longlong),
                ("n_pages", C.c_int), ("page_size", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int),
                ("batch", C.c_int), ("max_pages", C.c_int)]


class ficoco_append_args(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("cu_rows", C.c_void_p), ("k_stride", C.c_longlong),
                ("v_stride", C.c_longlong), ("dtype", C.c_int), ("rows", C.c_int)]


class ficoco_attention_args(C.Structure):
    _fields_ = [("q", C.c_void_p), ("cu_rows", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p),
                ("q_stride", C.c_longlong), ("scale", C.c_float), ("dtype", C.c_int), ("rows", C.c_int),
                ("heads", C.c_int), ("window", C.c_int), ("sinks", C.c_int), ("flags", C.c_uint)]


class ficoco_compact_args(C.Structure):
    _fields_ = [("to_table", C.c_void_p), ("kept", C.c_void_p), ("cu_kept", C.c_void_p), ("lengths_out", C.c_void_p),
                ("to_stride", C.c_longlong), ("to_pages", C.c_int), ("n_kept", C.c_int), ("first", C.c_int),
                ("reserved", C.c_int)]


class FicocoError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libficoco error {code}: {msg}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Load libficoco.so; fails loudly when it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2411_17686_b200.build` "
            "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    lib.ficoco_create.argtypes = [C.POINTER(C.c_void_p), C.c_int, C.c_longlong, C.c_int, C.c_int, C.c_int]
    lib.ficoco_destroy.argtypes = [C.c_void_p]
    lib.ficoco_strerror.argtypes = [C.c_int]
    lib.ficoco_strerror.restype = C.c_char_p
    lib.ficoco_last_cuda_error.argtypes = [C.c_void_p]
    lib.ficoco_default_params.argtypes = [C.POINTER(ficoco_params)]
    lib.ficoco_default_params.restype = None
    lib.ficoco_equivalent_token.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int,
                                            C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    lib.ficoco_v_reduce.argtypes = [C.c_void_p, C.POINTER(ficoco_v_args), C.POINTER(ficoco_params), C.c_void_p]
    lib.ficoco_l_reduce.argtypes = [C.c_void_p, C.POINTER(ficoco_l_args), C.POINTER(ficoco_params), C.c_void_p]
    lib.ficoco_v_reduce_relation.argtypes = [C.c_void_p, C.POINTER(ficoco_v_args), C.c_void_p, C.c_int,
                                             C.POINTER(ficoco_params), C.c_void_p]
    lib.ficoco_v_reduce_host.argtypes = [C.c_void_p, C.POINTER(ficoco_v_args), C.POINTER(ficoco_params)]
    lib.ficoco_l_reduce_host.argtypes = [C.c_void_p, C.POINTER(ficoco_l_args), C.POINTER(ficoco_params)]
    lib.ficoco_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int)]
    lib.ficoco_debug_waits.argtypes = [C.c_void_p, C.c_longlong, C.c_int]
    lib.ficoco_debug_barrier_wait.argtypes = [C.c_void_p, C.POINTER(C.c_longlong)]
    lib.ficoco_v_plan.argtypes = [C.c_void_p, C.POINTER(ficoco_v_args), C.POINTER(ficoco_params), C.c_void_p]
    lib.ficoco_v_reduce_schedule.argtypes = [C.c_void_p, C.POINTER(ficoco_v_args), C.c_int, C.c_void_p, C.c_void_p,
                                             C.POINTER(ficoco_params), C.c_void_p]
    lib.ficoco_inspect.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_size_t, C.POINTER(C.c_size_t)]
    lib.ficoco_last_launch_count.argtypes = [C.c_void_p]
    lib.ficoco_profile.argtypes = [C.c_void_p, C.c_int]
    lib.ficoco_profile_read.argtypes = [C.c_void_p, C.c_int, C.c_char_p, C.c_int, C.POINTER(C.c_double),
                                        C.POINTER(C.c_longlong)]
    lib.ficoco_vision_redundancy_noalloc.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_uint,
                                                     C.c_void_p, C.c_void_p]
    lib.ficoco_cache_append.argtypes = [C.c_void_p, C.POINTER(ficoco_cache), C.POINTER(ficoco_append_args), C.c_void_p]
    lib.ficoco_cache_attention.argtypes = [C.c_void_p, C.POINTER(ficoco_cache), C.POINTER(ficoco_attention_args), C.c_void_p]
    lib.ficoco_cache_weights.argtypes = [C.c_void_p, C.POINTER(ficoco_cache), C.POINTER(ficoco_attention_args), C.c_int,
                                         C.c_int, C.c_int, C.c_void_p, C.c_void_p]
    lib.ficoco_cache_copy.argtypes = [C.c_void_p, C.POINTER(ficoco_cache), C.c_void_p, C.c_void_p, C.c_int, C.c_void_p]
    lib.ficoco_cache_compact.argtypes = [C.c_void_p, C.POINTER(ficoco_cache), C.POINTER(ficoco_compact_args), C.c_void_p]
    lib.ficoco_pool_create.argtypes = [C.POINTER(C.c_void_p), C.c_int]
    lib.ficoco_pool_destroy.argtypes = [C.c_void_p]
    lib.ficoco_pool_free_pages.argtypes = [C.c_void_p]
    lib.ficoco_pool_take.argtypes = [C.c_void_p, C.c_int, C.c_void_p]
    lib.ficoco_pool_give.argtypes = [C.c_void_p, C.c_int, C.c_void_p]
    lib.ficoco_pool_fork.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.POINTER(C.c_int),
                                     C.POINTER(C.c_int)]
    _lib = lib
    return lib


def ficoco_default_params() -> ficoco_params:
    p = ficoco_params()
    load_library().ficoco_default_params(C.byref(p))
    return p


def make_params(lam=0.35, beta=0.6, gamma=0.6, eps=0.998, penalty_coef=2.0, window=2,
                max_targets=-1, has_cls=True, local_penalty=True, average_compression=False,
                back_to_back=False, convergent=False) -> ficoco_params:
    p = ficoco_params()
    p.lambda_, p.beta, p.gamma, p.eps, p.penalty_coef = lam, beta, gamma, eps, penalty_coef
    p.window, p.max_targets = window, -1 if max_targets is None else max_targets
    p.flags = ((FICOCO_HAS_CLS if has_cls else 0) | (FICOCO_LOCAL_PENALTY if local_penalty else 0) |
               (FICOCO_AVERAGE_COMPRESSION if average_compression else 0) |
               (FICOCO_BACK_TO_BACK if back_to_back else 0) | (FICOCO_CONVERGENT if convergent else 0))
    return p


def _check(ctx, rc: int) -> None:
    if rc != 0:
        lib = load_library()
        msg = lib.ficoco_strerror(rc).decode()
        if rc == -5 and ctx is not None:
            msg += f" (cudaError {lib.ficoco_last_cuda_error(ctx)})"
        raise FicocoError(rc, msg)


def _int_array(v: Union[int, Sequence[int]]) -> Tuple[np.ndarray, int]:
    a = np.ascontiguousarray(np.atleast_1d(np.asarray(v, dtype=np.int32)))
    return a, int(a.shape[0])


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.bfloat16:
        return FICOCO_BF16
    if t.dtype == torch.float32:
        return FICOCO_FP32
    raise TypeError(f"tokens must be bf16 or fp32, got {t.dtype}")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _shape_key(v):
    """Hashable form of a per-image count or list of counts."""
    if v is None or isinstance(v, int):
        return v
    return tuple(v) if isinstance(v, (list, tuple)) else tuple(np.atleast_1d(np.asarray(v)).tolist())


def _current_stream(dev) -> int:
    import torch
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    if raw is not None and dev.index is not None:
        return raw(dev.index)
    return torch.cuda.current_stream(dev).cuda_stream


@dataclass
class _Shapes:
    """The marshalled shapes of a call: the struct with everything but the data pointers filled in, the int32
    arrays its pointers refer to, and the sizes of the outputs."""
    args: "object"
    arrays: "object"
    out_rows: List[int]
    n_out: int
    n_keep: int
    n_patch: int


_SHAPES_KEPT = 64       # marshalled shapes a context remembers


@dataclass
class VResult:
    out_tokens: "object"
    kept_idx: "object"
    pos_out: "object"
    scores: "object"
    out_rows: List[int]   # output rows per image


_torch = None


def _load_torch():
    """torch, imported by the first call that needs it (an import statement in each of the cache's calls took a twentieth of them)."""
    global _torch
    if _torch is None:
        import torch
        _torch = torch
    return _torch


class PagedCache:
    """The 8-bit paged key/value cache of one decoder layer: tensors that the caller owns, described once.

    ``k_codes`` / ``v_codes``: cuda float8_e4m3fn (or uint8) [n_pages, kv_heads, page_size, head_dim];
    ``k_scale`` / ``v_scale``: cuda fp32 [n_pages, kv_heads]; ``page_table``: cuda int32 [batch, max_pages] (rows may be
    strided); ``lengths``: cuda int32 [batch].  Their contents may change between calls, the tensors may not: a cache with other
    tensors is another ``PagedCache``."""

    __slots__ = ("k_codes", "v_codes", "k_scale", "v_scale", "page_table", "lengths", "struct", "device", "scale")

    def __init__(self, k_codes, v_codes, k_scale, v_scale, page_table, lengths):
        import torch
        self.device = k_codes.device
        n_pages, kv_heads, page_size, head_dim = k_codes.shape
        for name, t, dtypes, shape in (
                ("k_codes", k_codes, (torch.float8_e4m3fn, torch.uint8), (n_pages, kv_heads, page_size, head_dim)),
                ("v_codes", v_codes, (torch.float8_e4m3fn, torch.uint8), (n_pages, kv_heads, page_size, head_dim)),
                ("k_scale", k_scale, (torch.float32,), (n_pages, kv_heads)),
                ("v_scale", v_scale, (torch.float32,), (n_pages, kv_heads)),
                ("page_table", page_table, (torch.int32,), (page_table.shape[0], page_table.shape[-1])),
                ("lengths", lengths, (torch.int32,), (page_table.shape[0],))):
            if t.dtype not in dtypes:
                raise TypeError(f"{name} must be {' or '.join(map(str, dtypes))}, got {t.dtype}")
            if tuple(t.shape) != shape:
                raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")
            if t.device != self.device or not t.is_cuda:
                raise ValueError(f"{name} must be on the cuda device of k_codes, got {t.device}")
            if not (t.stride(-1) == 1 if name == "page_table" else t.is_contiguous()):
                raise ValueError(f"{name} must be contiguous")
        self.k_codes, self.v_codes, self.k_scale, self.v_scale = k_codes, v_codes, k_scale, v_scale
        self.page_table, self.lengths = page_table, lengths
        self.struct = ficoco_cache(k_codes.data_ptr(), v_codes.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                                   page_table.data_ptr(), lengths.data_ptr(), page_table.stride(0), n_pages, page_size,
                                   kv_heads, head_dim, page_table.shape[0], page_table.shape[1])
        self.scale = head_dim ** -0.5

    @classmethod
    def empty(cls, n_pages: int, kv_heads: int, page_size: int, head_dim: int, batch: int, max_pages: int,
              device="cuda:0") -> "PagedCache":
        """A cache of ``batch`` sequences without tokens."""
        import torch
        codes = [torch.zeros((n_pages, kv_heads, page_size, head_dim), dtype=torch.uint8, device=device)
                 .view(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.ones((n_pages, kv_heads), dtype=torch.float32, device=device) for _ in range(2)]
        return cls(codes[0], codes[1], scales[0], scales[1],
                   torch.zeros((batch, max_pages), dtype=torch.int32, device=device),
                   torch.zeros((batch,), dtype=torch.int32, device=device))

    @property
    def batch(self) -> int:
        return self.struct.batch


class PagePool:
    """Which pages of a cache are free, and how many sequences hold each of the others (host bookkeeping, ficoco_pool_*)."""

    def __init__(self, n_pages: int):
        self.lib = load_library()
        h = C.c_void_p()
        _check(None, self.lib.ficoco_pool_create(C.byref(h), n_pages))
        self.h = h

    def close(self) -> None:
        if getattr(self, "h", None):
            self.lib.ficoco_pool_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def free_pages(self) -> int:
        return int(self.lib.ficoco_pool_free_pages(self.h))

    def take(self, n: int) -> List[int]:
        a = np.zeros(max(n, 1), dtype=np.int32)
        _check(None, self.lib.ficoco_pool_take(self.h, n, a.ctypes.data))
        return a[:n].tolist()

    def give(self, pages: Sequence[int]) -> None:
        a = np.ascontiguousarray(np.asarray(pages, dtype=np.int32))
        _check(None, self.lib.ficoco_pool_give(self.h, a.shape[0], a.ctypes.data))

    def fork(self, pages: Sequence[int], page_size: int, length: int) -> Tuple[List[int], Optional[Tuple[int, int]]]:
        """The forked sequence's pages, and the (from, to) pair to copy with ``ficoco_cache_copy`` (None: nothing to copy)."""
        n = -(-length // page_size) if page_size > 0 else 0
        a = np.ascontiguousarray(np.asarray(pages, dtype=np.int32))
        if a.shape[0] < n:
            raise ValueError(f"{length} tokens need {n} pages, got {a.shape[0]}")
        out = np.zeros(max(n, 1), dtype=np.int32)
        src, dst = C.c_int(-1), C.c_int(-1)
        _check(None, self.lib.ficoco_pool_fork(self.h, page_size, length, a.ctypes.data, out.ctypes.data, C.byref(src),
                                               C.byref(dst)))
        return out[:n].tolist(), (None if src.value < 0 else (src.value, dst.value))


def _c_ints(**values: int) -> None:
    """Refuses what a C int does not hold (ctypes would cut it to its low 32 bits)."""
    for name, x in values.items():
        if not -(1 << 31) <= x < 1 << 31:
            raise ValueError(f"{name} = {x} is no 32-bit integer")


def _int32(name: str, t, n: Optional[int] = None, device=None) -> int:
    """Address of a contiguous cuda int32 tensor, on ``device`` if one is given."""
    if t.dtype is not _load_torch().int32 or not t.is_cuda or not t.is_contiguous() or (n is not None and t.numel() != n) or \
            (device is not None and t.device != device):
        raise ValueError(f"{name} must be a contiguous cuda int32 tensor" + (f" of {n} values" if n is not None else "") +
                         (f" on {device}" if device is not None else ""))
    return t.data_ptr()


def _rows3(name: str, t, dim: int) -> int:
    """Row stride of [rows, heads, dim] whose last two dimensions are contiguous."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != dim:
        raise ValueError(f"{name} must be [rows, heads, {dim}], got {tuple(shape)}")
    stride = t.stride()
    if not t.is_cuda or (shape[0] > 0 and (stride[2] != 1 or (stride[1] != dim and shape[1] > 1))):
        raise ValueError(f"{name} must be a cuda tensor with contiguous heads")
    return stride[0] if shape[0] > 1 else shape[1] * dim


def _new(like, shape, dtype):
    """A contiguous tensor on the device of ``like`` (half the time of torch.empty with a shape)."""
    strides, n = [], 1
    for x in reversed(shape):
        strides.append(n)
        n *= x
    return _load_torch().empty_strided(shape, strides[::-1], dtype=dtype, device=like.device)


class Context:
    """Owns one ficoco_ctx.  Methods mirror the C entry points."""

    def __init__(self, max_tokens: int, max_dim: int, max_batch: int, max_text: int = 0, device: int = 0):
        self.lib = load_library()
        self.device = device
        h = C.c_void_p()
        _check(None, self.lib.ficoco_create(C.byref(h), device, max_tokens, max_dim, max_batch, max_text))
        self.h = h
        # Marshalled shapes of earlier calls (a program meets few; the oldest are dropped).  Rebuilding the arrays
        # and structs took 20 us of every call, more than the kernels of a small image take.
        self._shapes = {}

    def _remember(self, key, make) -> _Shapes:
        s = self._shapes.get(key)
        if s is None:
            s = make()
            while len(self._shapes) >= _SHAPES_KEPT:
                self._shapes.pop(next(iter(self._shapes)), None)
            self._shapes[key] = s
        return s

    def _v_shapes(self, dim, dtype, rows, keep, grid_h, grid_w, heads, n_tokens, seqlens, flags) -> _Shapes:
        cls = 1 if (flags & FICOCO_HAS_CLS) else 0
        conv = bool(flags & FICOCO_CONVERGENT)          # one more row per image that discards something

        def make():
            keep_a, n_keep = _int_array(keep)
            gh_a, n_gh = _int_array(grid_h)
            gw_a, n_gw = _int_array(grid_w)
            assert n_gh == n_gw
            if seqlens is not None:
                sl, batch = _int_array(seqlens)
            else:
                sl, batch = None, rows // n_tokens if n_tokens else 0
            keeps = [int(keep_a[0 if n_keep == 1 else b]) for b in range(batch)]
            ntoks = [int(sl[b]) if sl is not None else n_tokens for b in range(batch)]
            out_rows = [cls + k + (1 if conv and n - cls - k > 0 else 0) for k, n in zip(keeps, ntoks)]
            a = ficoco_v_args()
            a.seqlens = sl.ctypes.data if sl is not None else None
            a.grid_h, a.grid_w, a.keep = gh_a.ctypes.data, gw_a.ctypes.data, keep_a.ctypes.data
            a.dtype, a.batch, a.n_tokens, a.dim, a.heads = dtype, batch, n_tokens, dim, heads
            a.n_grid, a.n_keep = n_gh, n_keep
            return _Shapes(a, (keep_a, gh_a, gw_a, sl), out_rows, sum(out_rows), sum(keeps), sum(ntoks) - cls * batch)

        key = ("v", dim, dtype, rows, _shape_key(keep), _shape_key(grid_h), _shape_key(grid_w), heads, n_tokens,
               _shape_key(seqlens), cls, conv)
        return self._remember(key, make)

    def _l_shapes(self, dim, dtype, rows, keep, n_vision, n_text, heads, flags) -> _Shapes:
        conv = bool(flags & FICOCO_CONVERGENT)

        def make():
            keep_a, n_keep = _int_array(keep)
            batch = rows // (n_vision + n_text)
            keeps = [int(keep_a[0 if n_keep == 1 else b]) for b in range(batch)]
            out_rows = [k + n_text + (1 if conv and n_vision - k > 0 else 0) for k in keeps]
            a = ficoco_l_args()
            a.keep = keep_a.ctypes.data
            a.dtype, a.batch, a.n_vision, a.n_text = dtype, batch, n_vision, n_text
            a.dim, a.heads, a.n_keep = dim, heads, n_keep
            return _Shapes(a, (keep_a,), out_rows, sum(out_rows), sum(keeps), batch * n_vision)

        return self._remember(("l", dim, dtype, rows, _shape_key(keep), n_vision, n_text, heads, conv), make)

    def close(self) -> None:
        if getattr(self, "h", None):
            self.lib.ficoco_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- device-pointer entry points -----------------------------------------------------
    def ficoco_v_reduce(self, tokens, attn, keep, grid_h, grid_w, heads: int, *, n_tokens: int = 0,
                        seqlens=None, pos=None, params: Optional[ficoco_params] = None,
                        out_tokens=None, kept_idx=None, pos_out=None, scores_out=None,
                        want_scores: bool = False, stream: Optional[int] = None,
                        relation=None, by_column: bool = False, out_cu_seqlens=None,
                        plan_only: bool = False) -> VResult:
        """tokens: cuda tensor [rows, D]; attn: cuda fp32 tensor (packed per image [H, Np]);
        keep / grid_h / grid_w: int or per-image list; seqlens: per-image rows incl. CLS or
        None with n_tokens given.  Output tensors are allocated with torch when not passed.
        relation: optional cuda fp32 tensor, the images' [Np, Np] relation blocks one after the
        other; when given the call goes to ficoco_v_reduce_relation."""
        import torch
        p = params or ficoco_default_params()
        dim, dev = tokens.shape[-1], tokens.device
        sh = self._v_shapes(dim, _dtype_code(tokens), tokens.shape[0], keep, grid_h, grid_w, heads, n_tokens, seqlens,
                            p.flags)
        a = ficoco_v_args.from_buffer_copy(sh.args)
        if stream is None:
            stream = _current_stream(dev)
        if plan_only:               # ficoco_v_plan: shapes only
            _check(self.h, self.lib.ficoco_v_plan(self.h, C.byref(a), C.byref(p), stream))
            return VResult(None, None, None, None, list(sh.out_rows))
        if out_tokens is None:
            out_tokens = torch.empty((sh.n_out, dim), dtype=tokens.dtype, device=dev)
        if kept_idx is None:
            kept_idx = torch.empty((sh.n_out,), dtype=torch.int32, device=dev)
        if pos_out is None:
            pos_out = torch.empty((max(sh.n_keep, 1),), dtype=torch.int32, device=dev)
        if scores_out is None and want_scores:
            scores_out = torch.empty((attn.numel() // heads,), dtype=torch.float32, device=dev)
        a.tokens, a.attn, a.pos = _ptr(tokens), _ptr(attn), _ptr(pos)
        a.out_tokens, a.kept_idx = _ptr(out_tokens), _ptr(kept_idx)
        a.pos_out, a.scores_out = _ptr(pos_out), _ptr(scores_out)
        a.out_cu_seqlens = _ptr(out_cu_seqlens)
        if relation is not None:
            rc = self.lib.ficoco_v_reduce_relation(self.h, C.byref(a), _ptr(relation), int(by_column), C.byref(p), stream)
        else:
            rc = self.lib.ficoco_v_reduce(self.h, C.byref(a), C.byref(p), stream)
        if rc:
            _check(self.h, rc)
        return VResult(out_tokens, kept_idx, pos_out, scores_out, list(sh.out_rows))

    def ficoco_v_reduce_schedule(self, tokens, attns, keeps, grid_h: int, grid_w: int, heads: int, *, n_tokens: int,
                                 pos=None, params: Optional[ficoco_params] = None, out_tokens=None, kept_idx=None,
                                 pos_out=None, stream: Optional[int] = None) -> VResult:
        """A progressive schedule in one call.  attns: list of cuda fp32 tensors, one per step
        ([B, H, Np_s] over the patch tokens alive at that step); keeps: patch tokens preserved by
        each step.  Returns the last step's tokens, kept_idx (into the original rows) and pos."""
        import torch
        p = params or ficoco_default_params()
        cls = 1 if (p.flags & FICOCO_HAS_CLS) else 0
        batch = tokens.shape[0] // n_tokens
        keep_a = np.ascontiguousarray(np.asarray(keeps, dtype=np.int32))
        n_steps = int(keep_a.shape[0])
        rows = cls + int(keep_a[-1])
        dim, dev = tokens.shape[-1], tokens.device
        if out_tokens is None:
            out_tokens = torch.empty((batch * rows, dim), dtype=tokens.dtype, device=dev)
        if kept_idx is None:
            kept_idx = torch.empty((batch * rows,), dtype=torch.int32, device=dev)
        if pos_out is None:
            pos_out = torch.empty((max(batch * int(keep_a[-1]), 1),), dtype=torch.int32, device=dev)
        gh_a, gw_a = _int_array(grid_h)[0], _int_array(grid_w)[0]
        a = ficoco_v_args()
        a.tokens, a.pos = _ptr(tokens), _ptr(pos)
        a.grid_h, a.grid_w = gh_a.ctypes.data, gw_a.ctypes.data
        a.out_tokens, a.kept_idx, a.pos_out = _ptr(out_tokens), _ptr(kept_idx), _ptr(pos_out)
        a.dtype, a.batch, a.n_tokens, a.dim, a.heads = _dtype_code(tokens), batch, n_tokens, dim, heads
        a.n_grid, a.n_keep = 1, 1
        ptrs = (C.c_void_p * n_steps)(*[t.data_ptr() for t in attns])
        if stream is None:
            stream = _current_stream(dev)
        _check(self.h, self.lib.ficoco_v_reduce_schedule(self.h, C.byref(a), n_steps, keep_a.ctypes.data, ptrs,
                                                         C.byref(p), stream))
        return VResult(out_tokens, kept_idx, pos_out, None, [rows] * batch)

    def ficoco_l_reduce(self, tokens, attn_t2v, keep, n_vision: int, n_text: int, heads: int, *,
                        params: Optional[ficoco_params] = None, out_tokens=None, kept_idx=None,
                        scores_out=None, want_scores: bool = False, stream: Optional[int] = None) -> VResult:
        """tokens: cuda tensor [B*(N+M), D]; attn_t2v: cuda fp32 [B, H, M, N]."""
        import torch
        p = params or ficoco_default_params()
        dim, dev = tokens.shape[-1], tokens.device
        sh = self._l_shapes(dim, _dtype_code(tokens), tokens.shape[0], keep, n_vision, n_text, heads, p.flags)
        a = ficoco_l_args.from_buffer_copy(sh.args)
        if out_tokens is None:
            out_tokens = torch.empty((sh.n_out, dim), dtype=tokens.dtype, device=dev)
        if kept_idx is None:
            kept_idx = torch.empty((sh.n_out,), dtype=torch.int32, device=dev)
        if scores_out is None and want_scores:
            scores_out = torch.empty((sh.n_patch,), dtype=torch.float32, device=dev)
        a.tokens, a.attn_t2v = _ptr(tokens), _ptr(attn_t2v)
        a.out_tokens, a.kept_idx, a.scores_out = _ptr(out_tokens), _ptr(kept_idx), _ptr(scores_out)
        if stream is None:
            stream = _current_stream(dev)
        rc = self.lib.ficoco_l_reduce(self.h, C.byref(a), C.byref(p), stream)
        if rc:
            _check(self.h, rc)
        return VResult(out_tokens, kept_idx, None, scores_out, list(sh.out_rows))

    # -- host-buffer entry points (tensors live in host memory, ideally pinned) ------------
    def ficoco_v_reduce_host(self, tokens, attn, keep, grid_h, grid_w, heads: int, *, n_tokens: int = 0,
                             seqlens=None, pos=None, params: Optional[ficoco_params] = None,
                             out_tokens=None, kept_idx=None, pos_out=None, scores_out=None) -> VResult:
        import torch
        p = params or ficoco_default_params()
        cls = 1 if (p.flags & FICOCO_HAS_CLS) else 0
        keep_a, n_keep = _int_array(keep)
        gh_a, n_gh = _int_array(grid_h)
        gw_a, _ = _int_array(grid_w)
        if seqlens is not None:
            sl, batch = _int_array(seqlens)
        else:
            sl, batch = None, tokens.shape[0] // n_tokens
        keeps = [int(keep_a[0 if n_keep == 1 else b]) for b in range(batch)]
        ntoks = [int(sl[b]) if sl is not None else n_tokens for b in range(batch)]
        conv = bool(p.flags & FICOCO_CONVERGENT)
        out_rows = [cls + k + (1 if conv and n - cls - k > 0 else 0) for k, n in zip(keeps, ntoks)]
        dim = tokens.shape[-1]
        if out_tokens is None:
            out_tokens = torch.empty((sum(out_rows), dim), dtype=tokens.dtype).pin_memory()
        if kept_idx is None:
            kept_idx = torch.empty((sum(out_rows),), dtype=torch.int32).pin_memory()
        a = ficoco_v_args()
        a.tokens, a.attn, a.pos = _ptr(tokens), _ptr(attn), _ptr(pos)
        a.seqlens = sl.ctypes.data if sl is not None else None
        a.grid_h, a.grid_w, a.keep = gh_a.ctypes.data, gw_a.ctypes.data, keep_a.ctypes.data
        a.out_tokens, a.kept_idx = _ptr(out_tokens), _ptr(kept_idx)
        a.pos_out, a.scores_out = _ptr(pos_out), _ptr(scores_out)
        a.dtype, a.batch, a.n_tokens, a.dim, a.heads = _dtype_code(tokens), batch, n_tokens, dim, heads
        a.n_grid, a.n_keep = n_gh, n_keep
        _check(self.h, self.lib.ficoco_v_reduce_host(self.h, C.byref(a), C.byref(p)))
        return VResult(out_tokens, kept_idx, pos_out, scores_out, out_rows)

    def ficoco_l_reduce_host(self, tokens, attn_t2v, keep, n_vision: int, n_text: int, heads: int, *,
                             params: Optional[ficoco_params] = None, out_tokens=None, kept_idx=None,
                             scores_out=None) -> VResult:
        import torch
        p = params or ficoco_default_params()
        keep_a, n_keep = _int_array(keep)
        batch = tokens.shape[0] // (n_vision + n_text)
        keeps = [int(keep_a[0 if n_keep == 1 else b]) for b in range(batch)]
        conv = bool(p.flags & FICOCO_CONVERGENT)
        out_rows = [k + n_text + (1 if conv and n_vision - k > 0 else 0) for k in keeps]
        dim = tokens.shape[-1]
        if out_tokens is None:
            out_tokens = torch.empty((sum(out_rows), dim), dtype=tokens.dtype).pin_memory()
        if kept_idx is None:
            kept_idx = torch.empty((sum(out_rows),), dtype=torch.int32).pin_memory()
        a = ficoco_l_args()
        a.tokens, a.attn_t2v, a.keep = _ptr(tokens), _ptr(attn_t2v), keep_a.ctypes.data
        a.out_tokens, a.kept_idx, a.scores_out = _ptr(out_tokens), _ptr(kept_idx), _ptr(scores_out)
        a.dtype, a.batch, a.n_vision, a.n_text = _dtype_code(tokens), batch, n_vision, n_text
        a.dim, a.heads, a.n_keep = dim, heads, n_keep
        _check(self.h, self.lib.ficoco_l_reduce_host(self.h, C.byref(a), C.byref(p)))
        return VResult(out_tokens, kept_idx, None, scores_out, out_rows)

    # -- 8-bit paged cache --------------------------------------------------------------------
    def ficoco_cache_append(self, cache: PagedCache, k, v, cu_rows, *, stream: Optional[int] = None) -> None:
        """Writes k, v (cuda [rows, kv_heads, head_dim], bf16 or fp32, rows may be strided) as the last tokens of the
        sequences; cu_rows: cuda int32 [batch + 1].  ``cache.lengths`` already counts them."""
        cs = cache.struct
        self._same_device(cache, k)
        if k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.shape[1:] != (cs.kv_heads, cs.head_dim):
            raise ValueError(f"k and v must both be [rows, {cs.kv_heads}, {cs.head_dim}] of one type")
        a = ficoco_append_args(k.data_ptr(), v.data_ptr(), _int32("cu_rows", cu_rows, cs.batch + 1, cache.device),
                               _rows3("k", k, cs.head_dim), _rows3("v", v, cs.head_dim), _dtype_code(k), k.shape[0])
        rc = self.lib.ficoco_cache_append(self.h, cs, a, _current_stream(cache.device) if stream is None else stream)
        if rc:
            _check(self.h, rc)

    def _same_device(self, cache: PagedCache, t) -> None:
        if cache.device.index != self.device or t.device != cache.device:
            raise ValueError(f"the context is on cuda:{self.device}, the cache on {cache.device}, the rows on {t.device}")

    def _attention_args(self, cache, q, cu_rows, scale, causal, window, sinks) -> ficoco_attention_args:
        cs = cache.struct
        self._same_device(cache, q)
        stride = _rows3("q", q, cs.head_dim)
        if (window | sinks) >> 31:
            _c_ints(window=window, sinks=sinks)
        return ficoco_attention_args(q.data_ptr(), _int32("cu_rows", cu_rows, cs.batch + 1, cache.device), None, None, stride,
                                     cache.scale if scale is None else scale, _dtype_code(q), q.shape[0], q.shape[1],
                                     window, sinks, FICOCO_CAUSAL if causal else 0)

    def ficoco_cache_attention(self, cache: PagedCache, q, cu_rows, *, scale: Optional[float] = None, causal: bool = True,
                               window: int = 0, sinks: int = 0, out=None, lse=None, want_lse: bool = False,
                               stream: Optional[int] = None):
        """Attention of q (cuda [rows, heads, head_dim], the last tokens of the sequences) over the cache.  Returns out, or
        (out, lse) with want_lse.  scale: 1 / sqrt(head_dim) by default; window / sinks: a row sees the last ``window`` tokens up to
        its own and the first ``sinks``."""
        torch = _load_torch()
        a = self._attention_args(cache, q, cu_rows, scale, causal, window, sinks)
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous() or out.device != cache.device:
            raise ValueError("out must be contiguous, with q's shape, type and device")
        if lse is None:
            if want_lse:
                lse = torch.empty_strided((a.rows, a.heads), (a.heads, 1), dtype=torch.float32, device=cache.device)
        elif lse.shape != q.shape[:2] or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != cache.device:
            raise ValueError("lse must be contiguous fp32 [rows, heads] on q's device")
        a.out = out.data_ptr()
        if lse is not None:
            a.lse = lse.data_ptr()
        rc = self.lib.ficoco_cache_attention(self.h, cache.struct, a, _current_stream(cache.device) if stream is None else stream)
        if rc:
            _check(self.h, rc)
        return (out, lse) if want_lse else out

    def ficoco_cache_weights(self, cache: PagedCache, q, lse, cu_rows, n_text: int, first: int, count: int, *,
                             scale: Optional[float] = None, causal: bool = True, window: int = 0, sinks: int = 0, out=None,
                             stream: Optional[int] = None):
        """fp32 [batch, heads, n_text, count]: what the last n_text rows of every sequence give the ``count`` tokens from
        ``first`` on.  q, cu_rows and the mask are those of the attention call that returned lse; the result is ``attn_t2v`` of
        ``ficoco_l_reduce``."""
        torch = _load_torch()
        a = self._attention_args(cache, q, cu_rows, scale, causal, window, sinks)
        if lse.shape != q.shape[:2] or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != cache.device:
            raise ValueError("lse must be contiguous fp32 [rows, heads] on q's device")
        if (n_text | first | count) >> 31:
            _c_ints(n_text=n_text, first=first, count=count)
        shape = (cache.struct.batch, q.shape[1], n_text, count)
        if out is None:
            out = _new(q, shape, torch.float32)
        elif tuple(out.shape) != shape or out.dtype != torch.float32 or not out.is_contiguous() or out.device != cache.device:
            raise ValueError(f"out must be contiguous fp32 {shape} on q's device")
        a.lse = lse.data_ptr()
        rc = self.lib.ficoco_cache_weights(self.h, cache.struct, a, n_text, first, count, out.data_ptr(),
                                           _current_stream(cache.device) if stream is None else stream)
        if rc:
            _check(self.h, rc)
        return out

    def ficoco_cache_copy(self, cache: PagedCache, src, dst, *, stream: Optional[int] = None) -> None:
        """Copies page src[i] to page dst[i] (cuda int32 tensors of one length; pairs with a negative page are skipped)."""
        self._same_device(cache, src)
        rc = self.lib.ficoco_cache_copy(self.h, cache.struct, _int32("src", src),
                                        _int32("dst", dst, src.numel(), cache.device), src.numel(),
                                        _current_stream(cache.device) if stream is None else stream)
        if rc:
            _check(self.h, rc)

    def ficoco_cache_compact(self, cache: PagedCache, to_table, kept, cu_kept, *, first: int = 0, lengths=None,
                             stream: Optional[int] = None):
        """Gathers the first ``first`` tokens of every sequence and its tokens first + kept[i] into the pages of ``to_table``
        (cuda int32 [batch, pages], other pages than the cache's).  Returns the new lengths (cuda int32 [batch])."""
        torch = _load_torch()
        cs = cache.struct
        self._same_device(cache, to_table)
        if first >> 31:
            _c_ints(first=first)
        if to_table.dtype != torch.int32 or to_table.dim() != 2 or to_table.shape[0] != cs.batch or not to_table.is_cuda or \
                to_table.stride(1) != 1:
            raise ValueError(f"to_table must be a cuda int32 tensor [{cs.batch}, pages]")
        if lengths is None:
            lengths = _new(to_table, (cs.batch,), torch.int32)
        a = ficoco_compact_args(to_table.data_ptr(), _int32("kept", kept, None, cache.device),
                                _int32("cu_kept", cu_kept, cs.batch + 1, cache.device),
                                _int32("lengths", lengths, cs.batch, cache.device), to_table.stride(0), to_table.shape[1], kept.numel(), first, 0)
        rc = self.lib.ficoco_cache_compact(self.h, cs, a, _current_stream(cache.device) if stream is None else stream)
        if rc:
            _check(self.h, rc)
        return lengths

    # -- status / inspection ----------------------------------------------------------------
    def ficoco_status(self, stream: Optional[int] = None) -> int:
        import torch
        if stream is None:
            stream = torch.cuda.current_stream().cuda_stream
        v = C.c_int(0)
        _check(self.h, self.lib.ficoco_status(self.h, C.c_void_p(stream), C.byref(v)))
        return v.value

    def ficoco_inspect(self, what: str) -> np.ndarray:
        code, dt, width = INSPECT[what]
        n = C.c_size_t(0)
        _check(self.h, self.lib.ficoco_inspect(self.h, code, None, 0, C.byref(n)))
        buf = np.empty(n.value // 4, dtype=dt)
        if n.value:
            _check(self.h, self.lib.ficoco_inspect(self.h, code, buf.ctypes.data, n.value, None))
        return buf.reshape(-1, width) if width > 1 else buf

    def ficoco_debug_waits(self, wait_ns: int = 0, extra_arrivals: int = 0) -> None:
        _check(self.h, self.lib.ficoco_debug_waits(self.h, wait_ns, extra_arrivals))

    def ficoco_debug_barrier_wait(self) -> int:
        v = C.c_longlong(0)
        _check(self.h, self.lib.ficoco_debug_barrier_wait(self.h, C.byref(v)))
        return v.value

    def ficoco_last_launch_count(self) -> int:
        return int(self.lib.ficoco_last_launch_count(self.h))

    def ficoco_profile(self, enable: bool) -> None:
        _check(self.h, self.lib.ficoco_profile(self.h, 1 if enable else 0))

    def ficoco_profile_read(self):
        """[(kernel name, total ms, launches), ...] since profiling was enabled."""
        out = []
        i = 0
        while True:
            name = C.create_string_buffer(64)
            ms, n = C.c_double(0), C.c_longlong(0)
            if self.lib.ficoco_profile_read(self.h, i, name, 64, C.byref(ms), C.byref(n)) != 0:
                break
            out.append((name.value.decode(), ms.value, n.value))
            i += 1
        return out


def ficoco_vision_redundancy_noalloc(tokens, n_tokens: int, has_cls: bool = True, v_out=None,
                                     stream: Optional[int] = None):
    """First term of Eq. 1 for a uniform batch, for callers that may not allocate device memory
    (for example a serving engine's step callback whose engine owns all of it): no context, the
    scratch is a fixed array inside the library.  ``tokens``: cuda tensor [batch * n_tokens, D];
    ``v_out``: cuda fp32 [batch * Np], which the caller should pass in (it is only created here,
    with torch, as a convenience for tests).  Limits and sharing rules: see ficoco.h."""
    import torch
    lib = load_library()
    batch = tokens.shape[0] // n_tokens
    np_ = n_tokens - (1 if has_cls else 0)
    if v_out is None:
        v_out = torch.empty((batch * np_,), dtype=torch.float32, device=tokens.device)
    if stream is None:
        stream = torch.cuda.current_stream(tokens.device).cuda_stream
    rc = lib.ficoco_vision_redundancy_noalloc(tokens.data_ptr(), _dtype_code(tokens), batch, n_tokens,
                                              tokens.shape[-1], FICOCO_HAS_CLS if has_cls else 0,
                                              v_out.data_ptr(), C.c_void_p(stream))
    _check(None, rc)
    return v_out


def ficoco_equivalent_token(keys, heads: int, head_dim: int, *, n_tokens: int = 0, seqlens=None,
                            has_cls: bool = False, a_eq=None, stream: Optional[int] = None):
    """a^Eq of the no-CLS variant.  ``keys``: cuda tensor [rows, heads * head_dim] (token-major
    key states, images packed); ``seqlens``: rows per image, or None with ``n_tokens`` given.
    Returns the cuda fp32 tensor of one value per patch token (allocated with torch when
    ``a_eq`` is not passed); use it as ``attn`` with ``heads = 1`` in ficoco_v_reduce."""
    import torch
    lib = load_library()
    cls = 1 if has_cls else 0
    if seqlens is not None:
        sl, batch = _int_array(seqlens)
        patches = int(sl.sum()) - cls * batch
        sl_ptr = sl.ctypes.data
    else:
        sl, batch = None, keys.shape[0] // n_tokens
        patches = batch * (n_tokens - cls)
        sl_ptr = None
    if a_eq is None:
        a_eq = torch.empty((patches,), dtype=torch.float32, device=keys.device)
    if stream is None:
        stream = _current_stream(keys.device)
    rc = lib.ficoco_equivalent_token(keys.data_ptr(), _dtype_code(keys), batch, n_tokens, sl_ptr, heads, head_dim, cls,
                                     a_eq.data_ptr(), stream)
    _check(None, rc)
    return a_eq


# ----------------------------------------------------------------------------------------
# numpy <-> torch helpers for the synthetic batches
# ----------------------------------------------------------------------------------------

def to_torch(arr: np.ndarray, device=None, pin: bool = False):
    """numpy fp32 / int32 / uint16(bf16 bits) -> torch tensor (bf16 for uint16)."""
    import torch
    if arr.dtype == np.uint16:
        t = torch.from_numpy(arr.view(np.int16).copy()).view(torch.bfloat16)
    else:
        t = torch.from_numpy(np.ascontiguousarray(arr).copy())
    if pin:
        t = t.pin_memory()
    if device is not None:
        t = t.to(device)
    return t


def to_numpy(t) -> np.ndarray:
    """torch tensor -> numpy (bf16 as uint16 bit patterns)."""
    import torch
    t = t.detach().cpu()
    if t.dtype == torch.bfloat16:
        return t.view(torch.int16).numpy().view(np.uint16).copy()
    return t.numpy().copy()
