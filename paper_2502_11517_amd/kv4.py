"""Thin ctypes binding of libpasta_kv4.so (include/pasta_kv4.h): the 4-bit paged KV cache, rows into it and out of it, and its attention.

Argument marshalling only, as in kv8.py, whose slots() gives the rows their places: a PastaKv8 handle over the same page table, without codes.
"""
from __future__ import annotations

import ctypes as C
import os
import subprocess

from .binding import BF16, E_CAPACITY, E_DEVICE, E_INVAL, E_NOMEM, E_STATE, F32, HIPCC_FLAGS, OK, PastaError  # noqa: F401
from .kv8 import _DTYPES, _I32, _ROWS, _U8, BLOCK, F16, AttendArgs, PlanArgs, _Attention, _p  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_HERE, "libpasta_kv4.so")
_lib = None

GROUP = 32  # dims of K under one scale
_CODES = ("torch.uint8",)


def library_path() -> str:
    return _LIB


def build_library(verbose: bool = False) -> str:
    """Compiles csrc/pasta_kv4.hip for gfx950 with hipcc (cross-compiles without a GPU)."""
    cmd = ["hipcc", *HIPCC_FLAGS, os.path.join(_HERE, "csrc", "pasta_kv4.hip"), "-o", _LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + r.stderr)
    if verbose:
        print(" ".join(cmd))
    return _LIB


class Config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("n_layers", C.c_int32), ("max_requests", C.c_int32), ("max_rows", C.c_int32), ("page_tokens", C.c_int32), ("n_phys_pages", C.c_int32),
        ("pages_per_request", C.c_int32), ("softmax_scale", C.c_float),
        ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("page_table", C.c_void_p),
        ("slot_tag", C.c_void_p), ("slot_position", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class AppendArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("layer", C.c_int32), ("n_rows", C.c_int32), ("dtype", C.c_int32),
        ("slot", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
    ]


class ReadArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("layer", C.c_int32), ("n_rows", C.c_int32), ("dtype", C.c_int32),
        ("slot", C.c_void_p), ("k_out", C.c_void_p), ("v_out", C.c_void_p), ("k_stride", C.c_int64), ("v_stride", C.c_int64),
    ]


def load_library():
    """Loads the built library; raises if it is missing (there is no other path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB):
            raise RuntimeError(f"{_LIB} is not built: run __graft_entry__.build() (hipcc, gfx950)")
        import torch  # noqa: F401  (binds the library to torch's HIP runtime, as in binding.load_library)
        L = C.CDLL(_LIB)
        L.pasta_kv4_create.restype, L.pasta_kv4_create.argtypes = C.c_int32, [C.POINTER(Config), C.POINTER(C.c_void_p)]
        L.pasta_kv4_destroy.restype, L.pasta_kv4_destroy.argtypes = C.c_int32, [C.c_void_p]
        for name, args in (("append", AppendArgs), ("read", ReadArgs), ("plan", PlanArgs), ("attend", AttendArgs)):
            f = getattr(L, "pasta_kv4_" + name)
            f.restype, f.argtypes = C.c_int32, [C.c_void_p, C.POINTER(args)]
        _lib = L
    return _lib


def make_config(dtype, n_q_heads, n_kv_heads, head_dim, softmax_scale, *, n_layers=1, max_requests=1, max_rows=1, page_tokens=16, n_phys_pages=1,
                pages_per_request=1) -> Config:
    c = Config()
    c.struct_size = C.sizeof(Config)
    c.dtype = _DTYPES.get(dtype, dtype)
    c.n_q_heads, c.n_kv_heads, c.head_dim, c.softmax_scale = n_q_heads, n_kv_heads, head_dim, softmax_scale
    c.n_layers, c.max_requests, c.max_rows = n_layers, max_requests, max_rows
    c.page_tokens, c.n_phys_pages, c.pages_per_request = page_tokens, n_phys_pages, pages_per_request
    return c


def query_workspace_bytes(cfg: Config) -> int:
    rc = load_library().pasta_kv4_create(C.byref(cfg), None)
    if rc != OK:
        raise PastaError(rc, "pasta_kv4_create(query)")
    return int(cfg.workspace_bytes)


def cache_shapes(cfg: Config):
    """(shape of k_codes, of v_codes, of k_scale, of v_scale), whole cache, all uint8."""
    block = (cfg.n_layers, cfg.n_phys_pages, cfg.n_kv_heads, cfg.page_tokens // BLOCK)
    return ((*block, cfg.head_dim // GROUP, BLOCK, GROUP // 2), (*block, cfg.head_dim, BLOCK // 2), (*block, BLOCK, cfg.head_dim // GROUP),
            (*block, BLOCK))


class PastaKv4(_Attention):
    """One handle.  Buffers are device addresses (or torch tensors, which are then kept alive and checked for type, contiguity,
    size and device) owned by the caller; those that no call needs may be left out.  `stream` is a hipStream_t as an int."""

    _prefix = "pasta_kv4_"

    def __init__(self, cfg: Config, workspace=None, *, page_table=None, k_codes=None, v_codes=None, k_scale=None, v_scale=None, slot_tag=None,
                 slot_position=None, stream=0, workspace_bytes=None):
        self._h = None
        self._lib = load_library()
        self.cfg = cfg
        self._keep = [workspace, page_table, k_codes, v_codes, k_scale, v_scale, slot_tag, slot_position]
        shapes, slots = cache_shapes(cfg), (cfg.n_phys_pages * cfg.page_tokens,)
        cfg.k_codes, cfg.v_codes = _p(k_codes, _CODES, shapes[0], "k_codes"), _p(v_codes, _CODES, shapes[1], "v_codes")
        cfg.k_scale, cfg.v_scale = _p(k_scale, _U8, shapes[2], "k_scale"), _p(v_scale, _U8, shapes[3], "v_scale")
        cfg.page_table = _p(page_table, _I32, (cfg.max_requests, cfg.pages_per_request), "page_table")
        cfg.slot_tag, cfg.slot_position = _p(slot_tag, _U8, slots, "slot_tag"), _p(slot_position, _I32, slots, "slot_position")
        cfg.workspace = _p(workspace, _U8, (1,), "workspace")
        cfg.workspace_bytes = workspace_bytes if workspace_bytes is not None else (0 if workspace is None or isinstance(workspace, int) else workspace.numel())
        cfg.hip_stream = stream
        h = C.c_void_p()
        rc = self._lib.pasta_kv4_create(C.byref(cfg), C.byref(h))
        if rc != OK:
            raise PastaError(rc, "pasta_kv4_create")
        self._h = h

    def _rows(self, x, n, of, what):
        """(address, stride) of rows [n, Hkv, D], which may lie apart from one another."""
        H, D = self.cfg.n_kv_heads, self.cfg.head_dim
        if x is None or isinstance(x, int):
            return x, 0
        return _strided(x, n, H, D, of, what)

    def prepare_append(self, layer, slot, k_new, v_new, *, n_rows=None, dtype=None):
        n = n_rows if n_rows is not None else int(slot.shape[0])
        dtype, of = _row_type(dtype, k_new)
        (k, ks), (v, vs) = self._rows(k_new, n, of, "k_new"), self._rows(v_new, n, of, "v_new")
        a = AppendArgs(C.sizeof(AppendArgs), 0, layer, n, dtype, _p(slot, _I32, (n,), "slot"), k, v, ks, vs)
        return self._prepared("append", a, (slot, k_new, v_new))

    def prepare_read(self, layer, slot, k_out=None, v_out=None, *, n_rows=None, dtype=None):
        n = n_rows if n_rows is not None else int(slot.shape[0])
        dtype, of = _row_type(dtype, k_out if k_out is not None else v_out)
        (k, ks), (v, vs) = self._rows(k_out, n, of, "k_out"), self._rows(v_out, n, of, "v_out")
        a = ReadArgs(C.sizeof(ReadArgs), 0, layer, n, dtype, _p(slot, _I32, (n,), "slot"), k, v, ks, vs)
        return self._prepared("read", a, (slot, k_out, v_out))

    def append(self, *args, **kw):
        self._now(self.prepare_append(*args, **kw))

    def read(self, *args, **kw):
        self._now(self.prepare_read(*args, **kw))


def _row_type(dtype, x):
    """(code of a type of rows, names of torch's types that it stands for)"""
    if dtype is None:
        dtype = _ROWS.get(str(getattr(x, "dtype", None)), -1)
    dtype = _DTYPES.get(dtype, dtype)
    return dtype, tuple(k for k, v in _ROWS.items() if v == dtype) or None


def _strided(x, n, heads, dim, of, what):
    """(address, values between rows) of a tensor of n rows [heads, dim], each in one piece."""
    if of is not None and str(x.dtype) not in of:
        raise ValueError(f"{what}: {x.dtype}, one of {of} is wanted")
    if x.dim() != 3 or x.shape[0] < n or tuple(x.shape[1:]) != (heads, dim):
        raise ValueError(f"{what}: {tuple(x.shape)}, {(n, heads, dim)} is wanted")
    if (dim > 1 and x.stride(2) != 1) or (heads > 1 and x.stride(1) != dim):
        raise ValueError(f"{what}: a row is not contiguous")
    if n > 1 and x.stride(0) < heads * dim:
        raise ValueError(f"{what}: rows overlap")
    if not x.is_cuda:
        raise ValueError(f"{what}: on {x.device}, device memory is wanted")
    return x.data_ptr(), x.stride(0) if n > 1 else 0
