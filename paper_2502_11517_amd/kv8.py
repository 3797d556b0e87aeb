"""Thin ctypes binding of libpasta_kv8.so (include/pasta_kv8.h): the 8-bit paged KV cache, its places and its attention.

Argument marshalling only, as in binding.py: torch is used for device memory and the stream, every step runs in the
library's HIP kernels, and there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import subprocess

from .binding import BF16, E_CAPACITY, E_DEVICE, E_INVAL, E_NOMEM, E_STATE, F32, HIPCC_FLAGS, OK, PastaError  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_HERE, "libpasta_kv8.so")
_lib = None

E4M3, INT8 = 0, 1
F16 = 2
BLOCK = 16  # tokens under one scale
_CODES = {"e4m3": E4M3, "int8": INT8}
_DTYPES = {"f32": F32, "bf16": BF16, "f16": F16}


def library_path() -> str:
    return _LIB


def build_library(verbose: bool = False) -> str:
    """Compiles csrc/pasta_kv8.hip for gfx950 with hipcc (cross-compiles without a GPU)."""
    cmd = ["hipcc", *HIPCC_FLAGS, os.path.join(_HERE, "csrc", "pasta_kv8.hip"), "-o", _LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + r.stderr)
    if verbose:
        print(" ".join(cmd))
    return _LIB


class Config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("codes", C.c_int32), ("dtype", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("n_layers", C.c_int32), ("max_requests", C.c_int32), ("max_rows", C.c_int32), ("page_tokens", C.c_int32),
        ("n_phys_pages", C.c_int32), ("pages_per_request", C.c_int32), ("softmax_scale", C.c_float),
        ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("page_table", C.c_void_p),
        ("free_pages", C.c_void_p), ("slot_tag", C.c_void_p), ("slot_position", C.c_void_p), ("workspace", C.c_void_p),
        ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class SlotsArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_requests", C.c_int32), ("n_rows", C.c_int32), ("length", C.c_void_p),
        ("keep", C.c_void_p), ("row_offsets", C.c_void_p), ("row_tag", C.c_void_p), ("row_position", C.c_void_p), ("free_count", C.c_void_p),
        ("slot", C.c_void_p), ("length_out", C.c_void_p), ("free_out", C.c_void_p),
    ]


class AppendArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("layer", C.c_int32), ("n_rows", C.c_int32), ("dtype", C.c_int32),
        ("slot", C.c_void_p), ("k_new", C.c_void_p), ("v_new", C.c_void_p),
    ]


class PlanArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_requests", C.c_int32), ("n_rows", C.c_int32), ("max_request_rows", C.c_int32),
        ("length", C.c_void_p), ("row_offsets", C.c_void_p), ("prefix_len", C.c_void_p), ("slot", C.c_void_p),
    ]


class AttendArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("layer", C.c_int32), ("n_rows", C.c_int32), ("logit_cap", C.c_float),
        ("q", C.c_void_p), ("out", C.c_void_p), ("lse", C.c_void_p), ("slopes", C.c_void_p), ("row_see", C.c_void_p), ("row_position", C.c_void_p),
    ]


def load_library():
    """Loads the built library; raises if it is missing (there is no other path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB):
            raise RuntimeError(f"{_LIB} is not built: run __graft_entry__.build() (hipcc, gfx950)")
        import torch  # noqa: F401  (binds the library to torch's HIP runtime, as in binding.load_library)
        L = C.CDLL(_LIB)
        L.pasta_kv8_create.restype, L.pasta_kv8_create.argtypes = C.c_int32, [C.POINTER(Config), C.POINTER(C.c_void_p)]
        L.pasta_kv8_destroy.restype, L.pasta_kv8_destroy.argtypes = C.c_int32, [C.c_void_p]
        for name, args in (("slots", SlotsArgs), ("append", AppendArgs), ("plan", PlanArgs), ("attend", AttendArgs)):
            f = getattr(L, "pasta_kv8_" + name)
            f.restype, f.argtypes = C.c_int32, [C.c_void_p, C.POINTER(args)]
        _lib = L
    return _lib


def make_config(codes, dtype, n_q_heads, n_kv_heads, head_dim, softmax_scale, *, n_layers=1, max_requests=1, max_rows=1, page_tokens=16,
                n_phys_pages=1, pages_per_request=1) -> Config:
    c = Config()
    c.struct_size = C.sizeof(Config)
    c.codes, c.dtype = _CODES.get(codes, codes), _DTYPES.get(dtype, dtype)
    c.n_q_heads, c.n_kv_heads, c.head_dim, c.softmax_scale = n_q_heads, n_kv_heads, head_dim, softmax_scale
    c.n_layers, c.max_requests, c.max_rows = n_layers, max_requests, max_rows
    c.page_tokens, c.n_phys_pages, c.pages_per_request = page_tokens, n_phys_pages, pages_per_request
    return c


def query_workspace_bytes(cfg: Config) -> int:
    rc = load_library().pasta_kv8_create(C.byref(cfg), None)
    if rc != OK:
        raise PastaError(rc, "pasta_kv8_create(query)")
    return int(cfg.workspace_bytes)


def cache_shapes(cfg: Config):
    """(shape of k_codes, of v_codes, of a scale array), whole cache; codes are one byte each."""
    head = (cfg.n_layers, cfg.n_phys_pages, cfg.n_kv_heads, cfg.page_tokens // BLOCK)
    return (*head, cfg.head_dim // 16, BLOCK, 16), (*head, cfg.head_dim, BLOCK), head


def _p(t, dtypes=None, shape=None, what=""):
    """Address of a tensor (or an address itself), after what can be checked of it: type, contiguity, number of values, and that it is the GPU's."""
    if t is None or isinstance(t, int):
        return t
    if dtypes is not None and str(t.dtype) not in dtypes:
        raise ValueError(f"{what}: {t.dtype}, one of {dtypes} is wanted")
    if not t.is_contiguous():
        raise ValueError(f"{what}: not contiguous")
    if shape is not None:
        want = 1
        for n in shape:
            want *= n
        if t.numel() < want:
            raise ValueError(f"{what}: {tuple(t.shape)}, {tuple(shape)} is wanted")
    if not t.is_cuda:
        raise ValueError(f"{what}: on {t.device}, device memory is wanted")
    return t.data_ptr()


_I32, _F32, _U8 = ("torch.int32",), ("torch.float32",), ("torch.uint8",)
_ROWS = {"torch.float32": F32, "torch.bfloat16": BF16, "torch.float16": F16}
_BYTES = {E4M3: ("torch.float8_e4m3fn", "torch.uint8"), INT8: ("torch.int8", "torch.uint8")}


class _Handle:
    """What handles have in common: prepared calls and their end."""

    _prefix = None  # of the library's symbols

    # Each operator as a prepared call (marshalled once: f() -> status) and as a call that raises.
    def _prepared(self, name, args, keep):
        fn, ref = getattr(self._lib, self._prefix + name), C.byref(args)

        def call(_keep=(args, keep)):
            return fn(self._h, ref)  # (destroyed meanwhile: None, which is E_STATE)
        call.operator = self._prefix + name
        return call

    @staticmethod
    def _now(call):
        rc = call()
        if rc != OK:
            raise PastaError(rc, call.operator)

    def destroy(self):
        if self._h is not None:
            getattr(self._lib, self._prefix + "destroy")(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


class _Attention(_Handle):
    """Plan and attention, alike for every paged cache."""

    def prepare_plan(self, length, row_offsets, n_rows, *, max_request_rows=None, prefix_len=None, slot=None, n_requests=None):
        R = n_requests if n_requests is not None else int(length.shape[0])
        a = PlanArgs(C.sizeof(PlanArgs), 0, R, n_rows, n_rows if max_request_rows is None else max_request_rows, _p(length, _I32, (R,), "length"),
                     _p(row_offsets, _I32, (R + 1,), "row_offsets"), _p(prefix_len, _I32, (R,), "prefix_len"), _p(slot, _I32, (n_rows,), "slot"))
        return self._prepared("plan", a, (length, row_offsets, prefix_len, slot))

    def prepare_attend(self, layer, q, out, *, lse=None, logit_cap=0.0, slopes=None, row_see=None, row_position=None, n_rows=None):
        c = self.cfg
        n = n_rows if n_rows is not None else int(q.shape[0])
        shape = (n, c.n_q_heads, c.head_dim)
        of = tuple(k for k, v in _ROWS.items() if v == c.dtype)
        a = AttendArgs(C.sizeof(AttendArgs), 0, layer, n, logit_cap, _p(q, of, shape, "q"), _p(out, of, shape, "out"),
                       _p(lse, _F32, (n, c.n_q_heads), "lse"), _p(slopes, _F32, (c.n_q_heads,), "slopes"),
                       _p(row_see, ("torch.int64", "torch.uint64"), (n,), "row_see"), _p(row_position, _I32, (n,), "row_position"))
        return self._prepared("attend", a, (q, out, lse, slopes, row_see, row_position))

    def plan(self, *args, **kw):
        self._now(self.prepare_plan(*args, **kw))

    def attend(self, *args, **kw):
        self._now(self.prepare_attend(*args, **kw))


class PastaKv8(_Attention):
    """One handle.  Buffers are device addresses (or torch tensors, which are then kept alive and checked for type, contiguity,
    size and device) owned by the caller; those that no call needs may be left out.  `stream` is a hipStream_t as an int."""

    _prefix = "pasta_kv8_"

    def __init__(self, cfg: Config, workspace, *, page_table=None, k_codes=None, v_codes=None, k_scale=None, v_scale=None, free_pages=None,
                 slot_tag=None, slot_position=None, stream=0, workspace_bytes=None):
        self._h = None
        self._lib = load_library()
        self.cfg = cfg
        self._keep = [workspace, page_table, k_codes, v_codes, k_scale, v_scale, free_pages, slot_tag, slot_position]
        k_shape, v_shape, s_shape = cache_shapes(cfg)
        slots = (cfg.n_phys_pages * cfg.page_tokens,)
        cfg.k_codes, cfg.v_codes = _p(k_codes, _BYTES.get(cfg.codes), k_shape, "k_codes"), _p(v_codes, _BYTES.get(cfg.codes), v_shape, "v_codes")
        cfg.k_scale, cfg.v_scale = _p(k_scale, _F32, s_shape, "k_scale"), _p(v_scale, _F32, s_shape, "v_scale")
        cfg.page_table = _p(page_table, _I32, (cfg.max_requests, cfg.pages_per_request), "page_table")
        cfg.free_pages = _p(free_pages, _I32, (cfg.n_phys_pages,), "free_pages")
        cfg.slot_tag, cfg.slot_position = _p(slot_tag, _U8, slots, "slot_tag"), _p(slot_position, _I32, slots, "slot_position")
        cfg.workspace = _p(workspace, _U8, (1,), "workspace")
        cfg.workspace_bytes = workspace_bytes if workspace_bytes is not None else (0 if isinstance(workspace, int) else workspace.numel())
        cfg.hip_stream = stream
        h = C.c_void_p()
        rc = self._lib.pasta_kv8_create(C.byref(cfg), C.byref(h))
        if rc != OK:
            raise PastaError(rc, "pasta_kv8_create")
        self._h = h

    def prepare_slots(self, length, row_offsets, n_rows, slot, length_out, free_count, free_out, *, keep=None, row_tag=None, row_position=None,
                      n_requests=None):
        R = n_requests if n_requests is not None else int(length.shape[0])
        a = SlotsArgs(C.sizeof(SlotsArgs), 0, R, n_rows, _p(length, _I32, (R,), "length"), _p(keep, _I32, (R,), "keep"),
                      _p(row_offsets, _I32, (R + 1,), "row_offsets"), _p(row_tag, _U8, (n_rows,), "row_tag"),
                      _p(row_position, _I32, (n_rows,), "row_position"), _p(free_count, _I32, (1,), "free_count"), _p(slot, _I32, (n_rows,), "slot"),
                      _p(length_out, _I32, (R,), "length_out"), _p(free_out, _I32, (1,), "free_out"))
        return self._prepared("slots", a, (length, row_offsets, slot, length_out, free_count, free_out, keep, row_tag, row_position))

    def prepare_append(self, layer, slot, k_new, v_new, *, n_rows=None, dtype=None):
        n = n_rows if n_rows is not None else int(slot.shape[0])
        if dtype is None:
            dtype = _ROWS.get(str(k_new.dtype), -1)
        shape = (n, self.cfg.n_kv_heads, self.cfg.head_dim)
        of = tuple(k for k, v in _ROWS.items() if v == _DTYPES.get(dtype, dtype)) or None
        a = AppendArgs(C.sizeof(AppendArgs), 0, layer, n, _DTYPES.get(dtype, dtype), _p(slot, _I32, (n,), "slot"), _p(k_new, of, shape, "k_new"),
                       _p(v_new, of, shape, "v_new"))
        return self._prepared("append", a, (slot, k_new, v_new))

    def slots(self, *args, **kw):
        self._now(self.prepare_slots(*args, **kw))

    def append(self, *args, **kw):
        self._now(self.prepare_append(*args, **kw))
