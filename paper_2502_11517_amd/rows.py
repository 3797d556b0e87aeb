"""Thin ctypes binding of libpasta_rows.so (include/pasta_rows.h): rotary positions of a step's rows, and drafted tokens against the target's probabilities.

Argument marshalling only, as in kv8.py; and the frequencies of a rotation, which the host computes once.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import subprocess

from .binding import BF16, E_CAPACITY, E_DEVICE, E_INVAL, E_NOMEM, E_STATE, F32, HIPCC_FLAGS, OK, PastaError  # noqa: F401
from .kv4 import _row_type, _strided
from .kv8 import _DTYPES, _F32, _I32, _U8, F16, _Handle, _p  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_HERE, "libpasta_rows.so")
_lib = None

HALF, INTERLEAVED = 0, 1
BACKWARD = 1  # flag of rotate
_LAYOUTS = {"half": HALF, "interleaved": INTERLEAVED}


def library_path() -> str:
    return _LIB


def build_library(verbose: bool = False) -> str:
    """Compiles csrc/pasta_rows.hip for gfx950 with hipcc (cross-compiles without a GPU)."""
    cmd = ["hipcc", *HIPCC_FLAGS, os.path.join(_HERE, "csrc", "pasta_rows.hip"), "-o", _LIB]
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError("hipcc failed:\n" + r.stderr)
    if verbose:
        print(" ".join(cmd))
    return _LIB


class Config(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("max_rows", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("rope_dims", C.c_int32), ("rope_layout", C.c_int32), ("rope_magnitude", C.c_float), ("rope_frequency", C.c_void_p), ("vocab", C.c_int32),
        ("max_sequences", C.c_int32), ("workspace", C.c_void_p), ("workspace_bytes", C.c_uint64), ("hip_stream", C.c_void_p),
    ]


class RotateArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_rows", C.c_int32), ("dtype", C.c_int32), ("position", C.c_void_p), ("q", C.c_void_p),
        ("k", C.c_void_p), ("q_out", C.c_void_p), ("k_out", C.c_void_p), ("q_stride", C.c_int64), ("k_stride", C.c_int64), ("q_out_stride", C.c_int64),
        ("k_out_stride", C.c_int64),
    ]


class VerifyArgs(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32), ("flags", C.c_uint32), ("n_sequences", C.c_int32), ("n_rows", C.c_int32), ("dtype", C.c_int32),
        ("row_offsets", C.c_void_p), ("token", C.c_void_p), ("slot", C.c_void_p), ("target", C.c_void_p), ("draft", C.c_void_p), ("target_stride", C.c_int64),
        ("draft_stride", C.c_int64), ("draw", C.c_void_p), ("last_draw", C.c_void_p), ("length", C.c_void_p), ("row_position", C.c_void_p),
        ("accepted", C.c_void_p), ("next_token", C.c_void_p), ("keep", C.c_void_p), ("position_out", C.c_void_p),
    ]


def load_library():
    """Loads the built library; raises if it is missing (there is no other path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB):
            raise RuntimeError(f"{_LIB} is not built: run __graft_entry__.build() (hipcc, gfx950)")
        import torch  # noqa: F401  (binds the library to torch's HIP runtime, as in binding.load_library)
        L = C.CDLL(_LIB)
        L.pasta_rows_create.restype, L.pasta_rows_create.argtypes = C.c_int32, [C.POINTER(Config), C.POINTER(C.c_void_p)]
        L.pasta_rows_destroy.restype, L.pasta_rows_destroy.argtypes = C.c_int32, [C.c_void_p]
        for name, args in (("rotate", RotateArgs), ("verify", VerifyArgs)):
            f = getattr(L, "pasta_rows_" + name)
            f.restype, f.argtypes = C.c_int32, [C.c_void_p, C.POINTER(args)]
        _lib = L
    return _lib


def rope_frequencies(dims, theta=10000.0, *, scaling="none", factor=1.0, trained=4096, slow=1.0, fast=32.0):
    """(radians a position, of each of dims / 2 planes; magnitude): theta^(-2i / dims), for contexts `factor` times as long as the `trained` one

      none    as they are
      linear  divided by the factor: positions are closer to each other
      base    theta times factor^(dims / (dims - 2)): the slowest plane is as much slower, the fastest as fast as before
      parts   planes with `fast` turns or more over the trained context stay, those with `slow` or fewer are divided by the factor, between them in proportion;
              the magnitude is 0.1 ln(factor) + 1
    """
    if dims < 2 or dims % 2 or not theta > 0 or not factor >= 1:
        raise ValueError("an even number of dims, theta > 0, factor >= 1")
    if scaling == "base" and dims > 2:
        theta *= factor ** (dims / (dims - 2.0))
    f = [theta ** (-2.0 * i / dims) for i in range(dims // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "parts":
        if not fast > slow:
            raise ValueError("fast > slow")
        kept = [min(max((trained * x / (2.0 * math.pi) - slow) / (fast - slow), 0.0), 1.0) for x in f]
        return [x * (k + (1.0 - k) / factor) for x, k in zip(f, kept)], 0.1 * math.log(factor) + 1.0
    if scaling not in ("none", "base"):
        raise ValueError(f"scaling {scaling!r}")
    return f, 1.0


def make_config(*, max_rows=1, n_q_heads=0, n_kv_heads=0, head_dim=0, rope_dims=0, rope_layout="half", rope_frequency=None, rope_magnitude=1.0, vocab=0,
                max_sequences=0) -> Config:
    """`rope_frequency`: radians a position, rope_dims / 2 numbers (rope_frequencies) or a float64 tensor of them on the GPU, which saves every handle a copy."""
    c = Config()
    c.struct_size = C.sizeof(Config)
    c.max_rows, c.n_q_heads, c.n_kv_heads, c.head_dim = max_rows, n_q_heads, n_kv_heads, head_dim
    c.rope_dims = rope_dims
    if rope_dims:
        c.rope_layout, c.rope_magnitude = _LAYOUTS.get(rope_layout, rope_layout), rope_magnitude
    c.vocab, c.max_sequences = vocab, max_sequences
    c.frequency = rope_frequency  # (PastaRows puts it on the device)
    return c


def query_workspace_bytes(cfg: Config) -> int:
    rc = load_library().pasta_rows_create(C.byref(cfg), None)
    if rc != OK:
        raise PastaError(rc, "pasta_rows_create(query)")
    return int(cfg.workspace_bytes)


class PastaRows(_Handle):
    """One handle.  Buffers are device addresses (or torch tensors, which are then kept alive and checked for type, contiguity, size and device) owned by
    the caller.  `stream` is a hipStream_t as an int; `device` is where frequencies given as numbers go, the current one by default."""

    _prefix = "pasta_rows_"

    def __init__(self, cfg: Config, workspace=None, *, stream=0, workspace_bytes=None, device=None):
        self._h = None
        self._lib = load_library()
        self.cfg = cfg
        f = cfg.frequency
        if cfg.rope_dims and f is not None and not isinstance(f, int):
            import torch

            if not torch.is_tensor(f):
                f = torch.tensor([float(x) for x in f], dtype=torch.float64, device=device if device is not None else "cuda")
            if f.numel() != cfg.rope_dims // 2:
                raise ValueError(f"rope_frequency: {f.numel()} numbers, {cfg.rope_dims // 2} are wanted")
            f = (f, _p(f, ("torch.float64",), (cfg.rope_dims // 2,), "rope_frequency"))
        self._keep = [workspace, f]
        cfg.rope_frequency = f[1] if isinstance(f, tuple) else f
        cfg.workspace = _p(workspace, _U8, (0,), "workspace") or None
        cfg.workspace_bytes = workspace_bytes if workspace_bytes is not None else (0 if workspace is None or isinstance(workspace, int) else workspace.numel())
        cfg.hip_stream = stream
        h = C.c_void_p()
        rc = self._lib.pasta_rows_create(C.byref(cfg), C.byref(h))
        if rc != OK:
            raise PastaError(rc, "pasta_rows_create")
        self._h = h

    def _rows(self, x, n, heads, of, what):
        return (x, 0) if x is None or isinstance(x, int) else _strided(x, n, heads, self.cfg.head_dim, of, what)

    def prepare_rotate(self, position, q=None, q_out=None, k=None, k_out=None, *, backward=False, n_rows=None, dtype=None):
        """q [n, Hq, D] to q_out, k [n, Hkv, D] to k_out; either pair may be left out, and out may be in."""
        c = self.cfg
        n = n_rows if n_rows is not None else int(position.shape[0])
        dtype, of = _row_type(dtype, q if q is not None else k)
        (qa, qs), (qo, qos) = self._rows(q, n, c.n_q_heads, of, "q"), self._rows(q_out, n, c.n_q_heads, of, "q_out")
        (ka, ks), (ko, kos) = self._rows(k, n, c.n_kv_heads, of, "k"), self._rows(k_out, n, c.n_kv_heads, of, "k_out")
        a = RotateArgs(C.sizeof(RotateArgs), BACKWARD if backward else 0, n, dtype, _p(position, _I32, (n,), "position"), qa, ka, qo, ko, qs, ks, qos, kos)
        return self._prepared("rotate", a, (position, q, q_out, k, k_out))

    def prepare_verify(self, row_offsets, token, target, draw, last_draw, accepted, next_token, *, draft=None, length=None, keep=None, row_position=None,
                       position_out=None, slot=None, n_sequences=None, n_rows=None, dtype=None):
        S = n_sequences if n_sequences is not None else int(row_offsets.shape[0]) - 1
        n = n_rows if n_rows is not None else int(token.shape[0])
        dtype, of = _row_type(dtype, target)
        (p, ps), (q, qs) = self._distributions(target, n, of, "target"), self._distributions(draft, n, of, "draft")
        i32 = lambda x, k, what: _p(x, _I32, (k,), what)  # noqa: E731
        a = VerifyArgs(C.sizeof(VerifyArgs), 0, S, n, dtype, i32(row_offsets, S + 1, "row_offsets"), i32(token, n, "token"), i32(slot, n, "slot"), p, q, ps, qs,
                       _p(draw, _F32, (n,), "draw"), _p(last_draw, _F32, (S,), "last_draw"), i32(length, S, "length"), i32(row_position, n, "row_position"),
                       i32(accepted, S, "accepted"), i32(next_token, S, "next_token"), i32(keep, S, "keep"), i32(position_out, n, "position_out"))
        return self._prepared("verify", a, (row_offsets, token, target, draw, last_draw, accepted, next_token, draft, length, keep, row_position, position_out, slot))

    def _distributions(self, x, n, of, what):
        """(address, values between rows) of a tensor [n, vocab or more]."""
        if x is None or isinstance(x, int):
            return x, 0
        if of is not None and str(x.dtype) not in of:
            raise ValueError(f"{what}: {x.dtype}, one of {of} is wanted")
        V = self.cfg.vocab
        if x.dim() != 2 or x.shape[0] < n or x.shape[1] < V or (V > 1 and x.stride(1) != 1) or (n > 1 and x.stride(0) < V):
            raise ValueError(f"{what}: {tuple(x.shape)}, strides {x.stride()}, {(n, V)} in rows of neighbouring values is wanted")
        if not x.is_cuda:
            raise ValueError(f"{what}: on {x.device}, device memory is wanted")
        return x.data_ptr(), x.stride(0) if n > 1 else 0

    def rotate(self, *args, **kw):
        self._now(self.prepare_rotate(*args, **kw))

    def verify(self, *args, **kw):
        self._now(self.prepare_verify(*args, **kw))
