"""Thin Python binding of liblosa.so (include/losa.h).

Argument marshalling only: torch tensors in, device pointers and sizes out,
the current HIP stream passed through.  Every step of the computation runs in
the library's HIP kernels; if the library is missing this module raises on
import instead of falling back to anything else.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# the in-tree build; LOSA_LIBRARY names another build of the same sources
# (the host-sanitizer check uses it)
LIB_PATH = os.environ.get("LOSA_LIBRARY") or os.path.join(_HERE, "liblosa.so")

LOSA_DTYPE_F32 = 0
LOSA_DTYPE_BF16 = 1
_DTYPES = {torch.float32: LOSA_DTYPE_F32, torch.bfloat16: LOSA_DTYPE_BF16}
STATUS = {0: "LOSA_OK", 1: "LOSA_ERR_NULL_POINTER", 2: "LOSA_ERR_INVALID_SHAPE",
          3: "LOSA_ERR_INVALID_TAU", 4: "LOSA_ERR_ALIGNMENT", 5: "LOSA_ERR_UNSUPPORTED",
          6: "LOSA_ERR_CAPACITY", 7: "LOSA_ERR_HIP"}

EXPORTED = ("losa_calibrate_mass", "losa_select_blocks", "losa_select_blocks_topk",
            "losa_block_recall", "losa_sparse_attn_fwd", "losa_sparse_attn_fwd_noalloc",
            "losa_construct", "losa_rope_table", "losa_rope", "losa_qk_norm_rope",
            "losa_packed_plan", "losa_packed_workspace_bytes", "losa_packed_attn_fwd",
            "losa_workspace_bytes", "losa_status_string", "losa_last_error",
            "losa_version")

# bytes of library-held scratch behind losa_sparse_attn_fwd_noalloc (per GPU)
NOALLOC_SCRATCH_BYTES = 128 << 20


PAIRS = {"interleaved": 0, "halves": 1}
NORMS = {"rms": 1, "layer": 2}
MAX_AXES = 4


# Structures of the C ABI as bytes, which ctypes passes by address: losa_view (data, batch,
# token, head), losa_rotation (n_axes, axis_dim, axis_len; table, pos, pos_batch, pairs) and
# losa_qk_norm_args (kind, all_heads, eps; weights and biases)
_VIEW = struct.Struct("@Qqqq").pack
_AXES = struct.Struct("@9i4x").pack
_ROTATION = struct.Struct("@QQqi4x").pack
_QK_NORM = struct.Struct("@iif4xQQQQ").pack


class _PackedInfo(ctypes.Structure):
    """losa_packed_info"""
    _fields_ = [("bytes", ctypes.c_int64), ("q_rows", ctypes.c_int64), ("k_rows", ctypes.c_int64),
                ("part_rows", ctypes.c_int64), ("q_run", ctypes.c_int64),
                ("n_tiles", ctypes.c_int32), ("n_few", ctypes.c_int32),
                ("n_joins", ctypes.c_int32), ("n_wide", ctypes.c_int32),
                ("tile_rows", ctypes.c_int32), ("H", ctypes.c_int32),
                ("H_kv", ctypes.c_int32), ("causal", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class LosaError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)}: {detail}")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2608_12032_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    P, I, F, Z, L = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.c_int64
    lib.losa_calibrate_mass.argtypes = [P, P, I, I, I, I, I, I, I, F, P, P, P, Z, P]
    lib.losa_calibrate_mass.restype = I
    lib.losa_select_blocks.argtypes = [P, I, I, I, I, I, F, P, P, L, P, Z, P]
    lib.losa_select_blocks.restype = I
    lib.losa_select_blocks_topk.argtypes = [P, I, I, I, I, I, I, P, P, L, P, Z, P]
    lib.losa_select_blocks_topk.restype = I
    lib.losa_block_recall.argtypes = [P, I, I, I, I, I, P, P, L, P, P, P, Z, P]
    lib.losa_block_recall.restype = I
    lib.losa_sparse_attn_fwd.argtypes = [P, P, P, I, I, I, I, I, I, I, F, P, P, L, P, P, P, Z, P]
    lib.losa_sparse_attn_fwd.restype = I
    lib.losa_sparse_attn_fwd_noalloc.argtypes = [P, P, P, I, I, I, I, I, I, I, F, P, P, L, P, P,
                                                 P]
    lib.losa_sparse_attn_fwd_noalloc.restype = I
    lib.losa_construct.argtypes = [P, P, P, I, I, I, I, I, I, I, F, P, P, P, P, Z, P]
    lib.losa_construct.restype = I
    # structures by address: a pointer to one, or None
    lib.losa_rope_table.argtypes = [I, P, P, ctypes.c_double, P, L]
    lib.losa_rope_table.restype = I
    lib.losa_rope.argtypes = [P, I, I, I, I, I, I, P, P, P]
    lib.losa_rope.restype = I
    lib.losa_qk_norm_rope.argtypes = [P, P, P, I, I, I, I, I, I, I, P, P, P, P, P, P]
    lib.losa_qk_norm_rope.restype = I
    lib.losa_packed_plan.argtypes = [P, P, P, P, I, I, I, I, I, P, Z, P]
    lib.losa_packed_plan.restype = I
    lib.losa_packed_workspace_bytes.argtypes = [P, I]
    lib.losa_packed_workspace_bytes.restype = Z
    lib.losa_packed_attn_fwd.argtypes = [P, P, P, L, L, P, P, I, F, P, P, L, P, Z, P]
    lib.losa_packed_attn_fwd.restype = I
    lib.losa_workspace_bytes.argtypes = [I, I, I, I, I, I, I, I]
    lib.losa_workspace_bytes.restype = Z
    lib.losa_status_string.argtypes = [I]
    lib.losa_status_string.restype = ctypes.c_char_p
    lib.losa_last_error.argtypes = []
    lib.losa_last_error.restype = ctypes.c_char_p
    lib.losa_version.argtypes = []
    lib.losa_version.restype = I
    return lib


lib = _load()


def _check(st: int, where: str):
    if st != 0:
        raise LosaError(st, where, lib.losa_last_error().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return LOSA_DTYPE_BF16
    if t.dtype == torch.float32:
        return LOSA_DTYPE_F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _stream(device) -> int:
    """The current stream's handle, without building a torch.cuda.Stream."""
    return torch._C._cuda_getCurrentRawStream(device.index)


def _arg(t, name, device, dtype=None, shape=None, numel=None, nbytes=None):
    """Check a tensor argument before its pointer reaches the library, which
    sees raw device pointers and cannot tell a host tensor, a wrong element
    type or a short buffer from a valid one."""
    # (a call makes up to eight of these: one expression for what is in order)
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.device == device and t.is_contiguous()
            and (dtype is None or t.dtype == dtype) and (shape is None or t.shape == shape)
            and (numel is None or t.numel() >= numel) and (nbytes is None or t.nbytes >= nbytes)):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must live on {device} (got {t.device})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {numel}")
    if nbytes is not None and t.numel() * t.element_size() < nbytes:
        raise ValueError(f"{name} holds {t.numel() * t.element_size()} bytes, needs {nbytes}")
    return t


def _qkv(q, others, N: int, block_q: int, block_k: int):
    """Shape of Q ([B, H, N_pad, d] on a GPU, N_pad = padded_len(N, ...)), and
    K / V alike."""
    if not isinstance(q, torch.Tensor) or q.dim() != 4:
        raise ValueError("q must be a [B, H, N_pad, d] tensor")
    _arg(q, "q", q.device)
    B, H, Np, d = q.shape
    if N < 1 or Np != padded_len(N, block_q, block_k):
        raise ValueError(f"q has N_pad = {Np}; N = {N} with blocks {block_q} x {block_k} "
                         f"needs {padded_len(max(N, 1), block_q, block_k)}")
    for name, t in others.items():
        _arg(t, name, q.device, dtype=q.dtype, shape=q.shape)
    return B, H, Np, d


def _mass_shape(mass, N: int, block_q: int, block_k: int):
    if not isinstance(mass, torch.Tensor) or mass.dim() != 4:
        raise ValueError("mass must be a [B, H, n_q, n_k] tensor")
    Np = padded_len(N, block_q, block_k)
    B, H = mass.shape[:2]
    _arg(mass, "mass", mass.device, dtype=torch.float32, shape=(B, H, Np // block_q,
                                                                  Np // block_k))
    return B, H, Np // block_q, Np // block_k


def padded_len(N: int, block_q: int, block_k: int) -> int:
    L = max(block_q, block_k)
    return -(-N // L) * L


def workspace_bytes(which: int, dtype_code: int, B, H, N, d, block_q, block_k) -> int:
    return int(lib.losa_workspace_bytes(which, dtype_code, B, H, N, d, block_q, block_k))


_kept = functools.lru_cache(maxsize=1024)(workspace_bytes)
_INTS = (int,) * 8


def _need(*args) -> int:
    """The same numbers, kept: a call with a workspace asks for its size each
    time.  Only for plain ints, which are their values: a size held in a tensor is
    hashed by identity, whatever it holds later, and one in an array not at all."""
    return (_kept if tuple(map(type, args)) == _INTS else workspace_bytes)(*args)


def losa_calibrate_mass(q, k, N: int, block_q: int, block_k: int | None = None,
                        scale: float | None = None, want_lse: bool = True, mass=None, lse=None,
                        workspace=None, two_sweep: bool = False):
    """Exact block masses of a dense step -> (mass [B,H,n_q,n_k] fp32, lse or None).

    bf16 takes one sweep over the keys plus a reduction of per-(query, key
    block) statistics held in ``workspace`` (allocated at the suggested size
    when not given); ``two_sweep=True`` passes no workspace and takes two
    sweeps instead."""
    block_k = block_k or block_q
    B, H, Np, d = _qkv(q, {"k": k}, N, block_q, block_k)
    dev = q.device
    n_q, n_k = Np // block_q, Np // block_k
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    if mass is None:
        mass = torch.empty((B, H, n_q, n_k), dtype=torch.float32, device=dev)
    _arg(mass, "mass", dev, dtype=torch.float32, shape=(B, H, n_q, n_k))
    if want_lse and lse is None:
        lse = torch.empty((B, H, Np), dtype=torch.float32, device=dev)
    if not want_lse:
        lse = None
    if lse is not None:
        _arg(lse, "lse", dev, dtype=torch.float32, shape=(B, H, Np))
    dcode = _dtype_code(q)
    if two_sweep or dcode != LOSA_DTYPE_BF16:
        workspace = None
    elif workspace is None:
        need = _need(0, dcode, B, H, N, d, block_q, block_k)
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if workspace is not None:
        _arg(workspace, "workspace", dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = lib.losa_calibrate_mass(_ptr(q), _ptr(k), dcode, B, H, N, d, block_q, block_k,
                                 scale, _ptr(mass), _ptr(lse), _ptr(workspace), ws_bytes,
                                 _stream(dev))
    _check(st, "losa_calibrate_mass")
    return mass, lse


def _csr_out(row_ptr, col_idx, workspace, rows, n_k, dev, need):
    if row_ptr is None:
        row_ptr = torch.empty(rows + 1, dtype=torch.int32, device=dev)
    if col_idx is None:
        col_idx = torch.empty(rows * n_k, dtype=torch.int32, device=dev)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    _arg(row_ptr, "row_ptr", dev, dtype=torch.int32, numel=rows + 1)
    _arg(col_idx, "col_idx", dev, dtype=torch.int32)
    _arg(workspace, "workspace", dev, nbytes=need)
    return row_ptr, col_idx, workspace


def losa_select_blocks(mass, N: int, block_q: int, block_k: int | None, tau: float,
                       row_ptr=None, col_idx=None, workspace=None):
    """Shortest-prefix selection -> (row_ptr int32 [rows+1], col_idx int32 buffer).

    col_idx has the worst-case capacity B*H*n_q*n_k; its first row_ptr[-1]
    entries are valid (read row_ptr[-1] after a sync, or use ``nnz``).
    """
    block_k = block_k or block_q
    B, H, n_q, n_k = _mass_shape(mass, N, block_q, block_k)
    rows = B * H * n_q
    dev = mass.device
    need = _need(1, LOSA_DTYPE_F32, B, H, N, 1, block_q, block_k)
    row_ptr, col_idx, workspace = _csr_out(row_ptr, col_idx, workspace, rows, n_k, dev, need)
    st = lib.losa_select_blocks(_ptr(mass), B, H, N, block_q, block_k, float(tau),
                                _ptr(row_ptr), _ptr(col_idx), col_idx.numel(), _ptr(workspace),
                                workspace.numel() * workspace.element_size(), _stream(dev))
    _check(st, "losa_select_blocks")
    return row_ptr, col_idx


def losa_select_blocks_topk(mass, N: int, block_q: int, block_k: int | None, k: int,
                            row_ptr=None, col_idx=None, workspace=None):
    """Fixed-ratio top-k selection (k blocks per row) -> (row_ptr, col_idx buffer)."""
    block_k = block_k or block_q
    B, H, n_q, n_k = _mass_shape(mass, N, block_q, block_k)
    rows = B * H * n_q
    dev = mass.device
    need = _need(1, LOSA_DTYPE_F32, B, H, N, 1, block_q, block_k)
    row_ptr, col_idx, workspace = _csr_out(row_ptr, col_idx, workspace, rows, n_k, dev, need)
    st = lib.losa_select_blocks_topk(_ptr(mass), B, H, N, block_q, block_k, int(k),
                                     _ptr(row_ptr), _ptr(col_idx), col_idx.numel(),
                                     _ptr(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(dev))
    _check(st, "losa_select_blocks_topk")
    return row_ptr, col_idx


def losa_block_recall(mass, N: int, block_q: int, block_k: int | None, row_ptr, col_idx,
                      want_rows: bool = True, want_heads: bool = True, workspace=None):
    """Recall of a frozen support on these masses -> (recall_rows or None, recall_heads or None)."""
    block_k = block_k or block_q
    B, H, n_q, n_k = _mass_shape(mass, N, block_q, block_k)
    dev = mass.device
    _arg(row_ptr, "row_ptr", dev, dtype=torch.int32, numel=B * H * n_q + 1)
    _arg(col_idx, "col_idx", dev, dtype=torch.int32)
    rec_rows = torch.empty(B * H * n_q, dtype=torch.float32, device=dev) if want_rows else None
    rec_heads = torch.empty((B, H), dtype=torch.float32, device=dev) if want_heads else None
    need = _need(3, LOSA_DTYPE_F32, B, H, N, 1, block_q, block_k)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    _arg(workspace, "workspace", dev, nbytes=need)
    st = lib.losa_block_recall(_ptr(mass), B, H, N, block_q, block_k, _ptr(row_ptr),
                               _ptr(col_idx), col_idx.numel(), _ptr(rec_rows), _ptr(rec_heads),
                               _ptr(workspace), workspace.numel() * workspace.element_size(),
                               _stream(dev))
    _check(st, "losa_block_recall")
    return rec_rows, rec_heads


def nnz(row_ptr) -> int:
    return int(row_ptr[-1].item())


def losa_sparse_attn_fwd(q, k, v, N: int, block_q: int, block_k: int | None, row_ptr, col_idx,
                         scale: float | None = None, want_lse: bool = False, out=None,
                         lse=None, workspace=None):
    """Frozen-support block-sparse attention -> o (and lse if requested)."""
    block_k = block_k or block_q
    B, H, Np, d = _qkv(q, {"k": k, "v": v}, N, block_q, block_k)
    dev = q.device
    _arg(row_ptr, "row_ptr", dev, dtype=torch.int32, numel=B * H * (Np // block_q) + 1)
    _arg(col_idx, "col_idx", dev, dtype=torch.int32)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    dcode = _dtype_code(q)
    o = torch.empty_like(q) if out is None else out
    _arg(o, "out", dev, dtype=q.dtype, shape=q.shape)
    if want_lse and lse is None:
        lse = torch.empty((B, H, Np), dtype=torch.float32, device=dev)
    if want_lse:
        _arg(lse, "lse", dev, dtype=torch.float32, shape=(B, H, Np))
    need = _need(2, dcode, B, H, N, d, block_q, block_k)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if workspace is not None:
        _arg(workspace, "workspace", dev, nbytes=need)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = lib.losa_sparse_attn_fwd(_ptr(q), _ptr(k), _ptr(v), dcode, B, H, N, d, block_q, block_k,
                                  scale, _ptr(row_ptr), _ptr(col_idx), col_idx.numel(), _ptr(o),
                                  _ptr(lse if want_lse else None), _ptr(workspace), ws_bytes,
                                  _stream(dev))
    _check(st, "losa_sparse_attn_fwd")
    return (o, lse) if want_lse else o


def losa_sparse_attn_fwd_noalloc(q, k, v, N: int, block_q: int, block_k: int | None, row_ptr,
                                 col_idx, scale: float | None = None, want_lse: bool = False,
                                 out=None, lse=None):
    """losa_sparse_attn_fwd without a workspace: the library's own scratch
    (NOALLOC_SCRATCH_BYTES per GPU) holds it.  Allocates only the outputs
    that are not given; pass ``out`` (and ``lse``) to allocate nothing."""
    block_k = block_k or block_q
    B, H, Np, d = _qkv(q, {"k": k, "v": v}, N, block_q, block_k)
    dev = q.device
    _arg(row_ptr, "row_ptr", dev, dtype=torch.int32, numel=B * H * (Np // block_q) + 1)
    _arg(col_idx, "col_idx", dev, dtype=torch.int32)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o = torch.empty_like(q) if out is None else out
    _arg(o, "out", dev, dtype=q.dtype, shape=q.shape)
    if want_lse and lse is None:
        lse = torch.empty((B, H, Np), dtype=torch.float32, device=dev)
    if want_lse:
        _arg(lse, "lse", dev, dtype=torch.float32, shape=(B, H, Np))
    if torch.cuda.current_device() != dev.index:
        raise ValueError(f"the tensors live on {dev}; make it the current device")
    st = lib.losa_sparse_attn_fwd_noalloc(_ptr(q), _ptr(k), _ptr(v), _dtype_code(q), B, H, N, d,
                                          block_q, block_k, scale, _ptr(row_ptr), _ptr(col_idx),
                                          col_idx.numel(), _ptr(o),
                                          _ptr(lse if want_lse else None), _stream(dev))
    _check(st, "losa_sparse_attn_fwd_noalloc")
    return (o, lse) if want_lse else o


def losa_construct(q, k, v, N: int, block_q: int, block_k: int | None = None,
                   scale: float | None = None, want_lse: bool = False, out=None, mass=None,
                   lse=None, workspace=None):
    """Construction step: dense attention output and exact block masses of the
    same step -> (o, mass) or (o, mass, lse)."""
    block_k = block_k or block_q
    B, H, Np, d = _qkv(q, {"k": k, "v": v}, N, block_q, block_k)
    dev = q.device
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    dcode = _dtype_code(q)
    o = torch.empty_like(q) if out is None else out
    _arg(o, "out", dev, dtype=q.dtype, shape=q.shape)
    if mass is None:
        mass = torch.empty((B, H, Np // block_q, Np // block_k), dtype=torch.float32, device=dev)
    _arg(mass, "mass", dev, dtype=torch.float32, shape=(B, H, Np // block_q, Np // block_k))
    if want_lse and lse is None:
        lse = torch.empty((B, H, Np), dtype=torch.float32, device=dev)
    if not want_lse:
        lse = None
    if lse is not None:
        _arg(lse, "lse", dev, dtype=torch.float32, shape=(B, H, Np))
    need = _need(4, dcode, B, H, N, d, block_q, block_k)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if workspace is not None:
        _arg(workspace, "workspace", dev)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = lib.losa_construct(_ptr(q), _ptr(k), _ptr(v), dcode, B, H, N, d, block_q, block_k, scale,
                            _ptr(o), _ptr(mass), _ptr(lse), _ptr(workspace), ws_bytes,
                            _stream(dev))
    _check(st, "losa_construct")
    return (o, mass, lse) if want_lse else (o, mass)


class RopeTable:
    """Cosines and sines by axis and position, on a device: what losa_rope_table returns.
    ``data`` fp32 (not to be replaced); ``axis_dim`` and ``axis_len`` as given."""

    def __init__(self, data, axis_dim, axis_len):
        self._data, self.axis_dim, self.axis_len = data, tuple(axis_dim), tuple(axis_len)
        floats = sum(a * b for a, b in zip(self.axis_dim, self.axis_len))
        if data.dtype != torch.float32 or not data.is_contiguous() or data.numel() < floats:
            raise ValueError(f"data must be contiguous fp32 of {floats} elements")
        self._axes = len(self.axis_dim)
        rest = (0,) * (MAX_AXES - self._axes)
        self._head = _AXES(self._axes, *self.axis_dim, *rest, *self.axis_len, *rest)

    @property
    def data(self):
        return self._data


def losa_rope_table(axis_dim, axis_len, base: float = 10000.0, device="cuda") -> RopeTable:
    """Table of a rotation: axis a turns ``axis_dim[a]`` dims by positions below
    ``axis_len[a]``, pair j of it by position * base^(-2j / axis_dim[a])."""
    axis_dim, axis_len = [int(x) for x in axis_dim], [int(x) for x in axis_len]
    if len(axis_dim) != len(axis_len):
        raise ValueError("axis_dim and axis_len must have the same length")
    n = len(axis_dim)
    host = torch.empty(max(0, sum(a * b for a, b in zip(axis_dim, axis_len))),
                       dtype=torch.float32)
    ints = ctypes.c_int * max(n, 1)
    # (a table without a float is refused: the pointer is never used)
    st = lib.losa_rope_table(n, ints(*axis_dim), ints(*axis_len), float(base),
                             host.data_ptr() or 16, host.numel())
    _check(st, "losa_rope_table")
    return RopeTable(host.to(device), axis_dim, axis_len)


def _wrong(t, name, device, dtype, shape):
    """Raises what is wrong with a view's tensor."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must live on {device} (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    raise ValueError(f"{name} must have contiguous rows (stride 1 in the last dim)")


def _view(t, name, device, dtype, shape):
    """losa_view of a [B, N, H, d] tensor of this shape whose rows of d are contiguous."""
    if (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype
            and t.shape == shape):
        sb, sn, sh, sd = t.stride()
        if sd == 1 and t.is_cuda:
            return _VIEW(t.data_ptr(), sb, sn, sh)
    _wrong(t, name, device, dtype, shape)


def _view_out(t, name, device, dtype, shape):
    """losa_view, as of [B, N, H, d], of a [B, H, N, d] tensor."""
    if (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype
            and t.shape == shape):
        sb, sh, sn, sd = t.stride()
        if sd == 1:
            return _VIEW(t.data_ptr(), sb, sn, sh)
    _wrong(t, name, device, dtype, shape)


def _rotation(table, pos, pairing, B, N, device):
    """losa_rotation of a table and positions int32 [axes, N] or [B, axes, N]."""
    if not isinstance(table, RopeTable):
        raise TypeError("table must be a RopeTable (losa_rope_table)")
    n, data = table._axes, table._data
    if data.device != device:
        raise ValueError(f"table must live on {device} (got {data.device})")
    _arg(pos, "pos", device, dtype=torch.int32)
    shape = pos.shape
    if shape == (n, N):
        batch = 0
    elif shape == (B, n, N):
        batch = n * N
    else:
        raise ValueError(f"pos must have shape {(n, N)} or {(B, n, N)} (got {tuple(shape)})")
    if pairing not in PAIRS:
        raise ValueError(f"pairing must be one of {tuple(PAIRS)} (got {pairing!r})")
    return table._head + _ROTATION(data.data_ptr(), pos.data_ptr(), batch, PAIRS[pairing])


def _rows_in(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 4:
        raise ValueError(f"{name} must be a [B, N, H, d] tensor")
    return t.shape


def _call(device, fn, *args):
    """fn(*args, stream) on the device's current stream, with that device current."""
    if torch._C._cuda_getDevice() == device.index:
        return fn(*args, _stream(device))
    with torch.cuda.device(device):
        return fn(*args, _stream(device))


def losa_rope(x, table: RopeTable, pos, n_pad: int | None = None, pairing: str = "interleaved",
              out=None):
    """Rotary positions of x [B, N, H, d] (any strides, rows of d contiguous) ->
    [B, H, n_pad, d], rows from N on 0.  ``pos`` int32 [axes, N] or [B, axes, N];
    ``out`` may have any strides, and may be x itself
    (x.transpose(1, 2) with n_pad = N)."""
    shape = B, N, H, d = _rows_in(x, "x")
    n_pad = N if n_pad is None else n_pad
    dev, dt, code = x.device, x.dtype, _dtype_code(x)
    xv = _view(x, "x", dev, dt, shape)
    rot = _rotation(table, pos, pairing, B, N, dev)
    if out is None:
        out = torch.empty((B, H, n_pad, d), dtype=dt, device=dev)
    yv = _view_out(out, "out", dev, dt, (B, H, n_pad, d))
    st = _call(dev, lib.losa_rope, xv, code, B, N, n_pad, H, d, rot, yv)
    if st:
        _check(st, "losa_rope")
    return out


def losa_qk_norm_rope(q, k, v=None, *, norm: str | None = "rms", over: str = "head",
                      q_weight=None, q_bias=None, k_weight=None, k_bias=None, eps: float = 1e-6,
                      table: RopeTable | None = None, pos=None, pairing: str = "interleaved",
                      n_pad: int | None = None, q_out=None, k_out=None, v_out=None):
    """Norms of q [B, N, H, d] and k [B, N, H_kv, d] over each head ("head") or all of a
    token's heads ("all"), then their rotary positions, in one pass; v beside them ->
    (q, k) or (q, k, v), each [B, heads, n_pad, d].  Inputs and outputs may have any
    strides; weights and biases fp32 of d or heads * d elements."""
    shape = B, N, H, d = _rows_in(q, "q")
    Hkv = _rows_in(k, "k")[2]
    dev, dt, code = q.device, q.dtype, _dtype_code(q)
    shape_kv = (B, N, Hkv, d)
    n_pad = N if n_pad is None else n_pad
    if over not in ("head", "all"):
        raise ValueError(f"over must be 'head' or 'all' (got {over!r})")
    qi, ki = _view(q, "q", dev, dt, shape), _view(k, "k", dev, dt, shape_kv)
    vi = None if v is None else _view(v, "v", dev, dt, shape_kv)
    args = None
    if norm is not None:
        if norm not in NORMS:
            raise ValueError(f"norm must be None or one of {tuple(NORMS)} (got {norm!r})")
        every = over == "all"
        span, span_kv = (H * d, Hkv * d) if every else (d, d)
        at = []
        for name, t, n in (("q_weight", q_weight, span), ("q_bias", q_bias, span),
                           ("k_weight", k_weight, span_kv), ("k_bias", k_bias, span_kv)):
            at.append(0 if t is None else
                      _arg(t, name, dev, dtype=torch.float32, shape=(n,)).data_ptr())
        args = _QK_NORM(NORMS[norm], every, eps, *at)
    elif not (q_weight is q_bias is k_weight is k_bias is None):
        raise ValueError("weights and biases need a norm")
    if (table is None) != (pos is None):
        raise ValueError("table and pos must both be given or both be None")
    rot = None if table is None else _rotation(table, pos, pairing, B, N, dev)
    if v is None and v_out is not None:
        raise ValueError("v_out needs v")
    shape, shape_kv = (B, H, n_pad, d), (B, Hkv, n_pad, d)
    if q_out is None:
        q_out = torch.empty(shape, dtype=dt, device=dev)
    if k_out is None:
        k_out = torch.empty(shape_kv, dtype=dt, device=dev)
    qo = _view_out(q_out, "q_out", dev, dt, shape)
    ko = _view_out(k_out, "k_out", dev, dt, shape_kv)
    vo = None
    if v is not None:
        if v_out is None:
            v_out = torch.empty(shape_kv, dtype=dt, device=dev)
        vo = _view_out(v_out, "v_out", dev, dt, shape_kv)
    st = _call(dev, lib.losa_qk_norm_rope, qi, ki, vi, code, B, N, n_pad, H, Hkv, d, args, rot, qo,
               ko, vo)
    if st:
        _check(st, "losa_qk_norm_rope")
    return (q_out, k_out) if v is None else (q_out, k_out, v_out)


class PackedPlan:
    """Plan of a batch of packed sequences on a device: what losa_packed_plan returns.
    ``info`` is a copy of its sizes (losa_packed_info), ``data`` the units of work (not to
    be replaced)."""

    def __init__(self, info, data, dtype):
        if _DTYPES.get(dtype) != info.dtype:
            raise ValueError(f"dtype {dtype} is not the one of the plan's sizes")
        if (data.dtype != torch.int64 or not data.is_contiguous()
                or data.numel() * 8 < max(8, info.bytes)):
            raise ValueError(f"data must be contiguous int64 of {info.bytes} bytes")
        # (as bytes, which belong to this object and its copies; ctypes passes their address)
        self._info, self._data, self._dtype = bytes(info), data, dtype
        self._heads, self._kv_heads = info.H, info.H_kv
        self._need = {d: int(lib.losa_packed_workspace_bytes(self._info, d)) for d in (64, 128)}

    @property
    def info(self):
        return _PackedInfo.from_buffer_copy(self._info)

    @property
    def data(self):
        return self._data

    @property
    def dtype(self):
        return self._dtype

    @property
    def heads(self):
        return self._heads

    @property
    def kv_heads(self):
        return self._kv_heads

    @property
    def q_rows(self):
        return self.info.q_rows

    @property
    def k_rows(self):
        return self.info.k_rows

    def workspace_bytes(self, d: int) -> int:
        return self._need.get(d, 0)

    def workspace(self, d: int):
        """A workspace for losa_packed_attn_fwd at head dim d, None where it needs none."""
        need = self.workspace_bytes(d)
        return torch.empty(need, dtype=torch.uint8, device=self._data.device) if need else None


def losa_packed_plan(q_lens, k_lens, heads: int, kv_heads: int, dtype, causal: bool = False,
                     q_starts=None, k_starts=None, device="cuda") -> PackedPlan:
    """Plan of sequences of ``q_lens`` query tokens over ``k_lens`` keys (None: the same),
    one after another in q and k or at ``q_starts`` and ``k_starts``.  Lengths and starts
    are host integers.  Keep the plan for every layer and step with these lengths; caches
    that grow by a token take a new one each time (its copy to the device waits for it), and
    a captured graph keeps the lengths of its plan."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype}")
    q_lens = [int(x) for x in q_lens]
    k_lens = q_lens if k_lens is None else [int(x) for x in k_lens]
    n = len(q_lens)
    arrays = []
    for name, x, kind in (("q_starts", q_starts, ctypes.c_int64), ("q_lens", q_lens, ctypes.c_int32),
                          ("k_starts", k_starts, ctypes.c_int64), ("k_lens", k_lens, ctypes.c_int32)):
        if x is not None:
            x = [int(y) for y in x]
            if len(x) != n:
                raise ValueError(f"{name} has {len(x)} entries, q_lens {n}")
            if any(abs(y) > 2 ** 31 - 1 for y in x) and kind is ctypes.c_int32:
                raise ValueError(f"{name} holds a length beyond 32 bits")
            x = (kind * max(n, 1))(*x)
        arrays.append(x)
    info = _PackedInfo()

    def call(plan, room):
        _check(lib.losa_packed_plan(*arrays, n, _DTYPES[dtype], heads, kv_heads, int(causal), plan,
                                    room, ctypes.addressof(info)), "losa_packed_plan")

    call(None, 0)
    host = torch.empty(max(1, info.bytes // 8), dtype=torch.int64)
    call(host.data_ptr(), host.numel() * 8)
    return PackedPlan(info, host.to(device), dtype)


def _packed_view(t, name, device, dtype, shape):
    """losa_view of a [rows, heads, d] tensor of this shape whose rows of d are contiguous."""
    if (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype
            and t.shape == shape):
        sn, sh, sd = t.stride()
        if sd == 1:
            return _VIEW(t.data_ptr(), 0, sn, sh)
    _wrong(t, name, device, dtype, shape)


def losa_packed_attn_fwd(q, k, v, plan: PackedPlan, scale: float | None = None,
                         want_lse: bool = False, out=None, lse=None, workspace=None):
    """Attention over the plan's sequences: q [rows, heads, d], k and v [rows, kv_heads, d]
    (any strides, rows of d contiguous) -> o like q (and lse fp32 [heads, rows]).  Rows
    of ``out`` and ``lse`` that no sequence owns are left as they are."""
    if not isinstance(plan, PackedPlan):
        raise TypeError("plan must be a PackedPlan (losa_packed_plan)")
    for name, t in (("q", q), ("k", k)):
        if not isinstance(t, torch.Tensor) or t.dim() != 3:
            raise ValueError(f"{name} must be a [rows, heads, d] tensor")
    rows, _, d = q.shape
    k_rows = k.shape[0]
    dev, dt, heads = q.device, plan._dtype, plan._heads
    shape, shape_kv = (rows, heads, d), (k_rows, plan._kv_heads, d)
    if not q.is_cuda:
        raise ValueError(f"q must live on a GPU (got {dev})")
    if plan._data.device != dev:
        raise ValueError(f"the plan must live on {dev} (got {plan._data.device})")
    qv = _packed_view(q, "q", dev, dt, shape)
    kv = _packed_view(k, "k", dev, dt, shape_kv)
    vv = _packed_view(v, "v", dev, dt, shape_kv)
    if out is None:
        out = torch.empty(shape, dtype=dt, device=dev)
    ov = _packed_view(out, "out", dev, dt, shape)
    lse_at = None
    if want_lse:
        if lse is None:
            lse = torch.empty((heads, rows), dtype=torch.float32, device=dev)
        lse_at = _arg(lse, "lse", dev, dtype=torch.float32, shape=(heads, rows)).data_ptr()
    need = plan.workspace_bytes(d)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    ws_at, ws_bytes = None, 0
    if workspace is not None:
        _arg(workspace, "workspace", dev, nbytes=need)
        ws_at, ws_bytes = workspace.data_ptr(), workspace.nbytes
    st = _call(dev, lib.losa_packed_attn_fwd, qv, kv, vv, rows, k_rows, plan._info,
               plan._data.data_ptr(), d, 1.0 / math.sqrt(d) if scale is None else scale, ov, lse_at,
               rows, ws_at, ws_bytes)
    if st:
        _check(st, "losa_packed_attn_fwd")
    return (out, lse) if want_lse else out


# shorter aliases
calibrate_mass = losa_calibrate_mass
select_blocks = losa_select_blocks
select_blocks_topk = losa_select_blocks_topk
block_recall = losa_block_recall
sparse_attn_fwd = losa_sparse_attn_fwd
sparse_attn_fwd_noalloc = losa_sparse_attn_fwd_noalloc
construct = losa_construct
rope_table = losa_rope_table
rope = losa_rope
qk_norm_rope = losa_qk_norm_rope
packed_plan = losa_packed_plan
packed_attn_fwd = losa_packed_attn_fwd
