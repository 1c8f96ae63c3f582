"""ctypes binding of the operators around a key/value cache held in 4 bits: argument marshalling only.

``Rope`` rotates a block's queries and keys by their position in time, height and width; ``PackedCache`` holds keys and values
in 4 bits, attends to them, adds up the attention weight that every token receives and evicts the tokens that receive the
least.  Every method mirrors the C entry point of the same name in include/headcast.h.  Tensors are CUDA tensors on the
current device; work runs on the current torch stream.  There is no fallback: a call that fails raises.
"""
from __future__ import annotations

import ctypes as C
import operator
from typing import Optional, Sequence, Union

import torch

from . import binding
from .binding import HeadCastError

_raw_stream = torch._C._cuda_getCurrentRawStream  # torch.cuda.current_stream(device).cuda_stream without making a Stream object


class RopeConfig(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32),
                ("dim_t", C.c_int32), ("dim_h", C.c_int32), ("dim_w", C.c_int32), ("halves", C.c_int32), ("theta", C.c_double),
                ("scale_t", C.c_double), ("scale_h", C.c_double), ("scale_w", C.c_double)]


class PackedConfig(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("capacity", C.c_int32), ("softmax_scale", C.c_float)]


_lib = None


def load_library() -> C.CDLL:
    """libheadcast.so with the prototypes of these operators declared."""
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load_library()
    vp, i32, i64, i32p = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(C.c_int32)
    lib.headcast_rope_default_config.argtypes = [C.POINTER(RopeConfig)]
    lib.headcast_rope_default_config.restype = None
    lib.headcast_rope.argtypes = [C.POINTER(RopeConfig), vp, vp, i64, vp, vp, i64, i32, i64, vp, i32, vp]
    lib.headcast_rope_last_error.argtypes = []
    lib.headcast_rope_last_error.restype = C.c_char_p
    lib.headcast_packed_bytes.argtypes = [C.POINTER(PackedConfig)]
    lib.headcast_packed_bytes.restype = i64
    lib.headcast_packed_create.argtypes = [C.POINTER(PackedConfig), vp, i64, vp, C.POINTER(vp)]
    lib.headcast_packed_destroy.argtypes = [vp]
    lib.headcast_packed_lengths.argtypes = [vp, i32p]
    lib.headcast_packed_clear.argtypes = [vp]
    lib.headcast_packed_drop_last.argtypes = [vp, i32]
    lib.headcast_packed_weights_offset.argtypes = [vp, C.POINTER(i64)]
    lib.headcast_packed_weights_offset.restype = i64
    lib.headcast_packed_append.argtypes = [vp, vp, vp, i32, i64, vp]
    lib.headcast_packed_export.argtypes = [vp, i32, i32, vp, vp, vp]
    lib.headcast_packed_workspace_bytes.argtypes = [vp, i32]
    lib.headcast_packed_workspace_bytes.restype = i64
    lib.headcast_packed_attend.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp]
    lib.headcast_packed_observe.argtypes = [vp, vp, vp, i32, C.c_float, vp, i64, vp]
    lib.headcast_packed_evict_workspace_bytes.argtypes = [vp]
    lib.headcast_packed_evict_workspace_bytes.restype = i64
    lib.headcast_packed_evict.argtypes = [vp, vp, i32p, i32, i32, vp, i32, vp, i64, vp]
    lib.headcast_packed_check.argtypes = [vp, vp]
    lib.headcast_packed_last_error.argtypes = [vp]
    lib.headcast_packed_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def _refuse(t, name: str, shape, dtype, device: int, contiguous: bool) -> None:
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a torch tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise ValueError(f"{name}: dtype must be {dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape must be {tuple(shape)}, got {tuple(t.shape)}")
    if t.get_device() != device:
        raise ValueError(f"{name}: lives on {t.device}, it has to be on cuda:{device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    raise ValueError(f"{name}: the heads of a token must be contiguous, and tokens must not overlap")


def _tensor(t, name: str, shape, dtype, device: int) -> int:
    """Rejects whatever would make a kernel read or write outside the caller's buffer; returns the address."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous()):
        _refuse(t, name, shape, dtype, device, True)
    return t.data_ptr()


def _rows(t, name: str, shape, device: int):
    """(address, elements between tokens, 0 for contiguous) of a [tokens, heads, d] bf16 tensor whose tokens may lie apart, as in a
    slice of a fused projection."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.bfloat16 and t.shape == shape and t.get_device() == device):
        _refuse(t, name, shape, torch.bfloat16, device, False)
    if t.is_contiguous():
        return t.data_ptr(), 0
    n, h, d = shape
    stride = t.stride(0) if n > 1 else 0
    if t.stride(2) != 1 or (h > 1 and t.stride(1) != d) or (n > 1 and stride < h * d):
        _refuse(t, name, shape, torch.bfloat16, device, False)
    return t.data_ptr(), stride


def _int(value, name: str, bits: int = 32) -> int:
    """ctypes would cut a number that is too large down to one that is not."""
    value = operator.index(value)
    if not -(1 << (bits - 1)) <= value < 1 << (bits - 1):
        raise ValueError(f"{name}: {value} is out of range")
    return value


def _count(t) -> int:
    """Tokens of a [tokens, heads, d] tensor; -1, which no shape matches, for anything else."""
    return t.shape[0] if isinstance(t, torch.Tensor) and t.dim() == 3 else -1


class Rope:
    """Rotary positions over time, height and width (headcast_rope): ``dims`` are the rotated widths of the three axes."""

    def __init__(self, n_heads: int, head_dim: int, grid_h: int = 0, grid_w: int = 0, n_kv_heads: Optional[int] = None,
                 dims: Optional[Sequence[int]] = None, theta: float = 10000.0, scales: Sequence[float] = (1.0, 1.0, 1.0), halves: bool = False):
        self.lib = load_library()
        if dims is None:  # the usual split of a video transformer: a third each, the remainder with time
            dims = (head_dim - 4 * (head_dim // 6), 2 * (head_dim // 6), 2 * (head_dim // 6))
        cfg = RopeConfig()
        self.lib.headcast_rope_default_config(C.byref(cfg))
        cfg.n_heads, cfg.n_kv_heads = _int(n_heads, "n_heads"), _int(n_heads if n_kv_heads is None else n_kv_heads, "n_kv_heads")
        cfg.head_dim, cfg.grid_h, cfg.grid_w = _int(head_dim, "head_dim"), _int(grid_h, "grid_h"), _int(grid_w, "grid_w")
        cfg.halves, cfg.theta = bool(halves), theta
        cfg.dim_t, cfg.dim_h, cfg.dim_w = (_int(v, "dims") for v in dims)
        cfg.scale_t, cfg.scale_h, cfg.scale_w = scales
        self.cfg, self._cfg = cfg, C.byref(cfg)

    def apply(self, q, q_out, k=None, k_out=None, first_frame: int = 0, positions=None, inverse: bool = False) -> None:
        """q [n, n_heads, d] into q_out, k [n, n_kv_heads, d] into k_out; outputs contiguous, in place allowed.  positions: int32 [n, 3]."""
        cfg, n, device = self.cfg, _count(q), torch.cuda.current_device()
        if (k is None) != (k_out is None):
            raise ValueError("k and k_out belong together")
        shape = (n, cfg.n_heads, cfg.head_dim)
        q_ptr, q_stride = _rows(q, "q", shape, device)
        q_out_ptr = _tensor(q_out, "q_out", shape, torch.bfloat16, device)
        k_ptr, k_stride, k_out_ptr = None, 0, None
        if k is not None:
            shape = (n, cfg.n_kv_heads, cfg.head_dim)
            k_ptr, k_stride = _rows(k, "k", shape, device)
            k_out_ptr = _tensor(k_out, "k_out", shape, torch.bfloat16, device)
        pos = None if positions is None else _tensor(positions, "positions", (n, 3), torch.int32, device)
        rc = self.lib.headcast_rope(self._cfg, q_ptr, q_out_ptr, q_stride, k_ptr, k_out_ptr, k_stride, n, _int(first_frame, "first_frame", 64), pos, bool(inverse), _raw_stream(device))
        if rc != 0:
            raise HeadCastError(rc, self.lib.headcast_rope_last_error().decode())


class PackedCache:
    """One layer's key/value cache in 4 bits (wraps headcast_packed*).  The storage is a torch tensor of the current device and stream
    (keep the cache until work on other streams is done); every call takes its workspace from torch's allocator on the current
    stream, so calls and captured graphs share none."""

    def __init__(self, n_heads: int, head_dim: int, capacity: int, n_kv_heads: Optional[int] = None, softmax_scale: float = 0.0):
        self._ptr = C.c_void_p()
        self.lib = load_library()
        self.n_heads, self.head_dim, self.capacity = n_heads, head_dim, capacity
        self.n_kv_heads = n_heads if n_kv_heads is None else n_kv_heads
        self.cfg = PackedConfig(_int(n_heads, "n_heads"), _int(self.n_kv_heads, "n_kv_heads"), _int(head_dim, "head_dim"), _int(capacity, "capacity"), softmax_scale)
        if softmax_scale != 0.0 and self.cfg.softmax_scale == 0.0:  # ctypes cut it down to the zero that selects the default
            raise ValueError(f"softmax_scale: {softmax_scale} is out of range")
        size = self.lib.headcast_packed_bytes(C.byref(self.cfg))
        if size < 0:
            raise HeadCastError(size, "sizes out of range (1..64 heads, a divisor of them for keys and values, head_dim 64 or 128, capacity 1..2^23, "
                                      "softmax_scale 0 or 2^-40..2^40)")
        self._device = torch.cuda.current_device()
        self._where = torch.device("cuda", self._device)
        self.storage = torch.empty(size, dtype=torch.uint8, device=self._where)
        rc = self.lib.headcast_packed_create(C.byref(self.cfg), self.storage.data_ptr(), size, _raw_stream(self._device), C.byref(self._ptr))
        if rc != 0:
            self._ptr = C.c_void_p()
            raise HeadCastError(rc, "headcast_packed_create failed")
        self._lengths = (C.c_int32 * self.n_kv_heads)()
        self._like = self.storage[:0].view(torch.bfloat16)  # what exported tensors are made like
        stride = C.c_int64()
        at = self.lib.headcast_packed_weights_offset(self._ptr, C.byref(stride))
        self._weights = self.storage[at:at + 4 * stride.value * self.n_kv_heads].view(torch.float32).view(self.n_kv_heads, stride.value)

    def destroy(self) -> None:
        if self._ptr:
            self.lib.headcast_packed_destroy(self._ptr)
            self._ptr = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _raise(self, rc: int):
        raise HeadCastError(rc, self.lib.headcast_packed_last_error(self._ptr).decode())

    def _workspace(self, size: int):
        return self.storage.new_empty(max(size, 0))

    @property
    def weights(self):
        """The accumulated attention weights, float32 [n_kv_heads, longest head]: a view of the storage, rows of a head behind its last token are not its."""
        return self._weights[:, : max(self.lengths())]

    def lengths(self):
        """Tokens per key/value head."""
        rc = self.lib.headcast_packed_lengths(self._ptr, self._lengths)
        if rc != 0:
            self._raise(rc)
        return self._lengths[:]

    def clear(self) -> None:
        rc = self.lib.headcast_packed_clear(self._ptr)
        if rc != 0:
            self._raise(rc)

    def drop_last(self, n_tokens: int) -> None:
        rc = self.lib.headcast_packed_drop_last(self._ptr, _int(n_tokens, "n_tokens"))
        if rc != 0:
            self._raise(rc)

    def append(self, k, v) -> None:
        """k, v [n, n_kv_heads, d] bf16; tokens may lie apart (both alike)."""
        n, device = _count(k), self._device
        shape = (n, self.n_kv_heads, self.head_dim)
        k_ptr, stride = _rows(k, "k", shape, device)
        v_ptr, v_stride = _rows(v, "v", shape, device)
        if stride != v_stride:
            raise ValueError(f"k and v: tokens must lie equally far apart, got {k.stride(0)} and {v.stride(0)} elements")
        rc = self.lib.headcast_packed_append(self._ptr, k_ptr, v_ptr, n, stride, _raw_stream(device))
        if rc != 0:
            self._raise(rc)

    def export(self, first: int = 0, n_tokens: Optional[int] = None):
        """(K, V) bf16 [n_kv_heads, n, d]: the held values, zeros where a head has no token."""
        lengths, first = self.lengths(), _int(first, "first")
        n = max(0, max(lengths) - first) if n_tokens is None else _int(n_tokens, "n_tokens")
        if n < 0:
            raise ValueError(f"n_tokens must not be negative, got {n}")
        if first + n <= min(lengths):
            k = self._like.new_empty((self.n_kv_heads, n, self.head_dim))
            v = torch.empty_like(k)
        else:
            k = self._like.new_zeros((self.n_kv_heads, n, self.head_dim))
            v = torch.zeros_like(k)
        rc = self.lib.headcast_packed_export(self._ptr, first, n, k.data_ptr() if n else None, v.data_ptr() if n else None, _raw_stream(self._device))
        if rc != 0:
            self._raise(rc)
        return k, v

    def attend(self, q, out, lse=None) -> None:
        """q, out [n, n_heads, d] bf16; lse float32 [n_heads, n] or None."""
        lib, ptr, n, device = self.lib, self._ptr, _count(q), self._device
        shape = (n, self.n_heads, self.head_dim)
        q_ptr = _tensor(q, "q", shape, torch.bfloat16, device)
        out_ptr = _tensor(out, "out", shape, torch.bfloat16, device)
        lse_ptr = None if lse is None else _tensor(lse, "lse", (self.n_heads, n), torch.float32, device)
        size = lib.headcast_packed_workspace_bytes(ptr, n)
        ws = self._workspace(size)
        rc = lib.headcast_packed_attend(ptr, q_ptr, out_ptr, lse_ptr, n, ws.data_ptr(), size, _raw_stream(device))
        if rc != 0:
            self._raise(rc)

    def observe(self, q, lse, decay: float = 1.0) -> None:
        """weights = decay * weights + the attention weight that every token receives from the queries, summed; lse as attend returned it."""
        lib, ptr, n, device = self.lib, self._ptr, _count(q), self._device
        q_ptr = _tensor(q, "q", (n, self.n_heads, self.head_dim), torch.bfloat16, device)
        lse_ptr = _tensor(lse, "lse", (self.n_heads, n), torch.float32, device)
        size = lib.headcast_packed_workspace_bytes(ptr, n)
        ws = self._workspace(size)
        rc = lib.headcast_packed_observe(ptr, q_ptr, lse_ptr, n, decay, ws.data_ptr(), size, _raw_stream(device))
        if rc != 0:
            self._raise(rc)

    def evict_into(self, other: "PackedCache", keep: Union[int, Sequence[int]], n_first: int = 0, n_recent: int = 0, index=None) -> None:
        """Moves into ``other`` (its tokens are replaced), per head and in order, the first n_first and newest n_recent tokens and the
        largest weights besides, ``keep`` tokens in all (one number, or one per key/value head; a shorter head moves whole).  index:
        int32 [n_kv_heads, >= longest result] or None, receives the places that the tokens had."""
        lib, kv, device = self.lib, self.n_kv_heads, self._device
        keep = [_int(keep, "keep")] * kv if hasattr(keep, "__index__") else [_int(v, "keep") for v in keep]
        if len(keep) != kv:
            raise ValueError(f"keep: expected {kv} entries, got {len(keep)}")
        if not isinstance(other, PackedCache) or not other._ptr:
            raise ValueError("other: expected a PackedCache")
        ptr, width, ws, size = None, 0, None, 0
        if index is not None:
            width = _int(index.shape[1], "index") if isinstance(index, torch.Tensor) and index.dim() == 2 else -1
            ptr = _tensor(index, "index", (kv, width), torch.int32, device)
        else:
            size = lib.headcast_packed_evict_workspace_bytes(self._ptr)
            ws = self._workspace(size)
        rc = lib.headcast_packed_evict(self._ptr, other._ptr, (C.c_int32 * kv)(*keep), _int(n_first, "n_first"), _int(n_recent, "n_recent"), ptr, width, None if ws is None else ws.data_ptr(), size,
                                       _raw_stream(device))
        if rc != 0:
            self._raise(rc)

    def check(self) -> None:
        """Synchronises the current stream; raises if a kernel of this cache gave up on a bounded wait."""
        rc = self.lib.headcast_packed_check(self._ptr, _raw_stream(self._device))
        if rc != 0:
            self._raise(rc)
