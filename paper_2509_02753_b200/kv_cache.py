"""Thin ctypes binding of the C ABI in ``include/moe_kv.h``: the operators around a paged cache of keys and values in 4 bits.

Argument marshalling only, like ``binding.py`` (whose ``MoEError`` it raises): every step runs in the CUDA kernels of
``liblexi_moe.so``, there is no fallback.  The calls of a step go through the native module ``_kv_native`` (3 to 6 us a
call on the host instead of 17 to 35 through ctypes), the others through ctypes.  A ``KVPlan`` is made for one shape of attention; the cache itself, the block
tables and the free list are the caller's tensors:

    plan = KVPlan(n_heads=32, n_kv_heads=8, head_dim=128, page_size=64, dtype=torch.bfloat16, max_requests=16, max_tokens=8192)
    cache = plan.new_cache(n_pages)                                   # one per layer
    turns = rope_table(128, 32768, base=10000.0)                      # cos, sin
    kv_len, cu, position, slot, taken = plan.tables(ctx_len, new_len, free_pages, block_table, n_tokens)
    q = plan.append(q, k, v, slot, cache, positions=position, turns=turns)      # turned queries; keys and values stored
    o = plan.attention(q, cu, kv_len, block_table, cache, max_new=1)

``decoder.py`` runs them together with the MoE layer.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding as B
from .binding import MoEError  # noqa: F401  (what the calls below raise)

STATUS_TIMEOUT, STATUS_BAD_INDEX, STATUS_NO_PAGES, STATUS_NONFINITE = 1, 2, 4, 8
LAYOUTS = {"half": 0, "pairs": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "parts": 3, "bands": 4}

EXPORTS = (
    "moe_kv_plan_create", "moe_kv_plan_destroy", "moe_kv_plan_workspace_bytes", "moe_kv_plan_launch_count", "moe_kv_page_bytes",
    "moe_kv_device_status", "moe_kv_tables", "moe_rope_table", "moe_rope", "moe_kv_append", "moe_kv_read", "moe_kv_attention",
)


class moe_kv_config_t(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_heads", "n_kv_heads", "head_dim", "page_size", "max_requests", "max_tokens", "dtype")]


class moe_kv_rows_t(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class moe_rope_config_t(ctypes.Structure):
    _fields_ = [("rope_dim", ctypes.c_int32), ("scaling", ctypes.c_int32)] + \
        [(n, ctypes.c_double) for n in ("base", "factor", "low", "high", "original_context", "magnitude")]


_lib = None
_native = None


def load_library() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    lib = B.load_library()
    vp, i32, i64, u64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float
    P = ctypes.POINTER
    rows = P(moe_kv_rows_t)
    lib.moe_kv_plan_create.argtypes = [P(moe_kv_config_t), P(vp)]
    lib.moe_kv_plan_destroy.argtypes = [vp]
    lib.moe_kv_plan_workspace_bytes.argtypes = [vp]
    lib.moe_kv_plan_launch_count.argtypes = [vp]
    lib.moe_kv_page_bytes.argtypes = [P(moe_kv_config_t)]
    lib.moe_kv_device_status.argtypes = [vp, P(i32), vp]
    lib.moe_rope_table.argtypes = [P(moe_rope_config_t), i32, vp, vp]
    lib.moe_kv_tables.argtypes = [vp, vp, vp, i32, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.moe_rope.argtypes = [vp, rows, i32, i32, vp, vp, i32, i32, i32, i32, vp, i64, i64, vp]
    lib.moe_kv_append.argtypes = [vp, rows, rows, rows, i32, vp, vp, i32, i32, i32, vp, f32, f32, vp, vp, i32, vp]
    lib.moe_kv_read.argtypes = [vp, vp, i32, vp, i32, f32, f32, vp, vp, vp]
    lib.moe_kv_attention.argtypes = [vp, rows, i32, vp, vp, i32, i32, vp, i32, vp, i32, f32, f32, f32, i32, i32, vp, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = u64 if name in ("moe_kv_plan_workspace_bytes", "moe_kv_plan_launch_count", "moe_kv_page_bytes") else ctypes.c_int
    _lib = lib
    return lib


def load_native():
    """The module ``_kv_native`` (built by ``paper_2509_02753_b200.build``); raises if absent."""
    global _native
    if _native is None:
        load_library()
        try:
            from . import _kv_native
        except ImportError as e:
            raise MoEError(f"native binding not built ({e}); run __graft_entry__.build()", -5)
        _native = _kv_native
    return _native


def rope_table(rope_dim: int, n_positions: int, *, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, low: float = 1.0,
               high: Optional[float] = None, original_context: float = 0.0, magnitude: float = 0.0, device="cuda", stream=None) -> torch.Tensor:
    """cos and sin of every position and pair, [n_positions, rope_dim/2, 2] fp32 (``moe_rope_table``).  The tensor belongs to `stream`."""
    with torch.cuda.stream(stream):          # None: the current one
        out = torch.empty((n_positions, rope_dim // 2, 2), dtype=torch.float32, device=device)
    if high is None:
        high = 4.0 if scaling == "bands" else 32.0
    cfg = moe_rope_config_t(rope_dim, SCALINGS[scaling], base, factor, low, high, original_context, magnitude)
    with torch.cuda.device(out.device):
        B._check("moe_rope_table", load_library().moe_rope_table(ctypes.byref(cfg), n_positions, out.data_ptr(), B._stream(stream)))
    return out


class KVPlan:
    """Owns one plan handle (workspace and status word) for one shape of attention; a wrapper over the C entry points."""

    def __init__(self, *, n_heads: int, n_kv_heads: int, head_dim: int, page_size: int, dtype: torch.dtype, max_requests: int, max_tokens: int):
        self.n_heads, self.n_kv_heads, self.head_dim, self.page_size, self.dtype = n_heads, n_kv_heads, head_dim, page_size, dtype
        self.cfg = moe_kv_config_t(n_heads, n_kv_heads, head_dim, page_size, max_requests, max_tokens, B._dtype_code(dtype))
        self._lib, self._native = load_library(), load_native()
        self.default_scale = 1.0 / math.sqrt(head_dim)
        self._plan = None
        self.handle = None
        out = ctypes.c_void_p()
        B._check("moe_kv_plan_create", self._lib.moe_kv_plan_create(ctypes.byref(self.cfg), ctypes.byref(out)))
        self.handle, self.device = out.value, torch.cuda.current_device()
        self._plan = (self.handle, n_heads, n_kv_heads, head_dim, self.page_bytes, self.cfg.dtype, self.device)

    def close(self):
        self._plan = None
        if getattr(self, "handle", None):
            B._check("moe_kv_plan_destroy", self._lib.moe_kv_plan_destroy(self.handle))          # on the plan's device
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    @property
    def page_bytes(self) -> int:
        return int(self._lib.moe_kv_page_bytes(ctypes.byref(self.cfg)))

    @property
    def workspace_bytes(self) -> int:
        return int(self._lib.moe_kv_plan_workspace_bytes(self.handle))

    @property
    def launch_count(self) -> int:
        return int(self._lib.moe_kv_plan_launch_count(self.handle))

    def device_status(self, stream=None):
        """(status, MOE_KV_STATUS bits) since the last read; synchronises.  Behind the plan's calls on `stream`, by default
        the current one of the plan's device, whichever device is current."""
        bits = ctypes.c_int32()
        with torch.cuda.device(self.device):
            status = int(self._lib.moe_kv_device_status(self.handle, ctypes.byref(bits), B._stream(stream)))
        if status == -5:
            raise MoEError("moe_kv_device_status", status)
        return status, int(bits.value)

    def new_cache(self, n_pages: int, device=None) -> torch.Tensor:
        """An empty cache of one layer, on the plan's device: [n_pages, n_kv_heads, page_size/16, block bytes] uint8."""
        blocks = self.page_size // 16
        return torch.zeros((n_pages, self.n_kv_heads, blocks, self.page_bytes // (self.n_kv_heads * blocks)), dtype=torch.uint8,
                           device=torch.device("cuda", self.device) if device is None else device)

    def _call(self, what: str, f, *args, stream=None):
        """One native call on the current stream, or on `stream` (what it allocates then belongs to that stream)."""
        if stream is not None and stream != torch.cuda.current_stream(self.device):
            with torch.cuda.stream(stream):
                got = f(*args)
        else:
            got = f(*args)
        if got[0] != 0:
            raise MoEError(what, got[0])
        return got

    def tables(self, ctx_len: torch.Tensor, new_len: torch.Tensor, free_pages: torch.Tensor, block_table: torch.Tensor, n_tokens: int, stream=None):
        """(kv_len, cu_new, positions, slots, pages_taken); block_table gets the fresh pages (``moe_kv_tables``)."""
        return self._call("moe_kv_tables", self._native.tables, self._plan, ctx_len, new_len, free_pages, block_table, n_tokens, stream=stream)[1:]

    def rope(self, x: torch.Tensor, positions: torch.Tensor, turns: torch.Tensor, *, layout: str = "half", inverse: bool = False,
             out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x [tokens, heads, head_dim] turned by its tokens' positions; inverse=True turns back, which is the gradient (``moe_rope``)."""
        return self._call("moe_rope", self._native.rope, self._plan, x, positions, turns, LAYOUTS[layout], inverse, out, stream=stream)[1]

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: torch.Tensor, *,
               positions: Optional[torch.Tensor] = None, turns: Optional[torch.Tensor] = None, layout: str = "half", k_scale: float = 1.0,
               v_scale: float = 1.0, q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """Stores keys (turned) and values at the slots and returns the turned queries (``moe_kv_append``)."""
        got = self._call("moe_kv_append", self._native.append, self._plan, q, k, v, slots, cache, positions, turns, LAYOUTS[layout], k_scale, v_scale,
                         q_out, stream=stream)
        return got[1] if q is not None else None

    def read(self, cache: torch.Tensor, slots: torch.Tensor, *, k_scale: float = 1.0, v_scale: float = 1.0, stream=None):
        """(keys, values) [tokens, n_kv_heads, head_dim] at the slots, as the numbers they stand for (``moe_kv_read``)."""
        return self._call("moe_kv_read", self._native.read, self._plan, cache, slots, k_scale, v_scale, stream=stream)[1:]

    def attention(self, q: torch.Tensor, cu_new: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, cache: torch.Tensor, *,
                  max_new: int = 0, window: int = 0, sinks: int = 0, softmax_scale: Optional[float] = None, k_scale: float = 1.0, v_scale: float = 1.0,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the new tokens' queries [tokens, n_heads, head_dim] over their requests' caches (``moe_kv_attention``).
        max_new: the largest number of new tokens of a request (0 = unknown); it chooses kernels, not results."""
        return self._call("moe_kv_attention", self._native.attention, self._plan, q, cu_new, kv_len, block_table, cache, max_new, window, sinks,
                          self.default_scale if softmax_scale is None else softmax_scale, k_scale, v_scale, out, stream=stream)[1]
