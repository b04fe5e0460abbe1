"""Thin ctypes binding of the C ABI in ``include/moe_kv.h``: the operators around a paged cache of keys and values in 4 bits.

Argument marshalling only, like ``binding.py`` (whose ``MoEError`` it raises): every step runs in the CUDA kernels of
``liblexi_moe.so``, there is no fallback.  A ``KVPlan`` is made for one shape of attention; the cache itself, the block
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
    lib.moe_kv_tables.argtypes = [vp, vp, vp, i32, vp, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.moe_rope_table.argtypes = [P(moe_rope_config_t), i32, vp, vp]
    lib.moe_rope.argtypes = [vp, rows, i32, i32, vp, vp, i32, i32, i32, i32, vp, i64, i64, vp]
    lib.moe_kv_append.argtypes = [vp, rows, rows, rows, i32, vp, vp, i32, i32, i32, vp, f32, f32, vp, vp, i32, vp]
    lib.moe_kv_read.argtypes = [vp, vp, i32, vp, i32, f32, f32, vp, vp, vp]
    lib.moe_kv_attention.argtypes = [vp, rows, i32, vp, vp, i32, i32, vp, i32, vp, i32, f32, f32, f32, i32, i32, vp, vp]
    for name in EXPORTS:
        getattr(lib, name).restype = u64 if name in ("moe_kv_plan_workspace_bytes", "moe_kv_plan_launch_count", "moe_kv_page_bytes") else ctypes.c_int
    _lib = lib
    return lib


def _rows(x: torch.Tensor) -> moe_kv_rows_t:
    ts, hs, one = x.stride()
    assert one == 1 or x.shape[2] == 1, "the dimensions of a head must be neighbours"
    return moe_kv_rows_t(x.data_ptr(), ts, hs)


def rope_table(rope_dim: int, n_positions: int, *, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, low: float = 1.0,
               high: Optional[float] = None, original_context: float = 0.0, magnitude: float = 0.0, device="cuda", stream=None) -> torch.Tensor:
    """cos and sin of every position and pair, [n_positions, rope_dim/2, 2] fp32 (``moe_rope_table``)."""
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
        self._lib = load_library()
        out = ctypes.c_void_p()
        self.handle = None
        B._check("moe_kv_plan_create", self._lib.moe_kv_plan_create(ctypes.byref(self.cfg), ctypes.byref(out)))
        self.handle = out.value

    def close(self):
        if getattr(self, "handle", None):
            B._check("moe_kv_plan_destroy", self._lib.moe_kv_plan_destroy(self.handle))
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
        """(status, MOE_KV_STATUS bits) since the last read; synchronises."""
        bits = ctypes.c_int32()
        status = int(self._lib.moe_kv_device_status(self.handle, ctypes.byref(bits), B._stream(stream)))
        if status == -5:
            raise MoEError("moe_kv_device_status", status)
        return status, int(bits.value)

    def new_cache(self, n_pages: int, device="cuda") -> torch.Tensor:
        """An empty cache of one layer: [n_pages, n_kv_heads, page_size/16, block bytes] uint8."""
        blocks = self.page_size // 16
        return torch.zeros((n_pages, self.n_kv_heads, blocks, self.page_bytes // (self.n_kv_heads * blocks)), dtype=torch.uint8, device=device)

    def _pages(self, cache: torch.Tensor) -> int:
        assert cache.is_cuda and cache.is_contiguous() and cache.dtype == torch.uint8
        n = cache.shape[0]
        assert cache.numel() == n * self.page_bytes, "cache of another shape"
        return n

    def _heads(self, x: torch.Tensor, heads: int, what: str) -> moe_kv_rows_t:
        assert x.is_cuda and x.dtype == self.dtype and x.dim() == 3 and x.shape[1] == heads and x.shape[2] == self.head_dim, what
        return _rows(x)

    def tables(self, ctx_len: torch.Tensor, new_len: torch.Tensor, free_pages: torch.Tensor, block_table: torch.Tensor, n_tokens: int, stream=None):
        """(kv_len, cu_new, positions, slots, pages_taken); block_table gets the fresh pages (``moe_kv_tables``)."""
        n, dev, i32 = ctx_len.shape[0], ctx_len.device, torch.int32
        assert ctx_len.is_cuda and ctx_len.dtype == new_len.dtype == free_pages.dtype == block_table.dtype == i32
        assert new_len.shape[0] == n and block_table.shape[0] == n
        assert ctx_len.is_contiguous() and new_len.is_contiguous() and free_pages.is_contiguous() and block_table.is_contiguous()
        kv_len = torch.empty((n,), dtype=i32, device=dev)
        cu = torch.empty((n + 1,), dtype=i32, device=dev)
        position = torch.empty((n_tokens,), dtype=i32, device=dev)
        slot = torch.empty((n_tokens,), dtype=torch.int64, device=dev)
        taken = torch.empty((1,), dtype=i32, device=dev)
        B._check("moe_kv_tables", self._lib.moe_kv_tables(
            self.handle, ctx_len.data_ptr(), new_len.data_ptr(), n, free_pages.data_ptr(), free_pages.numel(), block_table.data_ptr(),
            block_table.shape[1], n_tokens, kv_len.data_ptr(), cu.data_ptr(), position.data_ptr(), slot.data_ptr(), taken.data_ptr(), B._stream(stream)))
        return kv_len, cu, position, slot, taken

    def _turns(self, turns, positions, n):
        if turns is None:
            return None, None, 0, 0
        assert turns.is_cuda and turns.dtype == torch.float32 and turns.is_contiguous() and turns.dim() == 3 and turns.shape[2] == 2
        assert positions is not None and positions.is_cuda and positions.dtype == torch.int32 and positions.is_contiguous() and positions.shape[0] == n
        return positions.data_ptr(), turns.data_ptr(), turns.shape[0], 2 * turns.shape[1]

    def rope(self, x: torch.Tensor, positions: torch.Tensor, turns: torch.Tensor, *, layout: str = "half", inverse: bool = False,
             out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """x [tokens, heads, head_dim] turned by its tokens' positions; inverse=True turns back, which is the gradient (``moe_rope``)."""
        rows = self._heads(x, x.shape[1], "x")
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        assert out.shape == x.shape and out.dtype == x.dtype and (out.stride(2) == 1 or self.head_dim == 1)
        p, t, n_pos, rot = self._turns(turns, positions, x.shape[0])
        B._check("moe_rope", self._lib.moe_rope(self.handle, ctypes.byref(rows), x.shape[0], x.shape[1], p, t, n_pos, rot, LAYOUTS[layout], int(inverse),
                                                out.data_ptr(), out.stride(0), out.stride(1), B._stream(stream)))
        return out

    def append(self, q: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache: torch.Tensor, *,
               positions: Optional[torch.Tensor] = None, turns: Optional[torch.Tensor] = None, layout: str = "half", k_scale: float = 1.0,
               v_scale: float = 1.0, q_out: Optional[torch.Tensor] = None, stream=None) -> Optional[torch.Tensor]:
        """Stores keys (turned) and values at the slots and returns the turned queries (``moe_kv_append``)."""
        n = k.shape[0]
        assert v.shape[0] == n and slots.is_cuda and slots.dtype == torch.int64 and slots.is_contiguous() and slots.shape[0] == n
        kr, vr = self._heads(k, self.n_kv_heads, "k"), self._heads(v, self.n_kv_heads, "v")
        qr = None
        if q is not None:
            assert q.shape[0] == n
            qr = ctypes.byref(self._heads(q, self.n_heads, "q"))
            if q_out is None:
                q_out = torch.empty((n, self.n_heads, self.head_dim), dtype=self.dtype, device=k.device)
            assert q_out.is_contiguous() and q_out.shape == q.shape and q_out.dtype == self.dtype
        p, t, n_pos, rot = self._turns(turns, positions, n)
        B._check("moe_kv_append", self._lib.moe_kv_append(
            self.handle, qr, ctypes.byref(kr), ctypes.byref(vr), n, p, t, n_pos, rot, LAYOUTS[layout], slots.data_ptr(), k_scale, v_scale,
            None if q is None else q_out.data_ptr(), cache.data_ptr(), self._pages(cache), B._stream(stream)))
        return q_out if q is not None else None

    def read(self, cache: torch.Tensor, slots: torch.Tensor, *, k_scale: float = 1.0, v_scale: float = 1.0, stream=None):
        """(keys, values) [tokens, n_kv_heads, head_dim] at the slots, as the numbers they stand for (``moe_kv_read``)."""
        assert slots.is_cuda and slots.dtype == torch.int64 and slots.is_contiguous()
        n = slots.shape[0]
        k = torch.empty((n, self.n_kv_heads, self.head_dim), dtype=self.dtype, device=cache.device)
        v = torch.empty_like(k)
        B._check("moe_kv_read", self._lib.moe_kv_read(self.handle, cache.data_ptr(), self._pages(cache), slots.data_ptr(), n, k_scale, v_scale,
                                                      k.data_ptr(), v.data_ptr(), B._stream(stream)))
        return k, v

    def attention(self, q: torch.Tensor, cu_new: torch.Tensor, kv_len: torch.Tensor, block_table: torch.Tensor, cache: torch.Tensor, *,
                  max_new: int = 0, window: int = 0, sinks: int = 0, softmax_scale: Optional[float] = None, k_scale: float = 1.0, v_scale: float = 1.0,
                  out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """Attention of the new tokens' queries [tokens, n_heads, head_dim] over their requests' caches (``moe_kv_attention``).
        max_new: the largest number of new tokens of a request (0 = unknown); it chooses kernels, not results."""
        rows = self._heads(q, self.n_heads, "q")
        n = kv_len.shape[0]
        assert cu_new.dtype == kv_len.dtype == block_table.dtype == torch.int32 and cu_new.shape[0] == n + 1 and block_table.shape[0] == n
        assert cu_new.is_cuda and kv_len.is_cuda and block_table.is_cuda and cu_new.is_contiguous() and kv_len.is_contiguous() and block_table.is_contiguous()
        if out is None:
            out = torch.empty((q.shape[0], self.n_heads, self.head_dim), dtype=self.dtype, device=q.device)
        assert out.is_contiguous() and out.shape == q.shape and out.dtype == self.dtype
        if softmax_scale is None:
            softmax_scale = 1.0 / math.sqrt(self.head_dim)
        B._check("moe_kv_attention", self._lib.moe_kv_attention(
            self.handle, ctypes.byref(rows), q.shape[0], cu_new.data_ptr(), kv_len.data_ptr(), n, max_new, block_table.data_ptr(), block_table.shape[1],
            cache.data_ptr(), self._pages(cache), softmax_scale, k_scale, v_scale, window, sinks, out.data_ptr(), B._stream(stream)))
        return out
