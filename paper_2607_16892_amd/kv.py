"""Binding of the paged-cache entry points (block tables, store, attention;
include/dro.h).  Argument checks and marshalling only."""
from __future__ import annotations

import ctypes as ct
import math
from dataclasses import dataclass
from typing import Optional

import torch

from . import _native
from .api import Context, _need_dev, _out, _ptr, _stream

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}


def _share(stream, device, *tensors):
    """Tensors that a call uses on another stream than the current one stay allocated
    until that stream has passed the call."""
    if stream is not None and stream != torch.cuda.current_stream(device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


def _need_rows(t, name, device, heads, dim):
    """A [T, heads, dim] tensor whose rows of dim components are contiguous."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError(f"{name} must be torch.bfloat16 or torch.float16, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != dim:
        raise ValueError(f"{name} must have shape (T, {heads}, {dim}), got {tuple(t.shape)}")
    if dim > 1 and t.stride(2) != 1:
        raise ValueError(f"the components of {name} must be contiguous")


@dataclass
class BlockPool:
    """The blocks of a cache and who holds them (field meanings as in dro_kv_pool)."""
    block: int                 # tokens a block
    table: torch.Tensor        # int32 [R, max_blocks], rows may be strided
    held: torch.Tensor         # int32 [R] blocks held
    free_list: torch.Tensor    # int32 [num_blocks] stack of free blocks
    free: torch.Tensor         # int32 [1] blocks free

    @classmethod
    def empty(cls, R, max_blocks, num_blocks, block=16, device="cuda"):
        """A pool with every block free; block 0 is handed out first."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(block=block, table=torch.full((R, max_blocks), -1, **i32),
                   held=torch.zeros(R, **i32),
                   free_list=torch.arange(num_blocks - 1, -1, -1, **i32),
                   free=torch.full((1,), num_blocks, **i32))

    @property
    def R(self) -> int:
        return int(self.table.shape[0])

    @property
    def device(self):
        return self.table.device

    def take(self, step: dict) -> dict:
        """Makes the blocks held and free after `step` (of kv_block_tables) the pool's."""
        self.held, self.free = step["held"], step["free"]
        return step

    def struct(self) -> _native.KvPoolStruct:
        t = self.table
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError("table must be a CUDA tensor")
        if t.dtype != torch.int32 or t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
            raise ValueError("table must be an int32 [R, max_blocks] tensor with contiguous rows")
        _need_dev(self.held, torch.int32, "held", t.device)
        _need_dev(self.free_list, torch.int32, "free_list", t.device)
        _need_dev(self.free, torch.int32, "free", t.device)
        if self.held.numel() != t.shape[0] or self.free.numel() != 1:
            raise ValueError("held must hold R entries and free one")
        s = _native.KvPoolStruct()
        s.R, s.max_blocks = int(t.shape[0]), int(t.shape[1])
        s.block, s.num_blocks = self.block, self.free_list.numel()
        s.table_stride = t.stride(0) if t.shape[0] > 1 else t.shape[1]
        s.table, s.free_list = t.data_ptr(), self.free_list.data_ptr()
        s.held, s.free_count = self.held.data_ptr(), self.free.data_ptr()
        return s


@dataclass
class KvCache:
    """One layer's cache (field meanings as in dro_kv_cache): k and v are
    [num_blocks, block, heads, dim] tensors, strided as they like except for the
    contiguous components, in torch.bfloat16, torch.float16 or, with scales,
    torch.float8_e4m3fn."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None   # float32 [heads]
    v_scale: Optional[torch.Tensor] = None

    @classmethod
    def empty(cls, num_blocks, block, heads, dim, dtype=torch.bfloat16, device="cuda",
              k_scale=None, v_scale=None):
        """A zeroed cache whose blocks hold the tokens of a head next to one another."""
        k, v = (torch.zeros((num_blocks, heads, block, dim), dtype=dtype, device=device)
                .permute(0, 2, 1, 3) for _ in range(2))
        if dtype == torch.float8_e4m3fn:
            one = torch.ones(heads, dtype=torch.float32, device=device)
            k_scale = one if k_scale is None else k_scale
            v_scale = one if v_scale is None else v_scale
        return cls(k, v, k_scale, v_scale)

    @property
    def device(self):
        return self.k.device

    @property
    def heads(self) -> int:
        return int(self.k.shape[2])

    @property
    def dim(self) -> int:
        return int(self.k.shape[3])

    def struct(self) -> _native.KvCacheStruct:
        s = _native.KvCacheStruct()
        for name, t in (("k", self.k), ("v", self.v)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"cache {name} must be a CUDA tensor")
            if t.dtype not in DTYPES:
                raise TypeError(f"cache {name} must be bfloat16, float16 or float8_e4m3fn, got {t.dtype}")
            if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
                raise ValueError(f"cache {name} must be [num_blocks, block, heads, dim] with "
                                 "contiguous components")
        if self.v.shape != self.k.shape or self.v.dtype != self.k.dtype or self.v.device != self.k.device:
            raise ValueError("cache k and v differ in shape, type or device")
        for name, t in (("k_scale", self.k_scale), ("v_scale", self.v_scale)):
            if t is not None:
                _need_dev(t, torch.float32, name, self.k.device)
                if t.numel() != self.heads:
                    raise ValueError(f"{name} must hold one scale per head")
        s.dtype = DTYPES[self.k.dtype]
        s.num_blocks, s.block, s.heads, s.dim = self.k.shape
        s.k, s.v = self.k.data_ptr(), self.v.data_ptr()
        s.k_block, s.k_token, s.k_head = self.k.stride()[:3]
        s.v_block, s.v_token, s.v_head = self.v.stride()[:3]
        s.k_scale = None if self.k_scale is None else self.k_scale.data_ptr()
        s.v_scale = None if self.v_scale is None else self.v_scale.data_ptr()
        return s


def kv_block_tables(ctx: Context, pool: BlockPool, length: torch.Tensor, add: torch.Tensor,
                    tokens: int, reserve: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                    stream=None) -> dict:
    """Blocks and slots of one step's `tokens` new tokens (see kv_block_tables in dro.h): the
    pool's table and free_list change in place; held and free after the step are outputs, which
    pool.take makes the pool's."""
    dev, R, T = pool.device, pool.R, int(tokens)
    ps = pool.struct()
    for name, t in (("length", length), ("add", add), ("reserve", reserve)):
        if t is not None:
            _need_dev(t, torch.int32, name, dev)
            if t.numel() != R:
                raise ValueError(f"{name} must hold R entries")
    if T < 0:
        raise ValueError("tokens must not be negative")
    out = out or {}
    with torch.cuda.stream(stream):
        o = dict(held=_out(out.get("held"), (R,), torch.int32, dev, "held"),
                 free=_out(out.get("free"), (1,), torch.int32, dev, "free"),
                 context=_out(out.get("context"), (R,), torch.int32, dev, "context"),
                 start=_out(out.get("start"), (R + 1,), torch.int32, dev, "start"),
                 slot=_out(out.get("slot"), (T,), torch.int64, dev, "slot"),
                 pos=_out(out.get("pos"), (T,), torch.int32, dev, "pos"),
                 granted=_out(out.get("granted"), (R,), torch.uint8, dev, "granted"))
    rc = ctx._lib.kv_block_tables(ctx.handle, ct.byref(ps), _ptr(length), _ptr(add), _ptr(reserve), T,
                                  _ptr(o["held"]), _ptr(o["free"]), _ptr(o["context"]),
                                  _ptr(o["start"]), _ptr(o["slot"]), _ptr(o["pos"]),
                                  _ptr(o["granted"]), _stream(stream, dev))
    ctx.check(rc, "kv_block_tables")
    _share(stream, dev, pool.table, pool.held, pool.free_list, pool.free, length, add, reserve,
           *o.values())
    return o


def kv_store(ctx: Context, cache: KvCache, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor,
             stream=None) -> None:
    """The keys and values [T, heads, dim] of T tokens into their slots of the cache (see
    kv_store in dro.h); the tokens and heads may be strided (views of a joint projection)."""
    dev = cache.device
    cs = cache.struct()
    _need_rows(k, "k", dev, cache.heads, cache.dim)
    _need_rows(v, "v", dev, cache.heads, cache.dim)
    if v.dtype != k.dtype or v.shape != k.shape:
        raise ValueError("k and v differ in shape or type")
    _need_dev(slot, torch.int64, "slot", dev)
    T = int(k.shape[0])
    if slot.numel() != T:
        raise ValueError("slot must hold T entries")
    rc = ctx._lib.kv_store(ctx.handle, ct.byref(cs), DTYPES[k.dtype], T, _ptr(k), k.stride(0),
                           k.stride(1), _ptr(v), v.stride(0), v.stride(1), _ptr(slot),
                           _stream(stream, dev))
    ctx.check(rc, "kv_store")
    _share(stream, dev, cache.k, cache.v, cache.k_scale, cache.v_scale, k, v, slot)


def kv_attention(ctx: Context, cache: KvCache, q: torch.Tensor, table: torch.Tensor,
                 start: torch.Tensor, context: torch.Tensor, max_new: int, scale=None,
                 softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                 prefix: Optional[torch.Tensor] = None, out=None, lse=None, want_lse: bool = True,
                 stream=None) -> dict:
    """Attention of the rows q [T, Hq, dim] over the cache (see kv_attention in dro.h).  `table`
    is a BlockPool's, `start` and `context` come from kv_block_tables; max_new bounds the rows of
    one request.  scale defaults to dim ** -0.5."""
    dev = cache.device
    cs = cache.struct()
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise TypeError("q must be a [T, Hq, dim] CUDA tensor")
    T, Hq = int(q.shape[0]), int(q.shape[1])
    _need_rows(q, "q", dev, Hq, cache.dim)
    if not isinstance(table, torch.Tensor) or not table.is_cuda or table.device != dev:
        raise TypeError(f"table must be a CUDA tensor on {dev}")
    if table.dtype != torch.int32 or table.dim() != 2 or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be an int32 [R, max_blocks] tensor with contiguous rows")
    R = int(table.shape[0])
    for name, t, n in (("start", start, R + 1), ("context", context, R), ("prefix", prefix, R)):
        if t is not None:
            _need_dev(t, torch.int32, name, dev)
            if t.numel() != n:
                raise ValueError(f"{name} must hold {n} entries")
    if slopes is not None:
        _need_dev(slopes, torch.float32, "slopes", dev)
        if slopes.numel() != Hq:
            raise ValueError("slopes must hold one slope per query head")
    with torch.cuda.stream(stream):
        if out is None:
            out = torch.empty((T, Hq, cache.dim), dtype=q.dtype, device=dev)
        if want_lse or lse is not None:
            lse = _out(lse, (T, Hq), torch.float32, dev, "lse")
    _need_rows(out, "out", dev, Hq, cache.dim)
    if out.dtype != q.dtype or out.shape != q.shape:
        raise ValueError("out must have q's shape and type")
    s = _native.KvRowsStruct()
    s.dtype, s.R, s.Hq, s.T = DTYPES[q.dtype], R, Hq, T
    s.q, s.q_token, s.q_head = q.data_ptr(), q.stride(0), q.stride(1)
    s.out, s.out_token, s.out_head = out.data_ptr(), out.stride(0), out.stride(1)
    s.lse = None if lse is None else lse.data_ptr()
    s.start, s.context, s.table = start.data_ptr(), context.data_ptr(), table.data_ptr()
    s.table_stride = table.stride(0) if R > 1 else table.shape[1]
    s.max_blocks, s.max_new = int(table.shape[1]), int(max_new)
    s.scale = 1.0 / math.sqrt(cache.dim) if scale is None else float(scale)
    s.softcap, s.window = float(softcap), int(window)
    s.slopes = None if slopes is None else slopes.data_ptr()
    s.prefix = None if prefix is None else prefix.data_ptr()
    rc = ctx._lib.kv_attention(ctx.handle, ct.byref(cs), ct.byref(s), _stream(stream, dev))
    ctx.check(rc, "kv_attention")
    _share(stream, dev, cache.k, cache.v, cache.k_scale, cache.v_scale, q, table, start, context,
           slopes, prefix, out, lse)
    return dict(out=out, lse=lse)
