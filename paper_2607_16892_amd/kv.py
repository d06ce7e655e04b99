"""Binding of the paged-cache entry points (block tables, store, attention;
include/dro.h).  Argument checks and marshalling only."""
from __future__ import annotations

import ctypes as ct
from contextlib import nullcontext
from dataclasses import dataclass
from typing import Optional

import torch

from . import _native
from .api import Context, _need_dev, _out

DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float8_e4m3fn: 2}

_raw_stream = torch._C._cuda_getCurrentRawStream


def _queue(stream, device) -> int:
    """The hipStream_t of a call (a decode step makes many short calls: no Stream object)."""
    return _raw_stream(device.index) if stream is None else stream.cuda_stream


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
    if t.dtype is not torch.bfloat16 and t.dtype is not torch.float16:
        raise TypeError(f"{name} must be torch.bfloat16 or torch.float16, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name} must have shape (T, {heads}, {dim}), got {tuple(shape)}")
    stride = t.stride()
    if dim > 1 and stride[2] != 1:
        raise ValueError(f"the components of {name} must be contiguous")
    return shape[0], stride


def _need(t, dtype, name, device, n):
    """A contiguous tensor of n elements."""
    if (not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device
            or not t.is_contiguous()):
        _need_dev(t, dtype, name, device)
    if t.numel() != n:
        raise ValueError(f"{name} must hold {n} entries, got {t.numel()}")
    return t.data_ptr()


# (Checks that nearly every call passes stand in the calls themselves, as one comparison: a decode
# step makes a call a layer, and a Python call more takes a tenth of a microsecond.)
def _other_device(ctx, device):
    """The kernels run on the context's device: tensors of another one would be out of their reach."""
    if device.index != (ctx.device.index or 0):
        raise ValueError(f"the context is on {ctx.device}, the tensors are on {device}")


def _no_gradient(where):
    """The calls have no backward pass: rather an error than a gradient that is lost."""
    if torch.is_grad_enabled():
        raise RuntimeError(f"{where} has no backward pass, and an input requires grad: call it under "
                           "torch.no_grad() or on detached tensors")


def _int32(x):
    """x for a 32-bit field: beyond its ends, the end (ctypes would take the low 32 bits)."""
    return min(max(x, -2 ** 31), 2 ** 31 - 1)


def _need_table(t, device):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("table must be a CUDA tensor")
    if device is not None and t.device != device:
        raise TypeError(f"table is on {t.device}, expected {device}")
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or (shape[1] > 1 and stride[1] != 1):
        raise ValueError("table must be an int32 [R, max_blocks] tensor with contiguous rows")
    return shape[0], shape[1], stride[0] if shape[0] > 1 else shape[1]


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
        R, width, stride = _need_table(self.table, None)
        dev, nb = self.table.device, self.free_list.numel()
        return _native.KvPoolStruct(
            R, _int32(self.block), nb, width, stride, self.table.data_ptr(),
            _need(self.free_list, torch.int32, "free_list", dev, nb),
            _need(self.held, torch.int32, "held", dev, R),
            _need(self.free, torch.int32, "free", dev, 1))


@dataclass(frozen=True)
class KvCache:
    """One layer's cache (field meanings as in dro_kv_cache): k and v are
    [num_blocks, block, heads, dim] tensors, strided as they like except for the
    contiguous components, in torch.bfloat16, torch.float16 or, with scales,
    torch.float8_e4m3fn.  The tensors are checked once, here, and stay the cache's."""
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
        return self._struct.heads

    @property
    def dim(self) -> int:
        return self._struct.dim

    def __post_init__(self):
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
        s = _native.KvCacheStruct()
        s.dtype = DTYPES[self.k.dtype]
        s.num_blocks, s.block, s.heads, s.dim = self.k.shape
        s.k, s.v = self.k.data_ptr(), self.v.data_ptr()
        s.k_block, s.k_token, s.k_head = self.k.stride()[:3]
        s.v_block, s.v_token, s.v_head = self.v.stride()[:3]
        for name in ("k_scale", "v_scale"):
            t = getattr(self, name)
            if t is not None:
                setattr(s, name, _need(t, torch.float32, name, self.k.device, s.heads))
        object.__setattr__(self, "_struct", s)
        object.__setattr__(self, "_grad", any(t is not None and t.requires_grad for t in
                                              (self.k, self.v, self.k_scale, self.v_scale)))

    def struct(self) -> _native.KvCacheStruct:
        return self._struct


def kv_block_tables(ctx: Context, pool: BlockPool, length: torch.Tensor, add: torch.Tensor,
                    tokens: int, reserve: Optional[torch.Tensor] = None, out: Optional[dict] = None,
                    stream=None) -> dict:
    """Blocks and slots of one step's `tokens` new tokens (see kv_block_tables in dro.h): the
    pool's table and free_list change in place; held and free after the step are outputs, which
    pool.take makes the pool's."""
    ps = pool.struct()
    dev, R, T = pool.device, ps.R, int(tokens)
    if dev.index != ctx.device.index:
        _other_device(ctx, dev)
    if T < 0:
        raise ValueError("tokens must not be negative")
    i32 = torch.int32
    len_p, add_p = _need(length, i32, "length", dev, R), _need(add, i32, "add", dev, R)
    res_p = None if reserve is None else _need(reserve, i32, "reserve", dev, R)
    with nullcontext() if stream is None else torch.cuda.stream(stream):
        if out:
            o = {name: _out(out.get(name), (n,), dtype, dev, name)
                 for name, n, dtype in (("held", R, i32), ("free", 1, i32), ("context", R, i32),
                                        ("start", R + 1, i32), ("pos", T, i32),
                                        ("slot", T, torch.int64), ("granted", R, torch.uint8))}
        else:  # one buffer for the 32-bit ones
            parts = torch.empty(3 * R + 2 + T, dtype=i32, device=dev).split_with_sizes((R, 1, R, R + 1, T))
            o = dict(zip(("held", "free", "context", "start", "pos"), parts))
            o["slot"] = torch.empty(T, dtype=torch.int64, device=dev)
            o["granted"] = torch.empty(R, dtype=torch.uint8, device=dev)
    rc = ctx._lib.kv_block_tables(ctx.handle, ct.byref(ps), len_p, add_p, res_p, T,
                                  o["held"].data_ptr(), o["free"].data_ptr(), o["context"].data_ptr(),
                                  o["start"].data_ptr(), o["slot"].data_ptr(), o["pos"].data_ptr(),
                                  o["granted"].data_ptr(), _queue(stream, dev))
    if rc:
        ctx.check(rc, "kv_block_tables")
    if stream is not None:
        _share(stream, dev, pool.table, pool.held, pool.free_list, pool.free, length, add, reserve,
               *o.values())
    return o


def kv_store(ctx: Context, cache: KvCache, k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor,
             stream=None) -> None:
    """The keys and values [T, heads, dim] of T tokens into their slots of the cache (see
    kv_store in dro.h); the tokens and heads may be strided (views of a joint projection).
    No backward pass: inputs that require grad are refused where gradients are recorded."""
    dev, cs = cache.device, cache._struct
    if dev.index != ctx.device.index:
        _other_device(ctx, dev)
    T, ks = _need_rows(k, "k", dev, cs.heads, cs.dim)
    Tv, vs = _need_rows(v, "v", dev, cs.heads, cs.dim)
    if v.dtype is not k.dtype or Tv != T:
        raise ValueError("k and v differ in shape or type")
    if k.requires_grad or v.requires_grad or cache._grad:
        _no_gradient("kv_store")
    rc = ctx._lib.kv_store(ctx.handle, ct.byref(cs), DTYPES[k.dtype], T, k.data_ptr(), ks[0], ks[1],
                           v.data_ptr(), vs[0], vs[1], _need(slot, torch.int64, "slot", dev, T),
                           _queue(stream, dev))
    if rc:
        ctx.check(rc, "kv_store")
    if stream is not None:
        _share(stream, dev, cache.k, cache.v, cache.k_scale, cache.v_scale, k, v, slot)


def kv_attention(ctx: Context, cache: KvCache, q: torch.Tensor, table: torch.Tensor,
                 start: torch.Tensor, context: torch.Tensor, max_new: int, scale=None,
                 softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                 prefix: Optional[torch.Tensor] = None, out=None, lse=None, want_lse: bool = True,
                 stream=None) -> dict:
    """Attention of the rows q [T, Hq, dim] over the cache (see kv_attention in dro.h).  `table`
    is a BlockPool's, `start` and `context` come from kv_block_tables; max_new bounds the rows of
    one request.  scale defaults to dim ** -0.5.  No backward pass: inputs that require grad are
    refused where gradients are recorded."""
    dev, cs = cache.device, cache._struct
    if dev.index != ctx.device.index:
        _other_device(ctx, dev)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise TypeError("q must be a [T, Hq, dim] CUDA tensor")
    Hq, dim = q.shape[1], cs.dim
    T, qs = _need_rows(q, "q", dev, Hq, dim)
    R, width, table_stride = _need_table(table, dev)
    start_p = _need(start, torch.int32, "start", dev, R + 1)
    context_p = _need(context, torch.int32, "context", dev, R)
    prefix_p = None if prefix is None else _need(prefix, torch.int32, "prefix", dev, R)
    slopes_p = None if slopes is None else _need(slopes, torch.float32, "slopes", dev, Hq)
    if q.requires_grad or cache._grad or (slopes is not None and slopes.requires_grad):
        _no_gradient("kv_attention")
    if not 0 <= window < 2 ** 31 or not 0 <= max_new < 2 ** 31:
        window, max_new = _int32(window), _int32(max_new)
    with nullcontext() if stream is None else torch.cuda.stream(stream):
        if out is None:
            out = torch.empty((T, Hq, dim), dtype=q.dtype, device=dev)
            os = (Hq * dim, dim)
        else:
            To, os = _need_rows(out, "out", dev, Hq, dim)
            if out.dtype is not q.dtype or To != T:
                raise ValueError("out must have q's shape and type")
        if lse is not None:
            lse = _out(lse, (T, Hq), torch.float32, dev, "lse")
        elif want_lse:
            lse = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    rows = _native.KvRowsStruct(
        DTYPES[q.dtype], R, Hq, T, q.data_ptr(), qs[0], qs[1], out.data_ptr(), os[0], os[1],
        None if lse is None else lse.data_ptr(), start_p, context_p, table.data_ptr(), table_stride,
        width, int(max_new), dim ** -0.5 if scale is None else scale, softcap, window, slopes_p,
        prefix_p)
    rc = ctx._lib.kv_attention(ctx.handle, ct.byref(cs), ct.byref(rows), _queue(stream, dev))
    if rc:
        ctx.check(rc, "kv_attention")
    if stream is not None:
        _share(stream, dev, cache.k, cache.v, cache.k_scale, cache.v_scale, q, table, start, context,
               slopes, prefix, out, lse)
    return dict(out=out, lse=lse)
