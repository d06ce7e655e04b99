"""Binding of the paged-cache entry points (block tables, store, load, attention, attention
behind shared prefixes; include/dro.h).  Argument checks and marshalling only."""
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


def _need_table(t, device, name="table"):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if device is not None and t.device != device:
        raise TypeError(f"{name} is on {t.device}, expected {device}")
    shape, stride = t.shape, t.stride()
    if t.dtype is not torch.int32 or len(shape) != 2 or (shape[1] > 1 and stride[1] != 1):
        raise ValueError(f"{name} must be an int32 [R, max_blocks] tensor with contiguous rows")
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


MXFP4, MXFP8 = 3, 4
_GROUP = 32  # components that share a power of two


@dataclass(frozen=True)
class KvCache:
    """One layer's cache (field meanings as in dro_kv_cache): k and v are
    [num_blocks, block, heads, dim] tensors, strided as they like except for the
    contiguous components, in torch.bfloat16, torch.float16 or, with scales,
    torch.float8_e4m3fn.  With k_power and v_power, uint8 [num_blocks, block, heads,
    dim / 32] whose groups and tokens of a head lie next to one another, the cache is in
    shared scales: MXFP8 if k and v are torch.float8_e4m3fn, MXFP4 if they are torch.uint8
    [.., dim / 2], two components a byte.  The tensors are checked once, here, and stay the cache's."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: Optional[torch.Tensor] = None   # float32 [heads]
    v_scale: Optional[torch.Tensor] = None
    k_power: Optional[torch.Tensor] = None
    v_power: Optional[torch.Tensor] = None

    @classmethod
    def empty(cls, num_blocks, block, heads, dim, dtype=torch.bfloat16, device="cuda",
              k_scale=None, v_scale=None):
        """A zeroed cache whose blocks hold the tokens of a head next to one another; dtype is a
        torch one, "mxfp4" or "mxfp8"."""
        def zeros(width, t):
            return torch.zeros((num_blocks, heads, block, width), dtype=t, device=device).permute(0, 2, 1, 3)

        if dtype in ("mxfp4", "mxfp8"):
            if k_scale is not None or v_scale is not None:
                raise ValueError(f"{dtype} has no k_scale and v_scale")
            if dim % _GROUP:
                raise ValueError(f"dim={dim} is not a multiple of {_GROUP}, as {dtype} needs")
            code = (dim // 2, torch.uint8) if dtype == "mxfp4" else (dim, torch.float8_e4m3fn)
            return cls(zeros(*code), zeros(*code), k_power=zeros(dim // _GROUP, torch.uint8),
                       v_power=zeros(dim // _GROUP, torch.uint8))
        k, v = zeros(dim, dtype), zeros(dim, dtype)
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

    @property
    def tensors(self) -> tuple:
        """The tensors that it is made of."""
        return tuple(t for t in (self.k, self.v, self.k_scale, self.v_scale, self.k_power, self.v_power)
                     if t is not None)

    def __post_init__(self):
        mx = self.k_power is not None or self.v_power is not None
        for name, t in (("k", self.k), ("v", self.v)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"cache {name} must be a CUDA tensor")
            if mx and t.dtype not in (torch.uint8, torch.float8_e4m3fn):
                raise TypeError(f"cache {name} must be uint8 (MXFP4) or float8_e4m3fn (MXFP8) beside its "
                                f"powers, got {t.dtype}")
            if not mx and t.dtype not in DTYPES:
                raise TypeError(f"cache {name} must be bfloat16, float16 or float8_e4m3fn, got {t.dtype}")
            if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
                raise ValueError(f"cache {name} must be [num_blocks, block, heads, dim] with "
                                 "contiguous components")
        if self.v.shape != self.k.shape or self.v.dtype != self.k.dtype or self.v.device != self.k.device:
            raise ValueError("cache k and v differ in shape, type or device")
        s = _native.KvCacheStruct()
        four = self.k.dtype is torch.uint8
        s.dtype = DTYPES[self.k.dtype] if not mx else MXFP4 if four else MXFP8
        s.num_blocks, s.block, s.heads, s.dim = self.k.shape
        s.k, s.v = self.k.data_ptr(), self.v.data_ptr()
        of = 2 if four else 1  # (strides are in components)
        s.dim *= of
        s.k_block, s.k_token, s.k_head = (of * x for x in self.k.stride()[:3])
        s.v_block, s.v_token, s.v_head = (of * x for x in self.v.stride()[:3])
        if mx:
            if s.dim % _GROUP:
                raise ValueError(f"dim={s.dim} is not a multiple of {_GROUP}, as shared scales need")
            shape = tuple(self.k.shape[:3]) + (s.dim // _GROUP,)
            for name in ("k_power", "v_power"):
                t = getattr(self, name)
                if not isinstance(t, torch.Tensor) or t.dtype is not torch.uint8 or t.device != self.k.device:
                    raise TypeError(f"{name} must be a uint8 tensor on {self.k.device}")
                if (tuple(t.shape) != shape or (shape[3] > 1 and t.stride(3) != 1)
                        or (shape[1] > 1 and t.stride(1) != shape[3])):
                    raise ValueError(f"{name} must have shape {shape} with a head's tokens of a block next "
                                     f"to one another, got {tuple(t.shape)} strided {t.stride()}")
            s.k_power, s.v_power = self.k_power.data_ptr(), self.v_power.data_ptr()
            # (the stride of a dimension of one entry may be anything)
            for name in ("k_power", "v_power"):
                blocks, _, heads, _ = getattr(self, name).stride()
                setattr(s, name + "_block", blocks if shape[0] > 1 else 0)
                setattr(s, name + "_head", heads if shape[2] > 1 else 0)
        for name in ("k_scale", "v_scale"):
            t = getattr(self, name)
            if t is not None:
                setattr(s, name, _need(t, torch.float32, name, self.k.device, s.heads))
        object.__setattr__(self, "_struct", s)
        object.__setattr__(self, "_grad", any(t.requires_grad for t in self.tensors))

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
        _share(stream, dev, *cache.tensors, k, v, slot)


def kv_load(ctx: Context, cache: KvCache, slot: torch.Tensor, dtype=None, k=None, v=None,
            stream=None) -> dict:
    """The keys and values of the slots [T] out of the cache, as rows [T, heads, dim] (see kv_load
    in dro.h): of torch.bfloat16 or torch.float16, a 16-bit cache of its own type (the default; of
    a cache of 8 or 4 bits torch.bfloat16).  k and v are written if given, strided as kv_store's.
    No backward pass: inputs that require grad are refused where gradients are recorded."""
    dev, cs = cache.device, cache._struct
    if dev.index != ctx.device.index:
        _other_device(ctx, dev)
    if not isinstance(slot, torch.Tensor):
        raise TypeError("slot must be a CUDA tensor")
    T = slot.numel()
    if dtype is None:
        given = k if k is not None else v
        dtype = (getattr(given, "dtype", None) if given is not None else
                 torch.bfloat16 if cs.dtype not in (0, 1) else cache.k.dtype)
    if dtype is not torch.bfloat16 and dtype is not torch.float16:
        raise TypeError(f"dtype must be torch.bfloat16 or torch.float16, got {dtype}")
    slot_p = _need(slot, torch.int64, "slot", dev, T)
    with nullcontext() if stream is None else torch.cuda.stream(stream):
        out = []
        for name, t in (("k", k), ("v", v)):
            if t is None:
                out.append((torch.empty((T, cs.heads, cs.dim), dtype=dtype, device=dev),
                            (cs.heads * cs.dim, cs.dim)))
                continue
            rows, stride = _need_rows(t, name, dev, cs.heads, cs.dim)
            if t.dtype is not dtype or rows != T:
                raise ValueError(f"{name} must hold {T} rows of {dtype}")
            out.append((t, stride))
    (k, ks), (v, vs) = out
    if k.requires_grad or v.requires_grad or cache._grad:
        _no_gradient("kv_load")
    rc = ctx._lib.kv_load(ctx.handle, ct.byref(cs), DTYPES[dtype], T, k.data_ptr(), ks[0], ks[1],
                          v.data_ptr(), vs[0], vs[1], slot_p, _queue(stream, dev))
    if rc:
        ctx.check(rc, "kv_load")
    if stream is not None:
        _share(stream, dev, *cache.tensors, k, v, slot)
    return dict(k=k, v=v)


@dataclass
class SharedPrefixes:
    """Prefixes that groups of consecutive requests share (field meanings as in dro_kv_shared)."""
    first: torch.Tensor        # int32 [groups + 1] first request of each group, and the end
    context: torch.Tensor      # int32 [groups] tokens of each prefix
    table: torch.Tensor        # int32 [groups, max_blocks] its blocks, rows may be strided
    max_new: int               # bounds the rows of a group

    def struct(self, device) -> _native.KvSharedStruct:
        groups, width, stride = _need_table(self.table, device, "the table of the shared prefixes")
        return _native.KvSharedStruct(
            groups, _need(self.first, torch.int32, "first", device, groups + 1),
            _need(self.context, torch.int32, "context of the shared prefixes", device, groups),
            self.table.data_ptr(), stride, width, _int32(self.max_new))


def kv_attention(ctx: Context, cache: KvCache, q: torch.Tensor, table: torch.Tensor,
                 start: torch.Tensor, context: torch.Tensor, max_new: int, scale=None,
                 softcap: float = 0.0, window: int = 0, slopes: Optional[torch.Tensor] = None,
                 prefix: Optional[torch.Tensor] = None, out=None, lse=None, want_lse: bool = True,
                 stream=None) -> dict:
    """Attention of the rows q [T, Hq, dim] over the cache (see kv_attention in dro.h).  `table`
    is a BlockPool's, `start` and `context` come from kv_block_tables; max_new bounds the rows of
    one request.  scale defaults to dim ** -0.5.  No backward pass: inputs that require grad are
    refused where gradients are recorded."""
    return _attention(ctx, cache, q, table, start, context, max_new, None, scale, softcap, window,
                      slopes, prefix, out, lse, want_lse, stream)


def kv_shared_attention(ctx: Context, cache: KvCache, q: torch.Tensor, table: torch.Tensor,
                        start: torch.Tensor, context: torch.Tensor, max_new: int,
                        shared: SharedPrefixes, scale=None, softcap: float = 0.0, window: int = 0,
                        slopes: Optional[torch.Tensor] = None,
                        prefix: Optional[torch.Tensor] = None, out=None, lse=None,
                        want_lse: bool = True, stream=None) -> dict:
    """kv_attention behind prefixes that the cache holds, and the call reads, once for a group of
    requests (see kv_shared_attention in dro.h): `table`, `context` and `prefix` are of the
    requests' own tokens, which follow the group's in `shared`."""
    if not isinstance(shared, SharedPrefixes):
        raise TypeError("shared must be SharedPrefixes")
    return _attention(ctx, cache, q, table, start, context, max_new, shared, scale, softcap, window,
                      slopes, prefix, out, lse, want_lse, stream)


def _attention(ctx, cache, q, table, start, context, max_new, shared, scale, softcap, window, slopes,
               prefix, out, lse, want_lse, stream):
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
        _no_gradient("kv_attention" if shared is None else "kv_shared_attention")
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
    if shared is None:
        rc = ctx._lib.kv_attention(ctx.handle, ct.byref(cs), ct.byref(rows), _queue(stream, dev))
    else:
        prefixes = shared.struct(dev)
        rc = ctx._lib.kv_shared_attention(ctx.handle, ct.byref(cs), ct.byref(rows), ct.byref(prefixes),
                                          _queue(stream, dev))
    if rc:
        ctx.check(rc, "kv_attention" if shared is None else "kv_shared_attention")
    if stream is not None:
        _share(stream, dev, *cache.tensors, q, table, start, context, slopes, prefix, out, lse,
               *(() if shared is None else (shared.first, shared.context, shared.table)))
    return dict(out=out, lse=lse)
