"""Keys and values of passages in pages: the gorio_kv_* calls of libgorio.so.

A search returns the nodes whose passages a model reads next.  Their keys and
values are kept in pages in HBM:

    cache = g.KVCache(keys, values)                     # [pages, heads, page_tokens, D] tensors
    tables, fills, prefix, _ = g.kv_attach(ids, first_page, tokens, cache.page_tokens, width)
    plan = g.kv_plan(prefix, new_lengths, free_pages, tables, cache.page_tokens, total_new)
    cache.store(k, v, plan.slots)                       # in every layer
    out = cache.attend(q, plan.starts, plan.lens, tables, fills=fills, prefix=prefix)
    k, v = cache.load(slots)                            # rows of the pages back

Pages hold 16, 8 or 4 bits an element (KVCache).  Where neighbouring requests'
tables begin with the same pages, g.kv_share finds how far, and attend, told so,
reads those once for all of them.

Argument marshalling only; the work is done by the library's HIP kernels, on
torch's current stream of the tensors' device.  Nothing waits for the GPU.
The calls serve: there are no gradients through pages, and tensors that require
one are refused where torch records gradients.
"""
from __future__ import annotations

import ctypes
import struct
from typing import NamedTuple

BF16, F16, E4M3, MX8, MX4 = 0, 1, 2, 4, 5


class CacheDesc(ctypes.Structure):
    """gorio_kv_cache"""
    _fields_ = [(f, ctypes.c_uint32) for f in ("dtype", "heads", "D", "page_tokens")] + [
        ("num_pages", ctypes.c_uint64), ("keys", ctypes.c_void_p), ("values", ctypes.c_void_p)] + [
        (f, ctypes.c_uint64) for f in ("page_stride", "head_stride", "token_stride")] + [
        (f, ctypes.c_void_p) for f in ("key_scale", "value_scale", "key_powers", "value_powers")]


class AttentionDesc(ctypes.Structure):
    """gorio_kv_attention"""
    _fields_ = [(f, ctypes.c_uint32) for f in ("dtype", "heads", "requests", "width")] + [
        ("tokens", ctypes.c_uint64), ("q", ctypes.c_void_p), ("out", ctypes.c_void_p),
        ("q_stride", ctypes.c_uint64), ("out_stride", ctypes.c_uint64)] + [
        (f, ctypes.c_void_p) for f in ("lse", "starts", "lens", "tables", "fills", "prefix", "slopes")] + [
        ("scale", ctypes.c_float), ("cap", ctypes.c_float), ("window", ctypes.c_uint32),
        ("max_new", ctypes.c_uint32)]


class SharingDesc(ctypes.Structure):
    """gorio_kv_sharing"""
    _fields_ = [("groups", ctypes.c_uint32), ("first", ctypes.c_void_p), ("shared", ctypes.c_void_p)]


_ATTENTION = struct.Struct("4IQ2P2Q7P2f2I")   # AttentionDesc's fields, packed at once
_SHARING = struct.Struct("I4x2P")
assert _ATTENTION.size == ctypes.sizeof(AttentionDesc) and _SHARING.size == ctypes.sizeof(SharingDesc)


def declare(L):
    """Argument types of the gorio_kv_* symbols of the loaded library."""
    v, u32, u64, i32 = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_int
    L.gorio_kv_attach.restype = i32
    L.gorio_kv_attach.argtypes = [v, u64, u32, v, v, u64, u32, u32, u32, v, v, v, v, v]
    L.gorio_kv_plan.restype = i32
    L.gorio_kv_plan.argtypes = [v, v, u64, u32, v, u64, v, u32, u64, v, v, v, v, v, v]
    L.gorio_kv_store.restype = i32
    L.gorio_kv_store.argtypes = [v, i32, v, v, u64, u64, u64, v, v]
    L.gorio_kv_load.restype = i32
    L.gorio_kv_load.argtypes = [v, i32, v, u64, v, v, u64, u64, v]
    L.gorio_kv_share.restype = i32
    L.gorio_kv_share.argtypes = [v, v, v, u64, u32, u32, u32, v, v, v, v]
    L.gorio_kv_attend.restype = i32
    L.gorio_kv_attend.argtypes = [v, v, v, u64, v]
    L.gorio_kv_workspace.restype = i32
    L.gorio_kv_workspace.argtypes = [v, v, v]
    L.gorio_kv_attend_shared.restype = i32
    L.gorio_kv_attend_shared.argtypes = [v, v, v, v, u64, v]
    L.gorio_kv_workspace_shared.restype = i32
    L.gorio_kv_workspace_shared.argtypes = [v, v, v, v]


_torch = _L = None


def _bind():
    """torch and the loaded library, once: a step of a decoding loop is a few of these calls."""
    global _torch, _L
    if _L is None:
        import torch

        from . import lib
        _torch, _L = torch, lib()
    return _torch, _L


def _done(status: int):
    if status:
        from . import _check
        _check(status)


def _stream(device) -> int:
    """torch's current stream of the device, as a handle."""
    return _torch._C._cuda_getCurrentRawStream(device.index)


def _need(name: str, a, dtype, shape, device):
    """Plain pointers cross the C ABI: what they point to is checked here."""
    if a.dtype is dtype and a.shape == shape and a.device == device and a.is_contiguous():
        return
    if a.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {a.dtype}")
    if a.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(a.shape)}")
    if a.device != device:
        raise ValueError(f"{name} must be on {device}, not {a.device}")
    raise ValueError(f"{name} must be contiguous")


def _on_gpu(name: str, a):
    if not a.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    return a.device


def _no_gradients():
    raise ValueError("attend and store compute no gradients: call them under torch.no_grad(), or with tensors that "
                     "require none")


def _count(name: str, value, least: int = 0) -> int:
    value = int(value)
    if not least <= value < 1 << 31:
        raise ValueError(f"{name} is {value}, need {least}..2^31-1")
    return value


def kv_attach(nodes, first_page, tokens, page_tokens: int, width: int, limit: int | None = None):
    """(tables, fills, lens, attached): the pages of the passages that a search
    returned (gorio_kv_attach).  nodes: requests x k int32 or uint32 ids, as
    Index.search returns them; first_page, tokens: int32 per node, a first page
    below 0 for one that has no pages and is passed over; limit: table entries
    that passages may take of the `width` (default: all)."""
    torch, L = _bind()
    dev = _on_gpu("nodes", nodes)
    if nodes.dim() != 2:
        raise ValueError(f"nodes must be (requests, k), not {tuple(nodes.shape)}")
    if nodes.dtype not in (torch.int32, torch.uint32):
        raise TypeError(f"nodes must be int32 or uint32, not {nodes.dtype}")
    B, k = nodes.shape
    _need("nodes", nodes, nodes.dtype, nodes.shape, dev)
    _need("first_page", first_page, torch.int32, tokens.shape, dev)
    _need("tokens", tokens, torch.int32, (tokens.numel(),), dev)
    width = _count("width", width, 1)
    limit = width if limit is None else _count("limit", limit)
    tables = torch.empty((B, width), dtype=torch.int32, device=dev)
    fills = torch.empty_like(tables)
    lens = torch.empty(B, dtype=torch.int32, device=dev)
    attached = torch.empty_like(lens)
    _done(L.gorio_kv_attach(nodes.data_ptr(), B, k, first_page.data_ptr(), tokens.data_ptr(), tokens.numel(),
                            _count("page_tokens", page_tokens), width, limit, tables.data_ptr(), fills.data_ptr(),
                            lens.data_ptr(), attached.data_ptr(), _stream(dev)))
    return tables, fills, lens, attached


class KVPlan(NamedTuple):
    """What kv_plan returns, on the device: starts (requests + 1), lens
    (requests), positions (int32) and slots (int64) of the new tokens, and
    taken (1), the free pages that the step needed."""
    starts: object
    lens: object
    positions: object
    slots: object
    taken: object


def kv_plan(before, added, free_pages, tables, page_tokens: int, tokens: int) -> KVPlan:
    """A step's plan from request lengths (gorio_kv_plan): `tokens` new ones in
    all, or at most; the tables' new entries are written in place."""
    torch, L = _bind()
    dev = _on_gpu("before", before)
    B, width = tables.shape
    _need("before", before, torch.int32, (B,), dev)
    _need("added", added, torch.int32, (B,), dev)
    _need("free_pages", free_pages, torch.int32, (free_pages.numel(),), dev)
    _need("tables", tables, torch.int32, tables.shape, dev)
    T = _count("tokens", tokens)
    starts = torch.empty(B + 1, dtype=torch.int32, device=dev)
    lens = torch.empty_like(before)
    positions = torch.empty(T, dtype=torch.int32, device=dev)
    slots = torch.empty(T, dtype=torch.int64, device=dev)
    taken = torch.empty(1, dtype=torch.int32, device=dev)
    if B == 0:
        starts.zero_(), taken.zero_(), positions.fill_(-1), slots.fill_(-1)
        return KVPlan(starts, lens, positions, slots, taken)
    _done(L.gorio_kv_plan(before.data_ptr(), added.data_ptr(), B, _count("page_tokens", page_tokens),
                          free_pages.data_ptr(), free_pages.numel(), tables.data_ptr(), width, T, lens.data_ptr(),
                          starts.data_ptr(), positions.data_ptr() if T else None, slots.data_ptr() if T else None,
                          taken.data_ptr(), _stream(dev)))
    return KVPlan(starts, lens, positions, slots, taken)


class KVSharing(NamedTuple):
    """What kv_share returns, on the device, int32: first (requests + 1), the
    groups' first requests, and shared (requests), the positions that a request
    shares with its group; common (requests), those it shares with the request
    before it.  A program that knows its groups makes first (groups + 1) and
    shared by itself; a group's rows of the tables name the same pages so far."""
    first: object
    shared: object
    common: object = None


def kv_share(tables, held, page_tokens: int, *, fills=None, least: int = 256) -> KVSharing:
    """Which neighbouring requests have their first pages in common
    (gorio_kv_share), for KVCache.attend.  held (requests, int32): positions
    that all of a request's new tokens see, its tokens before the step or its
    prefix; least: fewer positions than this are not shared."""
    torch, L = _bind()
    dev = _on_gpu("tables", tables)
    if tables.dim() != 2:
        raise ValueError(f"tables must be (requests, width), not {tuple(tables.shape)}")
    B, width = tables.shape
    _need("tables", tables, torch.int32, tables.shape, dev)
    _need("held", held, torch.int32, (B,), dev)
    if fills is not None:
        _need("fills", fills, torch.int32, tables.shape, dev)
    first = torch.empty(B + 1, dtype=torch.int32, device=dev)
    shared, common = torch.empty_like(held), torch.empty_like(held)
    if B == 0:
        return KVSharing(first.zero_(), shared, common)
    _done(L.gorio_kv_share(tables.data_ptr(), None if fills is None else fills.data_ptr(), held.data_ptr(), B, width,
                           _count("page_tokens", page_tokens), _count("least", least), common.data_ptr(),
                           first.data_ptr(), shared.data_ptr(), _stream(dev)))
    return KVSharing(first, shared, common)


class KVCache:
    """The pages of one layer: `keys` and `values` are the program's own
    tensors, pages x heads x page_tokens x D (any strides that are multiples of
    8 elements, the last dimension contiguous), bfloat16, float16 or
    float8_e4m3fn; with 8 bits, key_scale and value_scale (float32, one a head)
    are what an element is to be multiplied by.

    Pages whose elements share a power of two by blocks of 32 (D a multiple of
    32): keys and values float8_e4m3fn, or float4_e2m1fn_x2 whose last dimension
    is D / 2, with key_scale and value_scale float8_e8m0fnu, pages x heads x
    page_tokens x D / 32, which `store` writes as well; their strides are those
    of the elements divided by 32."""

    def __init__(self, keys, values, key_scale=None, value_scale=None):
        import torch
        codes = {torch.bfloat16: BF16, torch.float16: F16, torch.float8_e4m3fn: E4M3, torch.float4_e2m1fn_x2: MX4}
        if keys.dtype not in codes:
            raise TypeError(f"keys must be bfloat16, float16, float8_e4m3fn or float4_e2m1fn_x2, not {keys.dtype}")
        if keys.dim() != 4:
            raise ValueError(f"keys must be (pages, heads, page_tokens, D), not {tuple(keys.shape)}")
        if any(n > 1 and step == 0 for n, step in zip(keys.shape, keys.stride())):
            raise ValueError(f"elements of keys must not share memory, its strides are {keys.stride()}")
        dev = _on_gpu("keys", keys)
        if (values.dtype, values.shape, values.stride(), values.device) != (
                keys.dtype, keys.shape, keys.stride(), keys.device):
            raise ValueError("values must be of the keys' type, shape, strides and device")
        pages, heads, page_tokens, D = keys.shape
        if keys.stride(3) != 1:
            raise ValueError("the last dimension of keys must be contiguous")
        code, wide = codes[keys.dtype], 1                              # wide: elements of one of torch's
        if code == MX4 or any(s is not None and s.dtype == torch.float8_e8m0fnu for s in (key_scale, value_scale)):
            if code not in (E4M3, MX4):
                raise ValueError("scales of float8_e8m0fnu belong to float8_e4m3fn and float4_e2m1fn_x2 pages")
            code, wide = (MX4, 2) if code == MX4 else (MX8, 1)
            D *= wide
            if D % 32:
                raise ValueError(f"D is {D}, need a multiple of 32 for these pages")
            steps = tuple(n * wide / 32 for n in keys.stride()[:3]) + (1,)
            if key_scale is None or value_scale is None:
                raise ValueError("key_scale and value_scale are needed for these pages")
            for name, scale in (("key_scale", key_scale), ("value_scale", value_scale)):
                if scale.dtype != torch.float8_e8m0fnu:
                    raise TypeError(f"{name} must be float8_e8m0fnu, not {scale.dtype}")
                if scale.shape != (pages, heads, page_tokens, D // 32) or scale.device != dev:
                    raise ValueError(f"{name} must have shape {(pages, heads, page_tokens, D // 32)} on {dev}")
                if any(n > 1 and a != b for n, a, b in zip(scale.shape, scale.stride(), steps)):
                    raise ValueError(f"the strides of {name} must be those of the elements divided by 32, {steps}")
        elif code == E4M3:
            for name, scale in (("key_scale", key_scale), ("value_scale", value_scale)):
                if scale is not None:
                    _need(name, scale, torch.float32, (heads,), dev)
        elif key_scale is not None or value_scale is not None:
            raise ValueError("key_scale and value_scale belong to float8_e4m3fn pages")
        self.keys, self.values, self.key_scale, self.value_scale = keys, values, key_scale, value_scale
        self.heads, self.page_tokens, self.D, self.device = heads, page_tokens, D, dev
        self._code = code
        self._codes = {torch.bfloat16: BF16, torch.float16: F16}
        at = [None if s is None else s.data_ptr() for s in (key_scale, value_scale)]
        scales = [None, None, *at] if code in (MX8, MX4) else [*at, None, None]
        self._desc = CacheDesc(code, heads, D, page_tokens, pages, keys.data_ptr(), values.data_ptr(),
                               *(n * wide for n in keys.stride()[:3]), *scales)
        self._ref = ctypes.addressof(self._desc)
        self._layouts, self._spaces = {}, {}    # what _rows found of a layout; workspace bytes of a call's sizes

    def _rows(self, name: str, x, heads: int | None = None):
        """Checks rows of a projection, tokens x heads x D; returns their type and row stride."""
        if x.device != self.device:
            raise ValueError(f"{name} must be on {self.device}, not {x.device}")
        key = (x.dtype, x.shape, x.stride(), heads)
        known = self._layouts.get(key)
        if known is not None:
            return known
        if x.dim() != 3 or x.shape[2] != self.D or (heads is not None and x.shape[1] != heads):
            raise ValueError(f"{name} must be (tokens, {heads or 'heads'}, {self.D}), not {tuple(x.shape)}")
        code = self._codes.get(x.dtype)
        if code is None:
            raise TypeError(f"{name} must be bfloat16 or float16, not {x.dtype}")
        T, H, D = x.shape
        if (D > 1 and x.stride(2) != 1) or (H > 1 and x.stride(1) != D):
            raise ValueError(f"each token's heads in {name} must be contiguous")
        if T > 1 and x.stride(0) < H * D:    # a stride of 0 would mean packed rows to the library
            raise ValueError(f"rows of {name} must not share memory, its strides are {x.stride()}")
        if len(self._layouts) > 4096:
            self._layouts.clear()
        self._layouts[key] = known = code, (x.stride(0) if T > 1 else H * D)
        return known

    def store(self, keys, values, slots):
        """Keys and values of new tokens (tokens x heads x D each; rows may be
        parts of wider ones) into their slots (int64; below 0: not stored)."""
        torch, L = _bind()
        if (keys.requires_grad or values.requires_grad) and torch.is_grad_enabled():
            _no_gradients()
        code, key_stride = self._rows("keys", keys, self.heads)
        code2, value_stride = self._rows("values", values, self.heads)
        if code != code2 or keys.shape != values.shape:
            raise ValueError("keys and values must be of one type and shape")
        T = keys.shape[0]
        _need("slots", slots, torch.int64, (T,), self.device)
        if T:
            _done(L.gorio_kv_store(self._ref, code, keys.data_ptr(), values.data_ptr(), T, key_stride, value_stride,
                                   slots.data_ptr(), _stream(self.device)))

    def load(self, slots, dtype=None, keys=None, values=None):
        """(keys, values): the rows of the pages at `slots` (int64), tokens x heads x
        D each, of the pages' type, or bfloat16 or float16 as `dtype` (or else the
        rows given) says where they hold 8 or 4 bits; zeros where a slot is below 0 or past the pages.
        keys, values: rows to write to (they may be parts of wider ones)."""
        torch, L = _bind()
        if dtype is None:
            given = keys if keys is not None else values
            dtype = given.dtype if given is not None else self.keys.dtype if self._code <= F16 else torch.bfloat16
        _need("slots", slots, torch.int64, (slots.numel(),), self.device)
        T, at = slots.numel(), []
        code = self._codes.get(dtype)
        if code is None:
            raise TypeError(f"rows are bfloat16 or float16, not {dtype}")
        rows = []
        for name, x in (("keys", keys), ("values", values)):
            stride = 0                                                 # packed
            if x is None:
                x = torch.empty((T, self.heads, self.D), dtype=dtype, device=self.device)
            else:
                got, stride = self._rows(name, x, self.heads)
                if got != code or x.shape[0] != T:
                    raise ValueError(f"{name} must be {T} rows of {dtype}")
                if x.requires_grad and torch.is_grad_enabled():
                    _no_gradients()
            rows.append(x)
            at.append(stride)
        if T:
            _done(L.gorio_kv_load(self._ref, code, slots.data_ptr(), T, rows[0].data_ptr(), rows[1].data_ptr(), *at,
                                  _stream(self.device)))
        return tuple(rows)

    def attend(self, q, starts, lens, tables, *, fills=None, prefix=None, slopes=None, scale: float | None = None,
               cap: float = 0.0, window: int = 0, max_new: int = 0, out=None, with_lse: bool = False,
               sharing: KVSharing | None = None):
        """Attention of the new tokens `q` (tokens x heads x D) over the pages
        (gorio_kv_attend): request b's are rows starts[b]..starts[b+1], the last
        of its lens[b] tokens, in the pages that tables[b] names.  Returns out,
        or (out, lse) with `with_lse`; rows past starts[-1] are not written.

        fills (as tables): tokens that each page holds.  prefix (requests): the
        first positions, which all of a request's new tokens see.  slopes
        (heads, float32): a score loses slope * distance.  scale: 1/sqrt(D) by
        default.  cap: scores become cap * tanh(score / cap).  window: the distance
        from which a key outside the prefix is not seen (0: none).
        max_new: the most new tokens of a request, where the program knows it.
        sharing: which requests have their first pages in common, from kv_share;
        these are then read once for all of a group (gorio_kv_attend_shared)."""
        torch, L = _bind()
        dev, i32 = self.device, torch.int32
        if (q.requires_grad or self.keys.requires_grad or self.values.requires_grad or (
                slopes is not None and slopes.requires_grad)) and torch.is_grad_enabled():
            _no_gradients()
        code, q_stride = self._rows("q", q)
        T, H, D = q.shape
        B, width = tables.shape
        _need("tables", tables, i32, (B, width), dev)
        _need("starts", starts, i32, (B + 1,), dev)
        _need("lens", lens, i32, (B,), dev)
        if fills is not None:
            _need("fills", fills, i32, (B, width), dev)
        if prefix is not None:
            _need("prefix", prefix, i32, (B,), dev)
        if slopes is not None:
            _need("slopes", slopes, torch.float32, (H,), dev)
        if out is None:
            out, out_stride = torch.empty((T, H, D), dtype=q.dtype, device=dev), H * D
        else:
            out_code, out_stride = self._rows("out", out, H)
            if out_code != code or out.shape[0] != T:
                raise ValueError("out must be of q's type and shape")
        lse = torch.empty((T, H), dtype=torch.float32, device=dev) if with_lse else None
        window, max_new = _count("window", window), _count("max_new", max_new)
        a = _ATTENTION.pack(code, H, B, width, T, q.data_ptr(), out.data_ptr(), q_stride, out_stride,
                            0 if lse is None else lse.data_ptr(), starts.data_ptr(), lens.data_ptr(),
                            tables.data_ptr(), 0 if fills is None else fills.data_ptr(),
                            0 if prefix is None else prefix.data_ptr(), 0 if slopes is None else slopes.data_ptr(),
                            D ** -0.5 if scale is None else scale, cap, window, max_new)
        groups, share = 0, None
        if sharing is not None and B:
            groups = sharing.first.numel() - 1
            _need("sharing.first", sharing.first, i32, (groups + 1,), dev)
            _need("sharing.shared", sharing.shared, i32, (B,), dev)
            share = _SHARING.pack(max(groups, 0), sharing.first.data_ptr(), sharing.shared.data_ptr())
        # a window without a prefix needs no room for what is shared
        sizes = (code, T, H, B, width, max_new, share and groups, share and window and prefix is None)
        need = self._spaces.get(sizes)
        if need is None:
            got = ctypes.c_uint64()
            if share is None:
                _done(L.gorio_kv_workspace(self._ref, a, ctypes.addressof(got)))
            else:
                _done(L.gorio_kv_workspace_shared(self._ref, a, share, ctypes.addressof(got)))
            if len(self._spaces) > 4096:
                self._spaces.clear()
            need = self._spaces[sizes] = got.value
        space = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
        at = None if space is None else space.data_ptr()
        if share is None:
            _done(L.gorio_kv_attend(self._ref, a, at, need, _stream(dev)))
        else:
            _done(L.gorio_kv_attend_shared(self._ref, a, share, at, need, _stream(dev)))
        return (out, lse) if with_lse else out
