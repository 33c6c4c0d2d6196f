"""A cache of keys and values in 8 bits, and attention over it: the calls of admmq_cache.h on torch tensors.

    cache = KVCache(n_pages, kv_heads, head_dim, page_size=64)
    plan = CachePlan(lengths, held, tables, group=q_heads // kv_heads)  # new rows, tokens before them, pages: per request
    cache.write(k, v, plan)                                             # rows as qk_norm_rope and the projections leave them
    out, lse = cache.attend(q, plan)                                    # every row sees what its request holds up to itself
    k, v = cache.read(plan)                                             # what the cache holds at the plan's rows
    plan.held += 1                                                      # the next token

16 neighbouring tokens of a head share a scale, max |x| / 127, for keys and for values; where a later token of the 16 is
larger, the codes that are there are rounded to the new scale.  Every step runs in the library's kernels, on the current
stream of the cache's device, and can be captured after a first call outside a capture; the device reads `held` and `tables`
when it runs, so a captured step follows them (keep the plan and the cache: a graph holds their pointers).  Argument errors
raise AdmmqError before anything is enqueued; a request that does not fit its table, or a page that does not exist, raises it
in adapt.check_device_status.  No call records an autograd graph: inputs that require grad are refused while grad mode is on.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple, Union

import numpy as np
import torch

from . import adapt, binding as B
from .adapt import _need, _no_graph

BLOCK = 16                        # tokens that share the scale of a head


class _Cache(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("n_pages", C.c_int), ("kv_heads", C.c_int), ("head_dim", C.c_int),
                ("page_size", C.c_int), ("d_codes", C.c_void_p), ("d_scale", C.c_void_p)]


class _Plan(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("n_requests", C.c_int), ("max_pages", C.c_int), ("group", C.c_int),
                ("n_blocks", C.c_int), ("n_small", C.c_int), ("n_big", C.c_int), ("small_rows", C.c_int), ("n_rows", C.c_longlong),
                ("d_tables", C.c_void_p), ("d_held", C.c_void_p), ("d_index", C.c_void_p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = adapt._library()
        vp, ci, cll = C.c_void_p, C.c_int, C.c_longlong
        for f in (lib.admmq_cache_code_bytes, lib.admmq_cache_scale_bytes):
            f.restype, f.argtypes = C.c_size_t, [ci] * 4
        lib.admmq_cache_plan_ints.restype, lib.admmq_cache_plan_ints.argtypes = cll, [vp, ci, ci]
        lib.admmq_cache_plan_fill.argtypes = [vp, ci, ci, vp, vp]
        for f in (lib.admmq_cache_write, lib.admmq_cache_read):
            f.argtypes = [vp, vp, ci, vp, cll, cll, vp, cll, cll, vp, vp]
        lib.admmq_cache_attend_workspace.restype, lib.admmq_cache_attend_workspace.argtypes = C.c_size_t, [vp, vp]
        lib.admmq_cache_attend.argtypes = [vp, vp, C.c_double, ci, vp, cll, cll, vp, cll, cll, vp, vp, C.c_size_t, vp, vp]
        _lib = lib
    return _lib


def _host(x, dtype, name):
    """A sequence as an array of whole numbers; what does not fit, or lists of different lengths, is refused."""
    try:
        a = np.ascontiguousarray(np.asarray(x, dtype=dtype))
        fits = x.__class__ is list or bool((a == np.asarray(x)).all())   # (of a list's numbers numpy refuses those that do not,
    except (TypeError, ValueError, OverflowError):                       # an array's it wraps around)
        fits = False
    _need(fits, f"CachePlan: {name}: whole numbers of {8 * np.dtype(dtype).itemsize} bits", B.ERR_SHAPE)
    return a


def _ints(x, shape, device, name):
    """An int32 tensor on the device, used in place; an array is copied there."""
    if not torch.is_tensor(x):
        x = torch.from_numpy(x).to(device)
    _need(x.dtype is torch.int32 and x.is_cuda and x.is_contiguous(), f"CachePlan: contiguous int32 {name} on a GPU")
    _need(x.dim() == len(shape) and all(s is None or s == n for s, n in zip(shape, x.shape)), f"CachePlan: {name} {shape}",
          B.ERR_SHAPE)
    return x


class CachePlan:
    """The rows of a call: request i has lengths[i] adjacent rows, at its positions held[i] .. held[i] + lengths[i] - 1, and
    its position p is token p % page_size of page tables[i, p // page_size].

    lengths are the host's.  held [requests] and tables [requests, pages], int32, may be tensors on the device, which are
    used in place: what is written into them later holds for later calls and replays.  held[i] < 0: request i takes no part.
    group: query heads to a key head, for `attend`."""

    def __init__(self, lengths: Sequence[int], held: Union[torch.Tensor, Sequence[int]],
                 tables: Union[torch.Tensor, Sequence[Sequence[int]]], group: int = 1, device="cuda"):
        lengths = _host(lengths, np.int64, "lengths").reshape(-1)
        lib, n = _library(), len(lengths)
        size = lib.admmq_cache_plan_ints(lengths.ctypes.data, n, group) if 0 < n < 2 ** 31 and 0 < group < 2 ** 31 else -1
        _need(size >= 0, "CachePlan: at least one request, no negative length, at most 2^30 rows, group 1 to 1024", B.ERR_SHAPE)
        self._c = _Plan(struct_size=C.sizeof(_Plan))
        host = np.empty(size, dtype=np.int32)
        st = lib.admmq_cache_plan_fill(lengths.ctypes.data, n, group, host.ctypes.data, C.addressof(self._c))
        _need(st == B.OK, "admmq_cache_plan_fill", st)
        if not torch.is_tensor(tables):
            tables = _host(tables, np.int32, "tables")
        if not torch.is_tensor(held):
            held = _host(held, np.int32, "held")
        device = tables.device if torch.is_tensor(tables) else held.device if torch.is_tensor(held) else device
        self.tables, self.held = _ints(tables, (n, None), device, "tables"), _ints(held, (n,), device, "held")
        self.device, self.index = self.tables.device, self.tables.get_device()
        _need(self.held.device == self.device, "CachePlan: one device")
        _need(self.tables.shape[1] > 0, "CachePlan: tables without a page", B.ERR_SHAPE)
        self._index = torch.from_numpy(host).to(self.device)
        self.n_requests, self.group, self.n_rows = n, group, self._c.n_rows
        self._c.max_pages = self.tables.shape[1]
        self._c.d_tables, self._c.d_held, self._c.d_index = self.tables.data_ptr(), self.held.data_ptr(), self._index.data_ptr()
        self._ref = C.addressof(self._c)

    def _in_place(self, name):
        _need(self.tables.data_ptr() == self._c.d_tables and self.held.data_ptr() == self._c.d_held,
              name + ": a tensor of the plan has other storage than when the plan was made")


class KVCache:
    """n_pages pages of page_size tokens (16, 32, 64, 128 or 256), kv_heads heads of head_dim values (a multiple of 16, at
    most 256).  codes and scale [n_pages, ...] hold page after page, in an order of the library's own: pages may be copied
    whole.  What a page held before does not matter once its tokens are written again from the start of a block on."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, page_size: int = 64, device="cuda"):
        lib = _library()
        sizes = (n_pages, kv_heads, head_dim, page_size)
        _need(all(0 < s < 2 ** 31 for s in sizes) and lib.admmq_cache_code_bytes(*sizes) > 0, "KVCache: head_dim a multiple of "
              "16 up to 256, pages of 16, 32, 64, 128 or 256 tokens, at most 4096 heads", B.ERR_SHAPE)
        device = torch.device(device)
        _need(device.type == "cuda", "KVCache: a GPU")
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.n_pages, self.kv_heads, self.head_dim, self.page_size = sizes
        self.codes = torch.empty(n_pages, lib.admmq_cache_code_bytes(*sizes) // n_pages, dtype=torch.uint8, device=device)
        self.scale = torch.empty(n_pages, lib.admmq_cache_scale_bytes(*sizes) // n_pages // 4, dtype=torch.float32, device=device)
        self.device, self.index = device, self.codes.get_device()
        self._c = _Cache(C.sizeof(_Cache), *sizes, self.codes.data_ptr(), self.scale.data_ptr())
        self._ref, self._status, self._softmax = C.addressof(self._c), adapt._status(self.index), head_dim ** -0.5

    def _check(self, plan, name):
        _need(isinstance(plan, CachePlan) and plan.index == self.index, name + ": a CachePlan on the cache's device")
        _need(self.codes.data_ptr() == self._c.d_codes and self.scale.data_ptr() == self._c.d_scale,
              name + ": the cache's tensors have other storage than when it was made")
        plan._in_place(name)

    def _strides(self, x, heads, dtype, plan, name):
        _need(x.dtype is dtype and x.get_device() == self.index, f"{name}: {dtype} on cuda:{self.index}")
        _need(x.dim() == 3 and tuple(x.shape) == (plan.n_rows, heads, self.head_dim),
              f"{name}: [{plan.n_rows}, {heads}, {self.head_dim}]", B.ERR_SHAPE)
        _need(x.numel() == 0 or x.stride(2) == 1, name + ": adjacent values of a head", B.ERR_SHAPE)
        return (x.stride(0) if x.shape[0] > 1 else 0), (x.stride(1) if heads > 1 else 0)

    def write(self, k: torch.Tensor, v: torch.Tensor, plan: CachePlan) -> None:
        """Rows k, v [rows, kv_heads, head_dim], bf16 or fp32, any row and head strides, to the plan's positions.  A
        page may be written through one entry of the tables only."""
        if plan.__class__ is CachePlan:
            r = adapt._fast.cache_write(self._status, self._ref, plan._ref, self.codes, self.scale, plan.tables, plan.held, k, v)
            if r is None:
                return
        name = "admmq_cache_write"
        self._check(plan, name)
        _no_graph(name, k, v)
        _need(k.dtype in (torch.bfloat16, torch.float32), name + ": bf16 or fp32")
        sk, sv = self._strides(k, self.kv_heads, k.dtype, plan, name + " k"), self._strides(v, self.kv_heads, k.dtype, plan, name + " v")
        adapt._call(_library().admmq_cache_write, name, self.index, self._ref, plan._ref, 1 if k.dtype is torch.bfloat16 else 0,
                    k.data_ptr(), *sk, v.data_ptr(), *sv, self._status)

    def read(self, plan: CachePlan, dtype: torch.dtype = torch.bfloat16, k: Optional[torch.Tensor] = None,
             v: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(k, v) [rows, kv_heads, head_dim]: scale * code at the plan's positions."""
        if k is None and v is None and plan.__class__ is CachePlan and (dtype is torch.bfloat16 or dtype is torch.float32):
            r = adapt._fast.cache_read(self._status, self._ref, plan._ref, self.codes, self.scale, plan.tables, plan.held,
                                       dtype is torch.bfloat16)
            if r.__class__ is tuple:
                return r
        name = "admmq_cache_read"
        self._check(plan, name)
        _need(dtype in (torch.bfloat16, torch.float32), name + ": bf16 or fp32")
        shape = (plan.n_rows, self.kv_heads, self.head_dim)
        k, v = [torch.empty(shape, dtype=dtype, device=self.device) if x is None else x for x in (k, v)]
        sk, sv = self._strides(k, self.kv_heads, dtype, plan, name + " k"), self._strides(v, self.kv_heads, dtype, plan, name + " v")
        adapt._call(_library().admmq_cache_read, name, self.index, self._ref, plan._ref, 1 if dtype is torch.bfloat16 else 0,
                    k.data_ptr(), *sk, v.data_ptr(), *sv, self._status)
        return k, v

    def attend(self, q: torch.Tensor, plan: CachePlan, scale: Optional[float] = None, window: int = 0,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """(out, lse): softmax attention of q [rows, kv_heads * group, head_dim] bf16 over what each row's request holds up
        to the row itself (written before), with window > 0 the last `window` positions of that (pages that no row sees may be gone
        from the tables); scale 1 / sqrt(head_dim) if not given.  out like q, lse [rows, heads] fp32 the logarithm of the sum of the weights' exponentials.  Rows of
        a request that takes no part get 0 and -inf."""
        if out is None and lse is None and plan.__class__ is CachePlan:
            r = adapt._fast.cache_attend(self._status, self._ref, plan._ref, self.codes, self.scale, plan.tables, plan.held, q,
                                         self._softmax if scale is None else scale, window)
            if r.__class__ is tuple:
                return r
        name = "admmq_cache_attend"
        self._check(plan, name)
        _no_graph(name, q)
        _need(0 <= window < 2 ** 31, name + ": a window of at least one position, or 0 for none")
        heads = self.kv_heads * plan.group
        sq = self._strides(q, heads, torch.bfloat16, plan, name + " q")
        if out is None:
            out = torch.empty(q.shape, dtype=q.dtype, device=self.device)
        so = self._strides(out, heads, torch.bfloat16, plan, name + " out")
        if lse is None:
            lse = torch.empty(plan.n_rows, heads, dtype=torch.float32, device=self.device)
        _need(lse.dtype is torch.float32 and lse.get_device() == self.index and lse.is_contiguous()
              and tuple(lse.shape) == (plan.n_rows, heads), f"{name}: contiguous fp32 lse [{plan.n_rows}, {heads}]", B.ERR_SHAPE)
        with torch.cuda.device(self.index):
            nbytes = _library().admmq_cache_attend_workspace(self._ref, plan._ref)
            work = torch.empty(max(16, nbytes), dtype=torch.uint8, device=self.device)
        adapt._call(_library().admmq_cache_attend, name, self.index, self._ref, plan._ref,
                    self._softmax if scale is None else float(scale), int(window), q.data_ptr(), *sq, out.data_ptr(), *so,
                    lse.data_ptr(), work.data_ptr(), nbytes, self._status)
        return out, lse
