"""Running and adapting quantized layers: the calls of admmq_adapt.h on torch tensors.

    layer = QuantLinear(codes, scale, zero, bits=4, group_size=128)      # what Solver.quantize_layer returned
    bank = AdapterBank(down, up, scale)                                  # low-rank adapters of many requests
    plan = RequestPlan(lengths, adapters, bank.n_adapters)               # which rows belong to which adapter
    y, h = layer.forward(x, bank, plan)
    kept = Checkpoint.save(x)                                            # 8 bits a value until the backward pass
    dx, u = layer.grad_input(dy, bank, plan)
    d_down, d_up = adapter_grads(bank, plan, kept, h, dy, u)
    q, k = qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps)

The common forms of the calls (new outputs, no conversion) go through the extension _adapt.so; the others, and every
call that fails, take the path written here, which names what is wrong.

torch is used for device memory and streams only; every step runs in the library's kernels, on the current stream of
the tensors' device.  Argument errors raise AdmmqError before anything is enqueued; errors met on the device by the calls
that return at once are kept in a status word, one a device, which `check_device_status` reads (it synchronises) and clears.
What QuantLinear and AdapterBank check of their arguments on the device they wait for, and raise, themselves.

No call records an autograd graph: the gradients have calls of their own.  QuantLinear.forward and qk_norm_rope refuse an
x, q or k that requires grad while grad mode is on, where a graph would end without a word; call them in torch.no_grad(),
from a torch.autograd.Function, or with detached tensors.  (Adapters and norm weights may require grad: whoever trains them
puts what adapter_grads and qk_norm_rope_backward return into their .grad.)
"""
from __future__ import annotations

import ctypes as C
import os
import struct
import threading
from typing import Optional, Sequence, Union

import numpy as np
import torch

from . import binding as B
from .binding import AdmmqError

BLOCK = 128                       # channels that share a scale of an 8-bit checkpoint


class PackedLayer(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("d_in", C.c_int), ("d_out", C.c_int), ("group_size", C.c_int),
                ("d_packed", C.c_void_p), ("d_grid", C.c_void_p)]


class Adapters(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("n_adapters", C.c_int), ("rank", C.c_int), ("d_down", C.c_void_p),
                ("d_up", C.c_void_p), ("d_scale", C.c_void_p)]


# The two larger argument structs are packed by format in one step, in native layout: filling a ctypes structure field by
# field takes longer than the launch that it describes.
_GRAD_ARGS = struct.Struct("@N4iq5Pq3Pq2P")       # admmq_adapter_grad_args
_GRAD_ARGS_BYTES = _GRAD_ARGS.size
_QK_ARGS = struct.Struct("@N5iqd2P4q4PqP2P4q2P4q3PNP")   # admmq_qk_args
_QK_ARGS_BYTES = _QK_ARGS.size


_lib = None
_fast = None                      # _adapt.so: the common forms of the calls in one step each


def _library():
    global _lib, _fast
    if _lib is None:
        lib = B.load_library()
        if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_adapt.so")):
            raise FileNotFoundError("_adapt.so not found: build it with `python -m paper_2605_11222_b200.build`")
        from . import _adapt
        _fast = _adapt
        vp, ci, cll = C.c_void_p, C.c_int, C.c_longlong
        lib.admmq_packed_bytes.restype = lib.admmq_grid_bytes.restype = C.c_size_t
        lib.admmq_qk_workspace_bytes.restype = C.c_size_t
        lib.admmq_packed_bytes.argtypes = [ci, ci]
        lib.admmq_grid_bytes.argtypes = [ci, ci, ci]
        lib.admmq_qk_workspace_bytes.argtypes = [ci]
        lib.admmq_pack_layer.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, vp]
        lib.admmq_adapters_check.argtypes = [vp, ci, ci, vp, vp]
        lib.admmq_linear_forward.argtypes = [vp, vp, cll, vp, vp, cll, vp, cll, vp, vp, vp]
        lib.admmq_linear_grad_input.argtypes = [vp, vp, cll, vp, vp, cll, vp, cll, vp, vp, vp]
        lib.admmq_adapter_grad.argtypes = [vp, vp]
        lib.admmq_checkpoint_save.argtypes = [vp, ci, cll, ci, cll, vp, vp, vp]
        lib.admmq_checkpoint_restore.argtypes = [vp, vp, cll, ci, vp, ci, cll, vp]
        lib.admmq_qk_norm_rope.argtypes = [vp, vp]
        lib.admmq_qk_norm_rope_backward.argtypes = [vp, vp]
        lib.admmq_test_linear_set_wait.argtypes = [cll, ci]
        lib.admmq_test_warp_wait.argtypes = [cll, cll, vp, vp, vp]
        lib.admmq_test_pair_rings.restype, lib.admmq_test_pair_rings.argtypes = None, [vp] * 5
        _lib = lib
    return _lib


def _need(ok: bool, what: str, status: int = B.ERR_INVALID_ARG):
    if not ok:
        raise AdmmqError(status, what)


def _call(fn, where: str, index: int, *args):
    """fn(*args, stream) with device `index` current, as the library asks, on that device's current stream."""
    if _current_device() == index:
        st = fn(*args, _current_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _current_stream(index))
    if st != 0:
        raise AdmmqError(st, where)


# The device and the stream as plain integers: these are on the path of every decoded token.
_current_device = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device
_current_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


_status_words: dict = {}
_status_lock = threading.Lock()


def _status(index: int) -> int:
    """Pointer of a device's status word, made (zeroed) at its first use and kept for good."""
    w = _status_words.get(index)
    if w is None:
        with _status_lock:                       # one word, whichever threads come first: kernels keep its pointer
            w = _status_words.get(index)
            if w is None:
                with torch.inference_mode(False):    # (cleared in place later, in whatever mode)
                    word = torch.zeros(4, dtype=torch.int32, device=f"cuda:{index}")
                torch.cuda.synchronize(index)
                w = _status_words[index] = (word.data_ptr(), word)
    return w[0]


def _call_and_wait(fn, where: str, index: int, *args):
    """fn(*args, status word, stream) with a word of its own, waited for: its error is not another call's, nor taken by
    one."""
    word = torch.zeros(1, dtype=torch.int32, device=f"cuda:{index}")
    _call(fn, where, index, *args, word.data_ptr())
    st = int(word.item())
    if st != B.OK:
        raise AdmmqError(st, where)


def check_device_status(device: Union[str, torch.device] = "cuda:0", where: str = "device status"):
    """Waits for the device, raises AdmmqError for the first error that a call of this module met on it, and clears it."""
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    _status(index)
    word = _status_words[index][1]
    torch.cuda.synchronize(index)
    with _status_lock:                           # (an error that is there stays until it is cleared here)
        st = int(word[0].item())
        if st != B.OK:
            word.zero_()
            torch.cuda.synchronize(index)
    if st != B.OK:
        raise AdmmqError(st, where)


def _fail(status: int, what: str):
    raise AdmmqError(status, what)


def _no_graph(name: str, *inputs: torch.Tensor):
    if torch.is_grad_enabled() and any(t.requires_grad for t in inputs):
        _fail(B.ERR_INVALID_ARG, f"{name}: an input requires grad, and the call records no graph (use torch.no_grad() or "
              "detach(), and the call that forms the gradient)")


def _rows(t: torch.Tensor, width: int, index: int, name: str) -> int:
    """Checks a [rows, width] bf16 tensor on device `index`, returns its row stride.  (The stride of a single row does
    not matter, and torch may give it any value.)"""
    if t.dim() != 2 or t.dtype is not torch.bfloat16 or t.get_device() != index:
        _fail(B.ERR_INVALID_ARG, f"{name}: a [rows, {width}] bf16 tensor on cuda:{index}")
    rows, w = t.shape
    ld, inner = t.stride()
    if w != width or (rows > 0 and inner != 1):
        _fail(B.ERR_SHAPE, f"{name}: rows of {width} adjacent values")
    return ld if rows > 1 else w


def _ld(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


class AdapterBank:
    """Low-rank adapters of one layer: adapter a adds scale[a] * up[a]^T (down[a] x).

    down [n, rank, d_in] and up [n, rank, d_out] bf16 (both rank-major), scale [n] fp32; the tensors are used in place,
    so a bank sees what an optimizer writes into them; one whose storage is replaced (`t.data = ...`, a module moved) needs a
    new bank, and calls with the old one are refused.  check: reads the bank once and raises if an entry is not
    finite (rows of different requests share tensor-core tiles; call `check` again after loading other values)."""

    def __init__(self, down: torch.Tensor, up: torch.Tensor, scale: torch.Tensor, check: bool = True):
        _need(down.dim() == 3 and up.dim() == 3 and down.shape[:2] == up.shape[:2], "AdapterBank: down [n, r, d_in], "
              "up [n, r, d_out]", B.ERR_SHAPE)
        _need(scale.shape == (down.shape[0],), "AdapterBank: one scale an adapter", B.ERR_SHAPE)
        _need(down.dtype == up.dtype == torch.bfloat16 and scale.dtype == torch.float32 and down.is_cuda
              and up.device == scale.device == down.device, "AdapterBank: bf16 down and up, fp32 scale, one device")
        _need(down.is_contiguous() and up.is_contiguous() and scale.is_contiguous(), "AdapterBank: contiguous tensors")
        self.down, self.up, self.scale, self.device = down, up, scale, down.device
        self.index = down.get_device()
        self.n_adapters, self.rank, self.d_in = down.shape
        self.d_out = up.shape[2]
        self._fits = (self.d_in, self.d_out, self.index, self.n_adapters)
        self._c = Adapters(C.sizeof(Adapters), self.n_adapters, self.rank, down.data_ptr(), up.data_ptr(),
                           scale.data_ptr())
        self._ref = C.addressof(self._c)
        if check:
            self.check()

    def _in_place(self, name: str):
        c = self._c
        if (self.down.data_ptr(), self.up.data_ptr(), self.scale.data_ptr()) != (c.d_down, c.d_up, c.d_scale):
            _fail(B.ERR_INVALID_ARG, name + ": a tensor of the bank has other storage than when the bank was made")

    def check(self):
        self._in_place("admmq_adapters_check")
        _call_and_wait(_library().admmq_adapters_check, "admmq_adapters_check", self.index, self._ref, self.d_in, self.d_out)


class RequestPlan:
    """The rows of a batch: request i has lengths[i] adjacent rows and adapter adapters[i] (-1: none).

    Built on the host and copied once; `row_adapter` [rows], and for the gradients `order` (rows sorted by adapter) and
    `offsets` [n_adapters + 1], all int32 on the device."""

    def __init__(self, lengths: Sequence[int], adapters: Sequence[int], n_adapters: int, device="cuda"):
        lengths = np.asarray(lengths, dtype=np.int64).reshape(-1)
        adapters = np.asarray(adapters, dtype=np.int64).reshape(-1)
        _need(lengths.shape == adapters.shape, "RequestPlan: one adapter a request", B.ERR_SHAPE)
        _need(n_adapters >= 0 and bool((lengths >= 0).all()), "RequestPlan: negative length", B.ERR_SHAPE)
        _need(bool(((adapters >= -1) & (adapters < n_adapters)).all()), "RequestPlan: no such adapter")
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.n_rows, self.n_adapters, self.device = int(lengths.sum()), n_adapters, device
        self.index = device.index
        _need(self.n_rows < 2 ** 30, "RequestPlan: too many rows", B.ERR_SHAPE)
        rows = np.repeat(adapters, lengths)
        order = np.argsort(rows, kind="stable")
        counts = np.bincount(rows + 1, minlength=n_adapters + 1)
        none = int(counts[0])
        pad = -self.n_rows % 4
        host = np.zeros(2 * (self.n_rows + pad) + n_adapters + 1, dtype=np.int32)
        at = self.n_rows + pad
        host[:self.n_rows] = rows
        host[at: at + self.n_rows - none] = order[none:]
        host[2 * at + 1:] = np.cumsum(counts[1: n_adapters + 1])
        buf = torch.from_numpy(host).to(device)
        self.row_adapter, self.order, self.offsets = buf[:self.n_rows], buf[at: at + self.n_rows], buf[2 * at:]
        self._ptr = tuple(buf.data_ptr() + 4 * o for o in (0, at, 2 * at))


class Checkpoint:
    """Activations kept in 8 bits: codes [rows, width] int8 and scale [rows, ceil(width / 128)] fp32, with
    scale = max |x| / 127 over 128 channels and code = round(x / scale)."""

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor):
        _need(codes.dim() == 2 and codes.dtype == torch.int8 and codes.is_cuda and codes.is_contiguous(),
              "Checkpoint: contiguous int8 codes [rows, width]")
        _need(scale.dtype == torch.float32 and scale.device == codes.device and scale.is_contiguous(),
              "Checkpoint: contiguous fp32 scales")
        _need(tuple(scale.shape) == (codes.shape[0], -(-codes.shape[1] // BLOCK)), "Checkpoint: one scale for 128 "
              "channels of a row", B.ERR_SHAPE)
        self.codes, self.scale = codes, scale

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    @classmethod
    def save(cls, x: torch.Tensor) -> "Checkpoint":
        if _lib is None:
            _library()
        r = _fast.checkpoint_save(x)
        if r.__class__ is tuple:
            self = cls.__new__(cls)
            self.codes, self.scale = r
            return self
        bf16 = x.dtype is torch.bfloat16
        if x.dim() != 2 or not x.is_cuda or not (bf16 or x.dtype is torch.float32):
            _fail(B.ERR_INVALID_ARG, "Checkpoint.save: [rows, width] fp32 or bf16 on a GPU")
        t, n = x.shape
        ld, inner = x.stride()
        if t > 0 and inner != 1:
            _fail(B.ERR_SHAPE, "Checkpoint.save: adjacent values")
        self = cls.__new__(cls)
        self.codes = codes = x.new_empty((t, n), dtype=torch.int8)
        self.scale = scale = x.new_empty((t, -(-n // BLOCK)), dtype=torch.float32)
        _call((_lib or _library()).admmq_checkpoint_save, "admmq_checkpoint_save", x.get_device(), x.data_ptr(),
              1 if bf16 else 0, t, n, ld if t > 1 else n, codes.data_ptr(), scale.data_ptr())
        return self

    def restore(self, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        codes = self.codes
        if out is None and (dtype is torch.bfloat16 or dtype is torch.float32):
            if _lib is None:
                _library()
            r = _fast.checkpoint_restore(codes, self.scale, dtype is torch.bfloat16)
            if r.__class__ is not int:
                return r
        if dtype is not torch.bfloat16 and dtype is not torch.float32:
            _fail(B.ERR_INVALID_ARG, "Checkpoint.restore: fp32 or bf16")
        t, n = codes.shape
        ld = n
        if out is None:
            out = codes.new_empty((t, n), dtype=dtype)
        else:
            _need(out.dtype == dtype and out.device == self.device and tuple(out.shape) == (t, n)
                  and (t == 0 or out.stride(1) == 1), "Checkpoint.restore: out [rows, width]", B.ERR_SHAPE)
            ld = _ld(out)
        _call((_lib or _library()).admmq_checkpoint_restore, "admmq_checkpoint_restore", codes.get_device(),
              codes.data_ptr(), self.scale.data_ptr(), t, n, out.data_ptr(), 1 if dtype is torch.bfloat16 else 0, ld)
        return out


class QuantLinear:
    """A quantized layer laid out for multiplication: codes [d_out, d_in] uint8 below 2^bits (bits 2..4), scale and
    zero [d_out, groups] fp32 as Solver.quantize_layer and Solver.local_search return them.  The codes are packed once,
    4 bits each; the arguments are not kept."""

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, zero: torch.Tensor, bits: int, group_size: int = 0):
        _need(codes.dim() == 2 and codes.dtype == torch.uint8 and codes.is_cuda and codes.is_contiguous(),
              "QuantLinear: contiguous uint8 codes [d_out, d_in]")
        self.d_out, self.d_in = codes.shape
        self.bits, self.group_size, self.device, self.index = bits, group_size, codes.device, codes.get_device()
        groups = 1 if group_size in (0, self.d_in) else self.d_in // max(1, group_size)
        for t in (scale, zero):
            _need(t.dtype == torch.float32 and t.device == codes.device and t.is_contiguous(),
                  "QuantLinear: contiguous fp32 scale and zero")
            _need(t.numel() == self.d_out * groups, "QuantLinear: one scale and zero a group", B.ERR_SHAPE)
        lib = _library()
        nb, ng = lib.admmq_packed_bytes(self.d_in, self.d_out), lib.admmq_grid_bytes(self.d_in, self.d_out, group_size)
        _need(nb > 0 and ng > 0, "QuantLinear: d_in and d_out multiples of 8, the group a multiple of 64", B.ERR_SHAPE)
        self.packed = torch.empty(nb, dtype=torch.uint8, device=self.device)
        self.grid = torch.empty(ng, dtype=torch.uint8, device=self.device)
        _call_and_wait(lib.admmq_pack_layer, "admmq_pack_layer", self.index, codes.data_ptr(), scale.data_ptr(),
                       zero.data_ptr(), self.d_in, self.d_out, bits, group_size, self.packed.data_ptr(),
                       self.grid.data_ptr())
        self._c = PackedLayer(C.sizeof(PackedLayer), self.d_in, self.d_out, group_size, self.packed.data_ptr(),
                              self.grid.data_ptr())
        self._ref, self._status = C.addressof(self._c), _status(self.index)

    def _quick(self, grad, x, bank, plan):
        """The call with new outputs; an int (a status) if the longer path has to say what is wrong."""
        if bank is None:
            return _fast.linear(grad, self._ref, self.d_in, self.d_out, self.index, self._status, x)
        if plan is None or bank._fits != (self.d_in, self.d_out, self.index, plan.n_adapters) or plan.index != self.index:
            return B.ERR_SHAPE
        return _fast.linear(grad, self._ref, self.d_in, self.d_out, self.index, self._status, x, bank._ref, bank.rank,
                            plan.n_rows, plan._ptr[0], bank.down, bank.up, bank.scale)

    def _run(self, fn, name, x, k, m, bank, plan, out, factor):
        index = self.index
        ldx = _rows(x, k, index, name)
        t = x.shape[0]
        if out is None:
            out, ldo = x.new_empty((t, m)), m
        else:
            ldo = _rows(out, m, index, name + " out")
            _need(out.shape[0] == t, name + ": out has other rows", B.ERR_SHAPE)
        if bank is None:
            _call(fn, name, index, self._ref, None, t, None, x.data_ptr(), ldx, out.data_ptr(), ldo, None,
                  _status(index))
            return out, None
        if plan is None or plan.n_rows != t:
            _fail(B.ERR_SHAPE, name + ": a plan of these rows goes with a bank")
        if bank.d_in != self.d_in or bank.d_out != self.d_out or plan.n_adapters != bank.n_adapters:
            _fail(B.ERR_SHAPE, name + ": bank, plan and layer differ")
        if bank.index != index or plan.index != index:
            _fail(B.ERR_INVALID_ARG, name + ": bank and plan on the layer's device")
        bank._in_place(name)
        if factor is None:
            factor = x.new_empty((t, bank.rank), dtype=torch.float32)
        else:
            _need(factor.dtype == torch.float32 and factor.is_contiguous() and factor.get_device() == index
                  and tuple(factor.shape) == (t, bank.rank), name + ": factor [rows, rank] fp32", B.ERR_SHAPE)
        _call(fn, name, index, self._ref, bank._ref, t, plan._ptr[0], x.data_ptr(), ldx, out.data_ptr(), ldo,
              factor.data_ptr(), _status(index))
        return out, factor

    def forward(self, x: torch.Tensor, bank: Optional[AdapterBank] = None, plan: Optional[RequestPlan] = None,
                out: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None):
        """(y, h):  y_t = W x_t + up_a^T h_t,  h_t = scale_a down_a x_t (None without a bank).  x [rows, d_in] bf16."""
        if out is None and h is None:
            r = self._quick(False, x, bank, plan)
            if r.__class__ is tuple:
                return r
        _no_graph("admmq_linear_forward", x)
        return self._run((_lib or _library()).admmq_linear_forward, "admmq_linear_forward", x, self.d_in, self.d_out, bank, plan,
                         out, h)

    def grad_input(self, dy: torch.Tensor, bank: Optional[AdapterBank] = None, plan: Optional[RequestPlan] = None,
                   out: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None):
        """(dx, u):  dx_t = W^T dy_t + down_a^T u_t,  u_t = scale_a up_a dy_t (None without a bank)."""
        if out is None and u is None:
            r = self._quick(True, dy, bank, plan)
            if r.__class__ is tuple:
                return r
        return self._run((_lib or _library()).admmq_linear_grad_input, "admmq_linear_grad_input", dy, self.d_out, self.d_in, bank,
                         plan, out, u)


def adapter_grads(bank: AdapterBank, plan: RequestPlan, x: Union[Checkpoint, torch.Tensor], h: torch.Tensor,
                  dy: torch.Tensor, u: torch.Tensor, grad_down: Optional[torch.Tensor] = None,
                  grad_up: Optional[torch.Tensor] = None):
    """(d_down, d_up), bf16 in the bank's layout: sums over an adapter's rows of u_t x_t^T and h_t dy_t^T.  x: the
    layer's input in bf16, or its Checkpoint.  An adapter without rows gets zeros."""
    if grad_down is None and grad_up is None and plan.n_adapters == bank.n_adapters and plan.index == bank.index:
        if _lib is None:
            _library()
        kept = x.__class__ is Checkpoint
        r = _fast.adapter_grad(bank.index, plan.n_rows, plan._ptr[1], plan._ptr[2], None if kept else x,
                               x.codes if kept else None, x.scale if kept else None, h, dy, u, bank.down, bank.up)
        if r.__class__ is tuple:
            return r
    index, name = bank.index, "admmq_adapter_grad"
    t, r = plan.n_rows, bank.rank
    if plan.n_adapters != bank.n_adapters:
        _fail(B.ERR_SHAPE, name + ": bank and plan differ")
    for f in (h, u):
        if f.dtype is not torch.float32 or not f.is_contiguous() or f.get_device() != index:
            _fail(B.ERR_INVALID_ARG, name + ": contiguous fp32 h and u")
        if f.shape != (t, r):
            _fail(B.ERR_SHAPE, name + ": h and u [rows, rank]")
    lddy = _rows(dy, bank.d_out, index, name + " dy")
    if dy.shape[0] != t or x.shape != (t, bank.d_in):
        _fail(B.ERR_SHAPE, name + ": x and dy of the plan's rows")
    if isinstance(x, Checkpoint):
        if plan.index != index or x.codes.get_device() != index:
            _fail(B.ERR_INVALID_ARG, name + ": one device")
        xp, ldx, codes, scale = 0, 0, x.codes.data_ptr(), x.scale.data_ptr()
    else:
        if plan.index != index:
            _fail(B.ERR_INVALID_ARG, name + ": one device")
        ldx = _rows(x, bank.d_in, index, name + " x")
        xp, codes, scale = x.data_ptr(), 0, 0
    out = []
    for g, like in ((grad_down, bank.down), (grad_up, bank.up)):
        if g is None:
            g = torch.empty_like(like)
        else:
            _need(g.dtype == torch.bfloat16 and g.is_contiguous() and g.device == like.device and g.shape == like.shape,
                  name + ": gradients of the bank's layout", B.ERR_SHAPE)
        out.append(g)
    args = _GRAD_ARGS.pack(_GRAD_ARGS_BYTES, bank.d_in, bank.d_out, bank.n_adapters, r, t, plan._ptr[1], plan._ptr[2],
                           h.data_ptr(), u.data_ptr(), xp, ldx, codes, scale, dy.data_ptr(), lddy, out[0].data_ptr(),
                           out[1].data_ptr())
    _call((_lib or _library()).admmq_adapter_grad, name, index, args)
    return out[0], out[1]


def _heads(x, t, h, d, dt, index, name):
    """Checks a [t, h, d] tensor, returns its row and head strides."""
    if x.dtype is not dt or x.get_device() != index:
        _fail(B.ERR_INVALID_ARG, name + ": one type, one device")
    if x.dim() != 3 or x.shape != (t, h, d):
        _fail(B.ERR_SHAPE, name + ": [rows, heads, dim]")
    row, head, inner = x.stride()
    if inner != 1 and x.numel() > 0:
        _fail(B.ERR_SHAPE, name + ": adjacent values of a head")
    return (row if t > 1 else 0), (head if h > 1 else 0)


def _qk(fn, name, q, k, wq, wk, cos, sin, positions, eps, dq, dk, out_q, out_k):
    if out_q is None and out_k is None and q.is_cuda:
        word = _status(q.get_device())
        r = _fast.qk(word, q, k, wq, wk, cos, sin, positions, eps) if dq is None else \
            _fast.qk(word, q, k, wq, wk, cos, sin, positions, eps, dq, dk)
        if r.__class__ is tuple:
            return r
    if dq is None:
        _no_graph(name, q, k)
    dt, index = q.dtype, q.get_device()
    bf16 = dt is torch.bfloat16
    if not q.is_cuda or not (bf16 or dt is torch.float32):
        _fail(B.ERR_INVALID_ARG, name + ": fp32 or bf16 on a GPU")
    if q.dim() != 3 or k.dim() != 3:
        _fail(B.ERR_SHAPE, name + ": q and k [rows, heads, dim]")
    t, hq, d = q.shape
    hk = k.shape[1]
    sq, sk = _heads(q, t, hq, d, dt, index, name), _heads(k, t, hk, d, dt, index, name)
    for w in (wq, wk):
        if w.dtype is not dt or w.get_device() != index or not w.is_contiguous():
            _fail(B.ERR_INVALID_ARG, name + ": weights of q's type")
        if w.shape != (d,):
            _fail(B.ERR_SHAPE, name + ": weights [dim]")
    for c in (cos, sin):
        if c.dtype is not torch.float32 or c.get_device() != index or not c.is_contiguous():
            _fail(B.ERR_INVALID_ARG, name + ": contiguous fp32 cos and sin")
    if cos.dim() != 2 or cos.shape != sin.shape:
        _fail(B.ERR_SHAPE, name + ": cos and sin [positions, rot / 2]")
    if positions.dtype is not torch.int32 or positions.get_device() != index or not positions.is_contiguous():
        _fail(B.ERR_INVALID_ARG, name + ": contiguous int32 positions")
    if positions.shape != (t,):
        _fail(B.ERR_SHAPE, name + ": a position a row")
    dense_q, dense_k = (hq * d, d), (hk * d, d)
    if out_q is None:
        out_q, oq = q.new_empty((t, hq, d)), dense_q
    else:
        oq = _heads(out_q, t, hq, d, dt, index, name)
    if out_k is None:
        out_k, ok = k.new_empty((t, hk, d)), dense_k
    else:
        ok = _heads(out_k, t, hk, d, dt, index, name)
    gw = None
    back = (0,) * 10
    if dq is not None:
        gq, gk = _heads(dq, t, hq, d, dt, index, name), _heads(dk, t, hk, d, dt, index, name)
        gw = q.new_empty((2, d))
        nbytes = _lib.admmq_qk_workspace_bytes(d)
        work = torch.empty(max(16, nbytes), dtype=torch.uint8, device=q.device)
        at = gw.data_ptr()
        back = (dq.data_ptr(), dk.data_ptr(), *gq, *gk, at, at + d * gw.element_size(), work.data_ptr(), nbytes)
    args = _QK_ARGS.pack(_QK_ARGS_BYTES, 1 if bf16 else 0, hq, hk, d, 2 * cos.shape[1], t, eps, q.data_ptr(),
                         k.data_ptr(), *sq, *sk, wq.data_ptr(), wk.data_ptr(), cos.data_ptr(), sin.data_ptr(),
                         cos.shape[0], positions.data_ptr(), out_q.data_ptr(), out_k.data_ptr(), *oq, *ok, *back,
                         _status(index))
    _call(fn, name, index, args)
    return (out_q, out_k) if gw is None else (out_q, out_k, gw[0], gw[1])


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, wq: torch.Tensor, wk: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, eps: float = 1e-6, out_q: Optional[torch.Tensor] = None,
                 out_k: Optional[torch.Tensor] = None):
    """(q', k'): every head normed by its root mean square, weighted, and its first rot values rotated by the row's
    position (pairs i, i + rot / 2).  q [rows, heads, dim] and k [rows, kv heads, dim] may be views into one buffer;
    cos, sin [positions, rot / 2] fp32; positions [rows] int32.  out_q, out_k may be q and k themselves."""
    return _qk((_lib or _library()).admmq_qk_norm_rope, "admmq_qk_norm_rope", q, k, wq, wk, cos, sin, positions, eps,
               None, None, out_q, out_k)


def qk_norm_rope_backward(q: torch.Tensor, k: torch.Tensor, wq: torch.Tensor, wk: torch.Tensor, cos: torch.Tensor,
                          sin: torch.Tensor, positions: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                          eps: float = 1e-6, out_q: Optional[torch.Tensor] = None,
                          out_k: Optional[torch.Tensor] = None):
    """Gradients (q, k, wq, wk) of qk_norm_rope from those of its results, with its inputs (before the norm)."""
    return _qk((_lib or _library()).admmq_qk_norm_rope_backward, "admmq_qk_norm_rope_backward", q, k, wq, wk, cos, sin,
               positions, eps, dq, dk, out_q, out_k)
