"""Running and adapting quantized layers: the calls of admmq_adapt.h on torch tensors.

    layer = QuantLinear(codes, scale, zero, bits=4, group_size=128)      # what Solver.quantize_layer returned
    bank = AdapterBank(down, up, scale)                                  # low-rank adapters of many requests
    plan = RequestPlan(lengths, adapters, bank.n_adapters)               # which rows belong to which adapter
    y, h = layer.forward(x, bank, plan)
    kept = Checkpoint.save(x)                                            # 8 bits a value until the backward pass
    dx, u = layer.grad_input(dy, bank, plan)
    d_down, d_up = adapter_grads(bank, plan, kept, h, dy, u)
    q, k = qk_norm_rope(q, k, wq, wk, cos, sin, positions, eps)

torch is used for device memory and streams only; every step runs in the library's kernels, on the current stream of
the tensors' device.  Argument errors raise AdmmqError before anything is enqueued; errors met on the device are kept in
a status word, which `check_device_status` reads (it synchronises) and clears.
"""
from __future__ import annotations

import contextlib
import ctypes as C
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


class AdapterGradArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("d_in", C.c_int), ("d_out", C.c_int), ("n_adapters", C.c_int),
                ("rank", C.c_int), ("n_rows", C.c_longlong), ("d_order", C.c_void_p), ("d_offsets", C.c_void_p),
                ("d_h", C.c_void_p), ("d_u", C.c_void_p), ("d_x", C.c_void_p), ("ldx", C.c_longlong),
                ("d_x_codes", C.c_void_p), ("d_x_scale", C.c_void_p), ("d_dy", C.c_void_p), ("lddy", C.c_longlong),
                ("d_grad_down", C.c_void_p), ("d_grad_up", C.c_void_p)]


class QkArgs(C.Structure):
    _fields_ = [("struct_size", C.c_size_t), ("dtype", C.c_int), ("q_heads", C.c_int), ("k_heads", C.c_int),
                ("head_dim", C.c_int), ("rot_dim", C.c_int), ("n_rows", C.c_longlong), ("eps", C.c_double),
                ("d_q", C.c_void_p), ("d_k", C.c_void_p), ("q_row", C.c_longlong), ("q_head", C.c_longlong),
                ("k_row", C.c_longlong), ("k_head", C.c_longlong), ("d_wq", C.c_void_p), ("d_wk", C.c_void_p),
                ("d_cos", C.c_void_p), ("d_sin", C.c_void_p), ("n_positions", C.c_longlong), ("d_pos", C.c_void_p),
                ("d_out_q", C.c_void_p), ("d_out_k", C.c_void_p), ("out_q_row", C.c_longlong),
                ("out_q_head", C.c_longlong), ("out_k_row", C.c_longlong), ("out_k_head", C.c_longlong),
                ("d_dy_q", C.c_void_p), ("d_dy_k", C.c_void_p), ("dy_q_row", C.c_longlong),
                ("dy_q_head", C.c_longlong), ("dy_k_row", C.c_longlong), ("dy_k_head", C.c_longlong),
                ("d_grad_wq", C.c_void_p), ("d_grad_wk", C.c_void_p), ("d_workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t), ("d_status", C.c_void_p)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = B.load_library()
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
        _lib = lib
    return _lib


def _need(ok: bool, what: str, status: int = B.ERR_INVALID_ARG):
    if not ok:
        raise AdmmqError(status, what)


def _check(st: int, where: str):
    if st != B.OK:
        raise AdmmqError(st, where)


def _on(device: torch.device):
    """The device made current for a call, as the library asks (a no-op when it is)."""
    if device.index == torch.cuda.current_device():
        return contextlib.nullcontext()
    return torch.cuda.device(device)


def _stream(device: torch.device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


_status_words: dict = {}


def _status(device: torch.device) -> int:
    """Pointer of the device's status word, made (zeroed) at its first use."""
    w = _status_words.get(device)
    if w is None:
        w = torch.zeros(4, dtype=torch.int32, device=device)
        torch.cuda.synchronize(device)
        w = _status_words[device] = (w, w.data_ptr())
    return w[1]


def check_device_status(device: Union[str, torch.device] = "cuda:0", where: str = "device status"):
    """Waits for the device, raises AdmmqError for the first error that a call of this module met on it, and clears it."""
    device = torch.device(device)
    _status(device)
    word = _status_words[device][0]
    torch.cuda.synchronize(device)
    st = int(word[0].item())
    if st != B.OK:
        word.zero_()
        torch.cuda.synchronize(device)
        raise AdmmqError(st, where)


def _rows(t: torch.Tensor, width: int, device: torch.device, name: str):
    _need(t.dim() == 2 and t.dtype == torch.bfloat16 and t.device == device,
          f"{name}: a [rows, {width}] bf16 tensor on {device}")
    _need(t.shape[1] == width and (t.shape[0] == 0 or t.stride(1) == 1), f"{name}: rows of {width} adjacent values",
          B.ERR_SHAPE)


def _ld(t: torch.Tensor) -> int:
    """Row stride in elements; that of a single row does not matter, and torch may give it any value."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


class AdapterBank:
    """Low-rank adapters of one layer: adapter a adds scale[a] * up[a]^T (down[a] x).

    down [n, rank, d_in] and up [n, rank, d_out] bf16 (both rank-major), scale [n] fp32; the tensors are used in place,
    so a bank sees what an optimizer writes into them.  check: reads the bank once and raises if an entry is not
    finite (rows of different requests share tensor-core tiles; call `check` again after loading other values)."""

    def __init__(self, down: torch.Tensor, up: torch.Tensor, scale: torch.Tensor, check: bool = True):
        _need(down.dim() == 3 and up.dim() == 3 and down.shape[:2] == up.shape[:2], "AdapterBank: down [n, r, d_in], "
              "up [n, r, d_out]", B.ERR_SHAPE)
        _need(scale.shape == (down.shape[0],), "AdapterBank: one scale an adapter", B.ERR_SHAPE)
        _need(down.dtype == up.dtype == torch.bfloat16 and scale.dtype == torch.float32 and down.is_cuda
              and up.device == scale.device == down.device, "AdapterBank: bf16 down and up, fp32 scale, one device")
        _need(down.is_contiguous() and up.is_contiguous() and scale.is_contiguous(), "AdapterBank: contiguous tensors")
        self.down, self.up, self.scale, self.device = down, up, scale, down.device
        self.n_adapters, self.rank, self.d_in = down.shape
        self.d_out = up.shape[2]
        self._c = Adapters(C.sizeof(Adapters), self.n_adapters, self.rank, down.data_ptr(), up.data_ptr(),
                           scale.data_ptr())
        self._ref = C.addressof(self._c)
        if check:
            self.check()

    def check(self):
        with _on(self.device):
            _check(_library().admmq_adapters_check(self._ref, self.d_in, self.d_out, _status(self.device),
                                                   _stream(self.device)), "admmq_adapters_check")
        check_device_status(self.device, "admmq_adapters_check")


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
        _need(x.dim() == 2 and x.is_cuda and x.dtype in (torch.float32, torch.bfloat16),
              "Checkpoint.save: [rows, width] fp32 or bf16 on a GPU")
        t, n = x.shape
        _need(t == 0 or x.stride(1) == 1, "Checkpoint.save: adjacent values", B.ERR_SHAPE)
        codes = torch.empty(t, n, dtype=torch.int8, device=x.device)
        scale = torch.empty(t, -(-n // BLOCK), dtype=torch.float32, device=x.device)
        with _on(x.device):
            _check(_library().admmq_checkpoint_save(x.data_ptr(), B.BF16 if x.dtype == torch.bfloat16 else B.F32, t, n,
                                                    _ld(x), codes.data_ptr(), scale.data_ptr(), _stream(x.device)),
                   "admmq_checkpoint_save")
        return cls(codes, scale)

    def restore(self, dtype: torch.dtype = torch.bfloat16, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        _need(dtype in (torch.float32, torch.bfloat16), "Checkpoint.restore: fp32 or bf16")
        t, n = self.codes.shape
        if out is None:
            out = torch.empty(t, n, dtype=dtype, device=self.device)
        else:
            _need(out.dtype == dtype and out.device == self.device and tuple(out.shape) == (t, n)
                  and (t == 0 or out.stride(1) == 1), "Checkpoint.restore: out [rows, width]", B.ERR_SHAPE)
        with _on(self.device):
            _check(_library().admmq_checkpoint_restore(self.codes.data_ptr(), self.scale.data_ptr(), t, n,
                                                       out.data_ptr(), B.BF16 if dtype == torch.bfloat16 else B.F32,
                                                       _ld(out), _stream(self.device)), "admmq_checkpoint_restore")
        return out


class QuantLinear:
    """A quantized layer laid out for multiplication: codes [d_out, d_in] uint8 below 2^bits (bits 2..4), scale and
    zero [d_out, groups] fp32 as Solver.quantize_layer and Solver.local_search return them.  The codes are packed once,
    4 bits each; the arguments are not kept."""

    def __init__(self, codes: torch.Tensor, scale: torch.Tensor, zero: torch.Tensor, bits: int, group_size: int = 0):
        _need(codes.dim() == 2 and codes.dtype == torch.uint8 and codes.is_cuda and codes.is_contiguous(),
              "QuantLinear: contiguous uint8 codes [d_out, d_in]")
        self.d_out, self.d_in = codes.shape
        self.bits, self.group_size, self.device = bits, group_size, codes.device
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
        with _on(self.device):
            _check(lib.admmq_pack_layer(codes.data_ptr(), scale.data_ptr(), zero.data_ptr(), self.d_in, self.d_out,
                                        bits, group_size, self.packed.data_ptr(), self.grid.data_ptr(),
                                        _status(self.device), _stream(self.device)), "admmq_pack_layer")
        check_device_status(self.device, "admmq_pack_layer")
        self._c = PackedLayer(C.sizeof(PackedLayer), self.d_in, self.d_out, group_size, self.packed.data_ptr(),
                              self.grid.data_ptr())
        self._ref = C.addressof(self._c)

    def _run(self, fn, name, x, k, m, bank, plan, out, factor):
        dev = self.device
        _rows(x, k, dev, name)
        t = x.shape[0]
        if out is None:
            out = torch.empty(t, m, dtype=torch.bfloat16, device=dev)
        else:
            _rows(out, m, dev, name + " out")
            _need(out.shape[0] == t, name + ": out has other rows", B.ERR_SHAPE)
        ref = row_ptr = f_ptr = None
        if bank is not None:
            _need(plan is not None and plan.n_rows == t, name + ": a plan of these rows goes with a bank", B.ERR_SHAPE)
            _need(bank.d_in == self.d_in and bank.d_out == self.d_out and plan.n_adapters == bank.n_adapters,
                  name + ": bank, plan and layer differ", B.ERR_SHAPE)
            _need(bank.device == dev and plan.device == dev, name + ": bank and plan on the layer's device")
            if factor is None:
                factor = torch.empty(t, bank.rank, dtype=torch.float32, device=dev)
            else:
                _need(factor.dtype == torch.float32 and factor.is_contiguous() and factor.device == dev
                      and tuple(factor.shape) == (t, bank.rank), name + ": factor [rows, rank] fp32", B.ERR_SHAPE)
            ref, row_ptr, f_ptr = bank._ref, plan._ptr[0], factor.data_ptr()
        with _on(dev):
            _check(fn(self._ref, ref, t, row_ptr, x.data_ptr(), _ld(x), out.data_ptr(), _ld(out), f_ptr, _status(dev),
                      _stream(dev)), name)
        return out, factor

    def forward(self, x: torch.Tensor, bank: Optional[AdapterBank] = None, plan: Optional[RequestPlan] = None,
                out: Optional[torch.Tensor] = None, h: Optional[torch.Tensor] = None):
        """(y, h):  y_t = W x_t + up_a^T h_t,  h_t = scale_a down_a x_t (None without a bank).  x [rows, d_in] bf16."""
        return self._run(_library().admmq_linear_forward, "admmq_linear_forward", x, self.d_in, self.d_out, bank, plan,
                         out, h)

    def grad_input(self, dy: torch.Tensor, bank: Optional[AdapterBank] = None, plan: Optional[RequestPlan] = None,
                   out: Optional[torch.Tensor] = None, u: Optional[torch.Tensor] = None):
        """(dx, u):  dx_t = W^T dy_t + down_a^T u_t,  u_t = scale_a up_a dy_t (None without a bank)."""
        return self._run(_library().admmq_linear_grad_input, "admmq_linear_grad_input", dy, self.d_out, self.d_in, bank,
                         plan, out, u)


def adapter_grads(bank: AdapterBank, plan: RequestPlan, x: Union[Checkpoint, torch.Tensor], h: torch.Tensor,
                  dy: torch.Tensor, u: torch.Tensor, grad_down: Optional[torch.Tensor] = None,
                  grad_up: Optional[torch.Tensor] = None):
    """(d_down, d_up), bf16 in the bank's layout: sums over an adapter's rows of u_t x_t^T and h_t dy_t^T.  x: the
    layer's input in bf16, or its Checkpoint.  An adapter without rows gets zeros."""
    dev, name = bank.device, "admmq_adapter_grad"
    t, r = plan.n_rows, bank.rank
    _need(plan.n_adapters == bank.n_adapters, name + ": bank and plan differ", B.ERR_SHAPE)
    _need(plan.device == dev and x.device == dev, name + ": one device")
    for f in (h, u):
        _need(f.dtype == torch.float32 and f.is_contiguous() and f.device == dev, name + ": contiguous fp32 h and u")
        _need(tuple(f.shape) == (t, r), name + ": h and u [rows, rank]", B.ERR_SHAPE)
    _rows(dy, bank.d_out, dev, name + " dy")
    _need(dy.shape[0] == t and tuple(x.shape) == (t, bank.d_in), name + ": x and dy of the plan's rows", B.ERR_SHAPE)
    kept = isinstance(x, Checkpoint)
    if not kept:
        _rows(x, bank.d_in, dev, name + " x")
    out = []
    for g, like in ((grad_down, bank.down), (grad_up, bank.up)):
        if g is None:
            g = torch.empty_like(like)
        else:
            _need(g.dtype == torch.bfloat16 and g.is_contiguous() and g.device == dev and g.shape == like.shape,
                  name + ": gradients of the bank's layout", B.ERR_SHAPE)
        out.append(g)
    args = AdapterGradArgs(C.sizeof(AdapterGradArgs), bank.d_in, bank.d_out, bank.n_adapters, r, t, plan._ptr[1],
                           plan._ptr[2], h.data_ptr(), u.data_ptr(), None if kept else x.data_ptr(),
                           0 if kept else _ld(x), x.codes.data_ptr() if kept else None,
                           x.scale.data_ptr() if kept else None, dy.data_ptr(), _ld(dy), out[0].data_ptr(),
                           out[1].data_ptr())
    with _on(dev):
        _check(_library().admmq_adapter_grad(C.addressof(args), _stream(dev)), name)
    return out[0], out[1]


def _qk(name, q, k, wq, wk, cos, sin, positions, eps, dq, dk, out_q, out_k):
    dev, dt = q.device, q.dtype
    _need(q.is_cuda and dt in (torch.float32, torch.bfloat16), name + ": fp32 or bf16 on a GPU")
    _need(q.dim() == 3 and k.dim() == 3 and k.shape[0] == q.shape[0] and k.shape[2] == q.shape[2],
          name + ": q [rows, heads, dim], k [rows, heads, dim]", B.ERR_SHAPE)
    t, hq, d = q.shape
    hk = k.shape[1]
    for x, h in ((q, hq), (k, hk), (dq, hq), (dk, hk), (out_q, hq), (out_k, hk)):
        if x is None:
            continue
        _need(x.dtype == dt and x.device == dev, name + ": one type, one device")
        _need(tuple(x.shape) == (t, h, d) and (x.numel() == 0 or x.stride(2) == 1),
              name + ": [rows, heads, dim] with adjacent values", B.ERR_SHAPE)
    for w in (wq, wk):
        _need(w.dtype == dt and w.device == dev and w.is_contiguous(), name + ": weights of q's type")
        _need(tuple(w.shape) == (d,), name + ": weights [dim]", B.ERR_SHAPE)
    _need(cos.dtype == sin.dtype == torch.float32 and cos.device == sin.device == dev and cos.is_contiguous()
          and sin.is_contiguous(), name + ": contiguous fp32 cos and sin")
    _need(cos.dim() == 2 and cos.shape == sin.shape, name + ": cos and sin [positions, rot / 2]", B.ERR_SHAPE)
    _need(positions.dtype == torch.int32 and positions.device == dev and positions.is_contiguous(),
          name + ": int32 positions")
    _need(tuple(positions.shape) == (t,), name + ": a position a row", B.ERR_SHAPE)
    if out_q is None:
        out_q = torch.empty(t, hq, d, dtype=dt, device=dev)
    if out_k is None:
        out_k = torch.empty(t, hk, d, dtype=dt, device=dev)
    args = QkArgs(C.sizeof(QkArgs), B.BF16 if dt == torch.bfloat16 else B.F32, hq, hk, d, 2 * cos.shape[1], t, eps,
                  q.data_ptr(), k.data_ptr(), q.stride(0), q.stride(1), k.stride(0), k.stride(1), wq.data_ptr(),
                  wk.data_ptr(), cos.data_ptr(), sin.data_ptr(), cos.shape[0], positions.data_ptr(),
                  out_q.data_ptr(), out_k.data_ptr(), out_q.stride(0), out_q.stride(1), out_k.stride(0),
                  out_k.stride(1))
    args.d_status = _status(dev)
    if dq is None:
        with _on(dev):
            _check(_library().admmq_qk_norm_rope(C.addressof(args), _stream(dev)), name)
        return out_q, out_k
    gw = torch.empty(2, d, dtype=dt, device=dev)
    args.d_dy_q, args.d_dy_k = dq.data_ptr(), dk.data_ptr()
    args.dy_q_row, args.dy_q_head, args.dy_k_row, args.dy_k_head = dq.stride(0), dq.stride(1), dk.stride(0), dk.stride(1)
    args.d_grad_wq, args.d_grad_wk = gw[0].data_ptr(), gw[1].data_ptr()
    args.workspace_bytes = _library().admmq_qk_workspace_bytes(d)
    work = torch.empty(max(16, args.workspace_bytes), dtype=torch.uint8, device=dev)
    args.d_workspace = work.data_ptr()
    with _on(dev):
        _check(_library().admmq_qk_norm_rope_backward(C.addressof(args), _stream(dev)), name)
    return out_q, out_k, gw[0], gw[1]


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, wq: torch.Tensor, wk: torch.Tensor, cos: torch.Tensor,
                 sin: torch.Tensor, positions: torch.Tensor, eps: float = 1e-6, out_q: Optional[torch.Tensor] = None,
                 out_k: Optional[torch.Tensor] = None):
    """(q', k'): every head normed by its root mean square, weighted, and its first rot values rotated by the row's
    position (pairs i, i + rot / 2).  q [rows, heads, dim] and k [rows, kv heads, dim] may be views into one buffer;
    cos, sin [positions, rot / 2] fp32; positions [rows] int32.  out_q, out_k may be q and k themselves."""
    return _qk("admmq_qk_norm_rope", q, k, wq, wk, cos, sin, positions, eps, None, None, out_q, out_k)


def qk_norm_rope_backward(q: torch.Tensor, k: torch.Tensor, wq: torch.Tensor, wk: torch.Tensor, cos: torch.Tensor,
                          sin: torch.Tensor, positions: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                          eps: float = 1e-6, out_q: Optional[torch.Tensor] = None,
                          out_k: Optional[torch.Tensor] = None):
    """Gradients (q, k, wq, wk) of qk_norm_rope from those of its results, with its inputs (before the norm)."""
    return _qk("admmq_qk_norm_rope_backward", q, k, wq, wk, cos, sin, positions, eps, dq, dk, out_q, out_k)
