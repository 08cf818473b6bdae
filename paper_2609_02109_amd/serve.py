"""The operators of a served model's 4-bit and 8-bit variants, over the C ABI.

The options that a search chooses from are variants (16-bit or 4-bit) and
runtime parameters of the co-running models.  These are the operators of the
step that a 4-bit option stands for, to run it or to profile it into an option
table: products with 4-bit weights (`W4Weight`), and a paged key/value cache
held in 4 bits (`KV4Cache`) with its append, which turns keys and queries by
their positions on the way, and its attention.  Between the two variants is one
in 8 bits: products of 8-bit rows with 8-bit weights (`W8Weight`), the steps
between them whose rows come out in 8 bits (`norm_rows`, `gate_rows`,
`quantise_rows`), and the same cache and attention in 8 bits (`KV8Cache`).

As in `mf`, this is marshalling only: torch supplies device memory and the
stream, the kernels of libmf.so do the work.  Calls enqueue on `stream` (None:
torch's current one), copies of what is not contiguous too, and do not
synchronise; include/mf.h has the definitions.  They are for inference: an
operand that requires a gradient is refused while gradients are recorded, and so is
one with a tangent of forward mode.  So are outputs that lie over operands other than
their own rows (a norm's h over x or the residual, turned queries and attention's
results over the queries).
"""
from __future__ import annotations

import ctypes as C
import math
import threading
from typing import NamedTuple

import torch
from torch.autograd import forward_ad

from . import mf
from .mf import _check, _ptr

_DTYPES = {torch.float32: mf.MF_F32, torch.bfloat16: mf.MF_BF16, torch.float16: mf.MF_F16}
_HALF = (torch.bfloat16, torch.float16)
_p, _i32, _i64 = C.c_void_p, C.c_int32, C.c_int64


class W4Desc(C.Structure):
    _fields_ = [("n_out", _i64), ("n_in", _i64), ("group", _i32), ("dtype", _i32)]


class W4Args(C.Structure):
    _fields_ = [("w", W4Desc), ("d_packed", _p), ("d_x", _p), ("d_bias", _p), ("d_y", _p), ("rows", _i64),
                ("x_stride", _i64), ("y_stride", _i64)]


class Cache(C.Structure):
    _fields_ = [("n_pages", _i32), ("page_size", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("group", _i32),
                ("d_pages", _p)]


class Cache8(C.Structure):
    _fields_ = [("n_pages", _i32), ("page_size", _i32), ("n_kv_heads", _i32), ("head_dim", _i32), ("d_pages", _p)]


class Batch(C.Structure):
    _fields_ = [("n_seq", _i32), ("max_new", _i32), ("max_kv", _i32), ("rows", _i64), ("d_q_start", _p), ("d_kv_len", _p),
                ("d_page_table", _p), ("table_stride", _i64), ("table_cols", _i32)]


class AppendArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("d_k", _p), ("d_v", _p), ("k_stride", _i64), ("k_head_stride", _i64), ("v_stride", _i64),
                ("v_head_stride", _i64), ("d_cos", _p), ("d_sin", _p), ("n_pos", _i32), ("rot_dim", _i32),
                ("interleaved", _i32), ("n_heads", _i32), ("d_q", _p), ("d_q_out", _p), ("q_stride", _i64),
                ("q_head_stride", _i64), ("qo_stride", _i64), ("qo_head_stride", _i64)]


class AttnArgs(C.Structure):
    _fields_ = [("dtype", _i32), ("n_heads", _i32), ("d_q", _p), ("d_out", _p), ("d_lse", _p), ("q_stride", _i64),
                ("q_head_stride", _i64), ("out_stride", _i64), ("out_head_stride", _i64), ("scale", C.c_float), ("window", _i32)]


class Rows8Args(C.Structure):
    _fields_ = [("dtype", _i32), ("rows", _i64), ("n", _i64), ("d_x", _p), ("x_stride", _i64), ("d_codes", _p), ("codes_stride", _i64),
                ("d_scales", _p)]


class Norm8Args(C.Structure):
    _fields_ = [("row", Rows8Args), ("d_residual", _p), ("residual_stride", _i64), ("d_sum", _p), ("sum_stride", _i64), ("d_weight", _p),
                ("eps", C.c_float)]


class Gate8Args(C.Structure):
    _fields_ = [("row", Rows8Args), ("d_up", _p), ("up_stride", _i64)]


class W8Desc(C.Structure):
    _fields_ = [("n_out", _i64), ("n_in", _i64), ("dtype", _i32)]


class W8Args(C.Structure):
    _fields_ = [("w", W8Desc), ("d_packed", _p), ("d_x", _p), ("d_x_scales", _p), ("d_bias", _p), ("d_y", _p), ("rows", _i64),
                ("x_stride", _i64), ("y_stride", _i64)]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_of(device):
    """hipStream_t of torch's current stream on `device` (whose Python object
    costs as much to make as a kernel launch)."""
    if _raw_stream is not None:
        return _raw_stream(device.index)
    return torch.cuda.current_stream(device).cuda_stream


def _tensors(x):
    if isinstance(x, (tuple, list)):
        return [t for y in x for t in _tensors(y)]
    return [x] if isinstance(x, torch.Tensor) and x.is_cuda else []


def _on(device, stream, tensors, call):
    """`call` with `device` as the current one and `stream` (None: the device's own) as torch's current
    one, so that whatever it copies, allocates and launches is in one order: HIP runs stream 0 on the
    current device.  What it reads is kept until that has run, what it returns until the caller's own
    stream has."""
    if stream is not None and stream.device != device:
        raise ValueError(f"stream: one of {device} is wanted")
    with torch.cuda.device(device):
        before = torch.cuda.current_stream(device)
        if stream is None or stream == before:
            return call()
        with torch.cuda.stream(stream):
            got = call()
    for t in _tensors(tensors):
        t.record_stream(stream)
    for t in _tensors(got):
        t.record_stream(before)
    return got


class _Workspaces(threading.local):
    """Device workspaces, one per stream and device of a thread, which hands them back when it ends: calls that overlap
    must not share one.  A call that is captured gets one of its own from the graph's pool: the graph holds its address
    for good, and a larger one may take the held one's place."""

    def __init__(self):
        self._held = {}

    def get(self, nbytes: int, device):
        if torch.cuda.is_current_stream_capturing():
            return torch.empty(nbytes, dtype=torch.uint8, device=device)
        key = (device, _stream_of(device))
        ws = self._held.get(key)
        if ws is None or ws.numel() < nbytes:
            ws = self._held[key] = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws


_workspaces = _Workspaces()


def _require(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int32(x, name):
    """x for a field of 32 bits, which would take a larger number without its upper bits."""
    x = int(x)
    _require(-2 ** 31 <= x < 2 ** 31, f"{name}: a number of 32 bits is wanted")
    return x


def _no_gradient(t):
    """For a t that requires a gradient, or any where tangents may be (a call looks at no more than these two): the operators have
    no backward and no forward mode, and a result without either would lose t's gradient or tangent silently."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError("an operand requires a gradient, and there is none through this call: torch.no_grad() or detach() is wanted")
    if forward_ad._current_level >= 0 and forward_ad.unpack_dual(t).tangent is not None:
        raise ValueError("an operand has a tangent, and there is none through this call: detach() is wanted")


def _rows(t, name, shape, dtype, device):
    """A tensor of `shape` whose last dimension is contiguous (a copy where it is not)."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name}: {tuple(shape)} {dtype} on {device} is wanted")
    return t if t.stride(-1) == 1 else t.contiguous()


def _like(t):
    """A new contiguous tensor of t's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


def _into(t, name, shape, dtype, device):
    """An output of the caller's."""
    _require(isinstance(t, torch.Tensor) and tuple(t.shape) == tuple(shape) and t.dtype is dtype and t.device == device
             and (t.stride(-1) == 1 or t.shape[-1] <= 1), f"{name}: {tuple(shape)} {dtype} on {device} with a contiguous last dimension is wanted")
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_gradient(t)
    return t


class W4Weight:
    """Packed 4-bit weights [N, K] with a scale (and a zero point) for every
    `K // scales.shape[1]` weights of a row: w = scale * (code - zero).

    codes: uint8 [N, K // 2], the even column in the low four bits; scales:
    bfloat16 or float16 [N, K // G], G 32, 64 or 128; zeros: uint8 [N, K // G],
    0..15, or None (8).  Laid out once, here; the arguments may be freed after."""

    def __init__(self, codes, scales, zeros=None, stream=None):
        _require(isinstance(codes, torch.Tensor) and codes.dtype is torch.uint8 and codes.dim() == 2 and codes.is_cuda,
                 "codes: a uint8 [N, K // 2] tensor on the GPU is wanted")
        _require(isinstance(scales, torch.Tensor) and scales.dtype in _HALF and scales.dim() == 2
                 and scales.shape[0] == codes.shape[0] and scales.device == codes.device and scales.shape[1] > 0
                 and (2 * codes.shape[1]) % scales.shape[1] == 0,
                 "scales: bfloat16 or float16 [N, K // G] beside the codes is wanted")
        if scales.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(scales)
        _require(zeros is None or (isinstance(zeros, torch.Tensor) and zeros.dtype is torch.uint8
                                   and zeros.shape == scales.shape and zeros.device == codes.device),
                 "zeros: uint8 of the scales' shape is wanted")
        self.n_out, self.n_in = int(codes.shape[0]), 2 * int(codes.shape[1])
        self.group, self.dtype, self.device = self.n_in // int(scales.shape[1]), scales.dtype, codes.device
        self.desc = W4Desc(self.n_out, self.n_in, self.group, _DTYPES[self.dtype])
        nb = C.c_size_t()
        _check(mf.lib.mf_w4_pack_bytes(C.byref(self.desc), C.byref(nb)), "mf_w4_pack_bytes")
        lay_out = lambda: self._pack(codes, scales, zeros, int(nb.value))
        self.packed = _on(self.device, stream, (codes, scales, zeros), lay_out)
        self._packed_ptr = self.packed.data_ptr()
        self._ws_bytes = {}   # by rows

    def _pack(self, codes, scales, zeros, nbytes):
        codes, scales = codes.contiguous(), scales.contiguous()
        zeros = zeros if zeros is None else zeros.contiguous()
        packed = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(mf.lib.mf_w4_pack(C.byref(self.desc), _ptr(codes), _ptr(scales), _ptr(zeros), _ptr(packed),
                                 C.c_size_t(nbytes), _stream_of(self.device)), "mf_w4_pack")
        return packed

    def matmul(self, x, bias=None, out=None, stream=None):
        """x [.., K] @ W.T + bias [N] -> [.., N], in the scales' type."""
        if stream is not None or self.device.index != _current_device():
            return _on(self.device, stream, (x, bias, out, self.packed), lambda: self.matmul(x, bias, out))
        lead = x.shape[:-1]
        if not lead or x.shape[-1] != self.n_in or x.dtype is not self.dtype or x.device != self.device:
            _require(x.dim() == 1 and x.shape[0] == self.n_in and x.dtype is self.dtype and x.device == self.device,
                     f"x: [.., {self.n_in}] {self.dtype} on {self.device} is wanted")
        if bias is not None:
            _require(bias.dtype is self.dtype and bias.device == self.device and tuple(bias.shape) == (self.n_out,)
                     and bias.is_contiguous(), f"bias: contiguous [{self.n_out}] {self.dtype} is wanted")
            if bias.requires_grad or forward_ad._current_level >= 0:
                _no_gradient(bias)
        if x.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(x)
        if len(lead) != 1:
            x = x.reshape(-1, self.n_in)
        m = x.shape[0]
        if x.stride(1) != 1 or (m > 1 and x.stride(0) < self.n_in):
            x = x.contiguous()
        if out is None:
            y = x.new_empty((m, self.n_out))
            out = y if len(lead) == 1 else y.view(*lead, self.n_out)
        else:
            _into(out, "out", (*lead, self.n_out), self.dtype, self.device)
            y = out if out.dim() == 2 else out.view(-1, self.n_out)
        args = W4Args(self.desc, self._packed_ptr, x.data_ptr(), None if bias is None else bias.data_ptr(), y.data_ptr(), m,
                      x.stride(0), y.stride(0))
        need = self._ws_bytes.get(m)
        if need is None:
            nb = C.c_size_t()
            _check(mf.lib.mf_w4_workspace_size(C.byref(args), C.byref(nb)), "mf_w4_workspace_size")
            need = self._ws_bytes[m] = nb.value
        ws = _workspaces.get(need, self.device) if need else None
        s = mf.lib.mf_w4_matmul(C.byref(args), ws.data_ptr() if need else None, need, _stream_of(self.device))
        if s:
            _check(s, "mf_w4_matmul")
        return out


def _matrix(t, name, n, dtype, device):
    """[.., n] as rows of n with a contiguous last dimension (a copy where they are none)."""
    if not isinstance(t, torch.Tensor) or t.dim() == 0 or t.shape[-1] != n or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{name}: [.., {n}] {dtype} on {device} is wanted")
    if t.requires_grad or forward_ad._current_level >= 0:
        _no_gradient(t)
    if t.dim() != 2:
        t = t.reshape(-1, n)
    if t.stride(1) != 1 or (t.shape[0] > 1 and t.stride(0) < n):
        t = t.contiguous()
    return t


class Rows8(NamedTuple):
    """Rows in 8 bits: codes int8 [.., N] and a scale float32 [..] for each row; the values are scale * code.
    Made by `norm_rows`, `gate_rows` and `quantise_rows`, or of tensors at hand."""

    codes: torch.Tensor
    scales: torch.Tensor

    def _checked(self):
        """Codes as a matrix, and the scales."""
        codes, scales = self
        if not isinstance(codes, torch.Tensor) or codes.dtype is not torch.int8 or not codes.is_cuda or codes.dim() == 0 or codes.shape[-1] == 0:
            raise ValueError("codes: an int8 [.., N] tensor on the GPU is wanted")
        if (not isinstance(scales, torch.Tensor) or scales.dtype is not torch.float32 or scales.device != codes.device
                or scales.shape != codes.shape[:-1]):
            raise ValueError("scales: float32 [..] beside the codes is wanted")
        if scales.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(scales)
        if codes.dim() != 2 or not codes.is_contiguous():
            codes = _matrix(codes, "codes", codes.shape[-1], torch.int8, codes.device)
        return codes, scales if scales.is_contiguous() else scales.contiguous()

    def values(self, dtype=torch.float32, stream=None):
        """What the rows stand for, [.., N] in dtype."""
        if _elsewhere(self[0], stream):
            return _on(self[0].device, stream, tuple(self), lambda: self.values(dtype))
        codes, scales = self._checked()
        if dtype not in _DTYPES:
            raise ValueError("dtype: float32, bfloat16 or float16 is wanted")
        out, n, device = codes.new_empty(self[0].shape, dtype=dtype), codes.shape[1], codes.device
        s = mf.lib.mf_rows8_values(_DTYPES[dtype], codes.shape[0], n, codes.data_ptr(), codes.stride(0), scales.data_ptr(), out.data_ptr(), n,
                                   _stream_of(device))
        if s:
            _check(s, "mf_rows8_values")
        return out


def _rows8_of(x, name):
    """x as a matrix, the Rows8 that it is put into, and the call's arguments."""
    if not isinstance(x, torch.Tensor) or x.dtype not in _HALF or not x.is_cuda or x.dim() == 0 or x.shape[-1] == 0:
        raise ValueError(f"{name}: bfloat16 or float16 [.., N] on the GPU is wanted")
    shape, dt = x.shape, x.dtype
    n = shape[-1]
    if len(shape) == 2 and x.is_contiguous() and not (x.requires_grad or forward_ad._current_level >= 0):
        m, codes, rows, stride = x, torch.empty_like(x, dtype=torch.int8), shape[0], n
    else:
        m, codes = _matrix(x, name, n, dt, x.device), x.new_empty(shape, dtype=torch.int8)
        rows, stride = m.shape[0], m.stride(0)
    scales = x.new_empty(shape[:-1], dtype=torch.float32)
    return m, Rows8(codes, scales), Rows8Args(_DTYPES[dt], rows, n, m.data_ptr(), stride, codes.data_ptr(), n, scales.data_ptr())


def _elsewhere(x, stream):
    """Whether a call with x has to change the current device or stream first."""
    if stream is not None:
        return True
    return isinstance(x, torch.Tensor) and x.is_cuda and x.device.index != _current_device()


def quantise_rows(x, stream=None) -> Rows8:
    """x [.., N], bfloat16 or float16, in 8 bits."""
    if _elsewhere(x, stream):
        return _on(x.device, stream, x, lambda: quantise_rows(x))
    x, rows, a = _rows8_of(x, "x")
    s = mf.lib.mf_rows8(C.byref(a), _stream_of(x.device))
    if s:
        _check(s, "mf_rows8")
    return rows


def norm_rows(x, weight, residual=None, eps=1e-6, out=None, stream=None):
    """The root-mean-square norm of h = x + residual (x without one), times weight [N], in 8 bits: (Rows8, h).
    x, residual and h [.., N] and weight are of one type; out: where h goes with a residual, e.g. the residual itself."""
    if _elsewhere(x, stream):
        return _on(x.device, stream, (x, weight, residual, out), lambda: norm_rows(x, weight, residual, eps, out))
    carried = x
    x, rows, a = _rows8_of(x, "x")
    n, dt, dev = a.n, x.dtype, x.device
    if not isinstance(weight, torch.Tensor) or weight.shape != (n,) or weight.dtype is not dt or weight.device != dev:
        raise ValueError(f"weight: [{n}] {dt} on {dev} is wanted")
    if weight.requires_grad or forward_ad._current_level >= 0:
        _no_gradient(weight)
    if not weight.is_contiguous():
        weight = weight.contiguous()
    if residual is None:
        _require(out is None, "out: with a residual only, without one h is x")
        a = Norm8Args(a, None, 0, None, 0, weight.data_ptr(), eps)
    else:
        if not isinstance(residual, torch.Tensor) or residual.shape != carried.shape:
            raise ValueError(f"residual: {tuple(carried.shape)} is wanted")
        residual = _matrix(residual, "residual", n, dt, dev)
        if out is None:
            carried = _like(carried)
        else:
            carried = _into(out, "out", carried.shape, dt, dev)
        h = carried if carried.dim() == 2 else carried.view(-1, n)
        a = Norm8Args(a, residual.data_ptr(), residual.stride(0), h.data_ptr(), h.stride(0), weight.data_ptr(), eps)
    s = mf.lib.mf_norm8(C.byref(a), _stream_of(dev))
    if s:
        _check(s, "mf_norm8")
    return rows, carried


def gate_rows(gate, up, stream=None) -> Rows8:
    """gate * sigmoid(gate) * up in 8 bits; gate and up [.., N] of one type, e.g. the halves of one product's results."""
    if _elsewhere(gate, stream):
        return _on(gate.device, stream, (gate, up), lambda: gate_rows(gate, up))
    x, rows, a = _rows8_of(gate, "gate")
    _require(isinstance(up, torch.Tensor) and up.shape == gate.shape, f"up: {tuple(gate.shape)} is wanted")
    u = _matrix(up, "up", x.shape[1], x.dtype, x.device)
    a = Gate8Args(a, u.data_ptr(), u.stride(0))
    s = mf.lib.mf_gate8(C.byref(a), _stream_of(x.device))
    if s:
        _check(s, "mf_gate8")
    return rows


class W8Weight:
    """8-bit weights [N, K] with a scale for every output: w = scale * code.

    codes: int8 [N, K], K a multiple of 16; scales: float32 [N]; dtype: of
    biases and results, bfloat16 or float16.  Laid out once, here; the arguments
    may be freed after."""

    def __init__(self, codes, scales, dtype=torch.bfloat16, stream=None):
        _require(isinstance(codes, torch.Tensor) and codes.dtype is torch.int8 and codes.dim() == 2 and codes.is_cuda,
                 "codes: an int8 [N, K] tensor on the GPU is wanted")
        _require(isinstance(scales, torch.Tensor) and scales.dtype is torch.float32 and scales.dim() == 1
                 and scales.shape[0] == codes.shape[0] and scales.device == codes.device, "scales: float32 [N] beside the codes is wanted")
        if scales.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(scales)
        _require(dtype in _HALF, "dtype: bfloat16 or float16 is wanted")
        self.n_out, self.n_in, self.dtype, self.device = int(codes.shape[0]), int(codes.shape[1]), dtype, codes.device
        self.desc = W8Desc(self.n_out, self.n_in, _DTYPES[dtype])
        nb = C.c_size_t()
        _check(mf.lib.mf_w8_pack_bytes(C.byref(self.desc), C.byref(nb)), "mf_w8_pack_bytes")
        self.packed = _on(self.device, stream, (codes, scales), lambda: self._pack(codes, scales, int(nb.value)))
        self._packed_ptr = self.packed.data_ptr()
        self._ws_bytes = {}   # by rows, and whether they come in 8 bits

    def _pack(self, codes, scales, nbytes):
        codes, scales = codes.contiguous(), scales.contiguous()
        packed = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(mf.lib.mf_w8_pack(C.byref(self.desc), _ptr(codes), _ptr(scales), _ptr(packed), C.c_size_t(nbytes), _stream_of(self.device)),
               "mf_w8_pack")
        return packed

    def matmul(self, x, bias=None, out=None, stream=None):
        """x @ W.T + bias [N] -> [.., N]; x: Rows8 of [.., K], or [.., K] in the weight's type, which is put into 8 bits on the way."""
        if stream is not None or self.device.index != _current_device():
            held = tuple(x) if isinstance(x, tuple) else x
            return _on(self.device, stream, (held, bias, out, self.packed), lambda: self.matmul(x, bias, out))
        dt, dev, k, n = self.dtype, self.device, self.n_in, self.n_out
        if isinstance(x, tuple):
            _require(len(x) == 2, "x: codes and scales are wanted")
            rows = x if type(x) is Rows8 else Rows8(*x)
            x, xs = rows._checked()
            if x.shape[1] != k or x.device != dev:
                raise ValueError(f"x: rows of {k} on {dev} are wanted")
            lead = rows[0].shape[:-1]
            scales = xs.data_ptr()
        else:
            if not isinstance(x, torch.Tensor):
                raise ValueError(f"x: Rows8, or [.., {k}] {dt}, is wanted")
            lead, scales = x.shape[:-1], None
            x = _matrix(x, "x", k, dt, dev)
        if bias is not None:
            _require(bias.dtype is dt and bias.device == dev and tuple(bias.shape) == (n,) and bias.is_contiguous(),
                     f"bias: contiguous [{n}] {dt} on {dev} is wanted")
            if bias.requires_grad or forward_ad._current_level >= 0:
                _no_gradient(bias)
        m = x.shape[0]
        if out is None:
            y = x.new_empty((m, n), dtype=dt)
            out = y if len(lead) == 1 else y.view(*lead, n)
        else:
            _into(out, "out", (*lead, n), dt, dev)
            y = out if out.dim() == 2 else out.view(-1, n)
        a = W8Args(self.desc, self._packed_ptr, x.data_ptr(), scales, None if bias is None else bias.data_ptr(), y.data_ptr(), m, x.stride(0),
                   y.stride(0))
        key = (m, scales is None)
        need = self._ws_bytes.get(key)
        if need is None:
            nb = C.c_size_t()
            _check(mf.lib.mf_w8_workspace_size(C.byref(a), C.byref(nb)), "mf_w8_workspace_size")
            need = self._ws_bytes[key] = nb.value
        ws = _workspaces.get(need, dev) if need else None
        s = mf.lib.mf_w8_matmul(C.byref(a), ws.data_ptr() if need else None, need, _stream_of(dev))
        if s:
            _check(s, "mf_w8_matmul")
        return out


def rope_table(n_pos: int, rot_dim: int, base: float = 10000.0, device="cuda"):
    """(cos, sin) [n_pos, rot_dim // 2] float32 for `KV4Cache.append`, computed in 64 bits."""
    half = rot_dim // 2
    inv = base ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * inv
    return a.cos().float(), a.sin().float()


class KV4Batch:
    """The sequences of one step (mf_kv4_batch), shared by its append, reads
    and attention; made by the cache's `batch`.  The device tensors are read by
    every call, so a server may update them in place between steps."""

    def __init__(self, q_start, kv_len, page_table, rows, max_new, max_kv):
        for t, name in ((q_start, "q_start"), (kv_len, "kv_len"), (page_table, "page_table")):
            _require(isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.is_cuda, f"{name}: int32 on the GPU is wanted")
        n = int(kv_len.shape[0])
        _require(kv_len.dim() == 1 and kv_len.is_contiguous(), "kv_len: contiguous [n_seq] is wanted")
        _require(tuple(q_start.shape) == (n + 1,) and q_start.is_contiguous(), "q_start: contiguous [n_seq + 1] is wanted")
        _require(page_table.dim() == 2 and page_table.shape[0] == n and (page_table.stride(1) == 1 or page_table.shape[1] <= 1),
                 "page_table: [n_seq, pages] with a contiguous last dimension is wanted")
        self.tensors, self.device = (q_start, kv_len, page_table), kv_len.device
        self._ws_bytes = {}   # of attention, by query heads, window and the cache's shape: a function of the sizes
        self.rows = int(rows)
        _require(-2 ** 63 <= self.rows < 2 ** 63, "rows: a number of 64 bits is wanted")
        self.raw = Batch(n, _int32(max_new, "max_new"), _int32(max_kv, "max_kv"), self.rows, q_start.data_ptr(), kv_len.data_ptr(), page_table.data_ptr(),
                         page_table.stride(0), int(page_table.shape[1]))


class _KVCache:
    """What the paged caches share: n_pages pages of page_size tokens for n_kv_heads heads of head_dim values."""

    def _lay_out(self, raw, bytes_call, n_pages, page_size, n_kv_heads, head_dim, kind, device):
        self.raw, self.device = raw, torch.device(device)
        nb = C.c_size_t()
        _check(getattr(mf.lib, bytes_call)(C.byref(self.raw), C.byref(nb)), bytes_call)
        self.pages = torch.empty(int(nb.value), dtype=torch.uint8, device=self.device)
        self.device = self.pages.device
        self.raw.d_pages = self.pages.data_ptr()
        self.n_kv_heads, self.head_dim, self.page_size = int(n_kv_heads), int(head_dim), int(page_size)
        self._shape = (self.n_kv_heads, self.head_dim, kind, self.page_size)
        self.bytes_per_token = int(nb.value) // (int(n_pages) * self.page_size)

    def batch(self, q_start, kv_len, page_table, rows, max_new, max_kv) -> KV4Batch:
        """q_start int32 [n_seq + 1], kv_len int32 [n_seq] (tokens of each
        sequence, the step's new ones included), page_table int32 [n_seq, ..];
        rows: of the step's tensors; max_new, max_kv: the largest number of new
        tokens and of tokens of a sequence, known on the host."""
        b = KV4Batch(q_start, kv_len, page_table, rows, max_new, max_kv)
        _require(all(t.device == self.device for t in b.tensors), f"the batch's tensors: on {self.device} is wanted")
        b.device = self.device
        return b

    def _beside(self, batch):
        if batch.device != self.device:
            raise ValueError(f"batch: on {self.device} is wanted")

    def append(self, batch: KV4Batch, k, v, cos=None, sin=None, q=None, interleaved=False, q_out=None, stream=None):
        """Writes k and v [rows, n_kv_heads, head_dim] into the cache, the keys
        turned by their positions when cos / sin [n_pos, rot_dim // 2] are given;
        with q [rows, n_heads, head_dim] also returns the queries turned the
        same way (q_out: where to, e.g. q itself)."""
        if batch.device is not self.device:
            self._beside(batch)
        if stream is not None or self.device.index != _current_device():
            return _on(self.device, stream, (k, v, cos, sin, q, q_out, self.pages, batch.tensors),
                       lambda: self.append(batch, k, v, cos, sin, q, interleaved, q_out))
        if k.requires_grad or v.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(k)
            _no_gradient(v)
        dt, dev = k.dtype, self.device
        _require(dt in _HALF, "k: bfloat16 or float16 is wanted")
        shape = (batch.rows, self.n_kv_heads, self.head_dim)
        k, v = _rows(k, "k", shape, dt, dev), _rows(v, "v", shape, dt, dev)
        ks, vs = k.stride(), v.stride()
        if cos is None:
            _require(sin is None, "cos and sin: both or neither are wanted")
            _require(q is None, "q: only turned here, so cos and sin are wanted with it")
            a = AppendArgs(_DTYPES[dt], k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1])
        else:
            _require(sin is not None, "cos and sin: both or neither are wanted")
            n_pos, half = cos.shape
            _require(cos.shape == sin.shape and cos.dtype is sin.dtype is torch.float32 and cos.device == sin.device == dev
                     and cos.is_contiguous() and sin.is_contiguous(), f"cos, sin: contiguous float32 [n_pos, rot_dim // 2] on {dev} is wanted")
            if cos.requires_grad or sin.requires_grad or forward_ad._current_level >= 0:
                _no_gradient(cos)
                _no_gradient(sin)
            turn = (cos.data_ptr(), sin.data_ptr(), n_pos, 2 * half, 1 if interleaved else 0)
            if q is None:
                a = AppendArgs(_DTYPES[dt], k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1], *turn)
            else:
                _require(q.dim() == 3, "q: [rows, n_heads, head_dim] is wanted")
                heads = q.shape[1]
                if q.requires_grad or forward_ad._current_level >= 0:
                    _no_gradient(q)
                q = _rows(q, "q", (batch.rows, heads, self.head_dim), dt, dev)
                q_out = _like(q) if q_out is None else _into(q_out, "q_out", q.shape, dt, dev)
                qs, os = q.stride(), q_out.stride()
                a = AppendArgs(_DTYPES[dt], k.data_ptr(), v.data_ptr(), ks[0], ks[1], vs[0], vs[1], *turn, heads, q.data_ptr(),
                               q_out.data_ptr(), qs[0], qs[1], os[0], os[1])
        s = getattr(mf.lib, self._APPEND)(C.byref(self.raw), C.byref(batch.raw), C.byref(a), _stream_of(dev))
        if s:
            _check(s, self._APPEND)
        return q_out

    def read(self, batch: KV4Batch, dtype=torch.float32, stream=None):
        """(keys, values) [rows, n_kv_heads, head_dim] that the cache holds for the batch's rows."""
        if batch.device is not self.device:
            self._beside(batch)
        if stream is not None or self.device.index != _current_device():
            return _on(self.device, stream, (self.pages, batch.tensors), lambda: self.read(batch, dtype))
        _require(dtype in _DTYPES, "dtype: float32, bfloat16 or float16 is wanted")
        k = torch.empty((batch.rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device)
        v = torch.empty_like(k)
        s = getattr(mf.lib, self._READ)(C.byref(self.raw), C.byref(batch.raw), _DTYPES[dtype], k.data_ptr(), v.data_ptr(),
                               _stream_of(self.device))
        if s:
            _check(s, self._READ)
        return k, v

    def attention(self, batch: KV4Batch, q, scale=None, window=0, lse=False, out=None, stream=None):
        """Causal attention of q [rows, n_heads, head_dim] over the cached
        tokens: [rows, n_heads, head_dim], with lse=True also the log of the
        softmax sums [rows, n_heads] float32.  scale: 1 / sqrt(head_dim) by
        default; window > 0: only the newest `window` tokens up to each row's."""
        if batch.device is not self.device:
            self._beside(batch)
        if stream is not None or self.device.index != _current_device():
            return _on(self.device, stream, (q, out, self.pages, batch.tensors), lambda: self.attention(batch, q, scale, window, lse, out))
        _require(q.dim() == 3 and q.dtype in _HALF, "q: bfloat16 or float16 [rows, n_heads, head_dim] is wanted")
        if q.requires_grad or forward_ad._current_level >= 0:
            _no_gradient(q)
        heads = q.shape[1]
        q = _rows(q, "q", (batch.rows, heads, self.head_dim), q.dtype, self.device)
        out = _like(q) if out is None else _into(out, "out", q.shape, q.dtype, self.device)
        ls = torch.empty((batch.rows, heads), dtype=torch.float32, device=self.device) if lse else None
        a = AttnArgs(_DTYPES[q.dtype], heads, q.data_ptr(), out.data_ptr(), None if ls is None else ls.data_ptr(), *q.stride()[:2],
                     *out.stride()[:2], 1.0 / math.sqrt(self.head_dim) if scale is None else float(scale), _int32(window, "window"))
        key = (heads, a.window, self._shape)
        need = batch._ws_bytes.get(key)
        if need is None:
            nb = C.c_size_t()
            _check(getattr(mf.lib, self._WORKSPACE)(C.byref(self.raw), C.byref(batch.raw), C.byref(a), C.byref(nb)), self._WORKSPACE)
            need = batch._ws_bytes[key] = nb.value
        ws = _workspaces.get(need, self.device) if need else None
        s = getattr(mf.lib, self._ATTENTION)(C.byref(self.raw), C.byref(batch.raw), C.byref(a), ws.data_ptr() if need else None, need, _stream_of(self.device))
        if s:
            _check(s, self._ATTENTION)
        return out if ls is None else (out, ls)


class KV4Cache(_KVCache):
    """A paged key/value cache in 4 bits: n_pages pages of page_size tokens for
    n_kv_heads heads of head_dim values; `group` neighbouring values share a
    scale and an offset.  `bytes_per_token` is what a token costs."""

    _APPEND, _READ, _WORKSPACE, _ATTENTION = "mf_kv4_append", "mf_kv4_read", "mf_kv4_workspace_size", "mf_kv4_attention"

    def __init__(self, n_pages, page_size, n_kv_heads, head_dim, group=64, device="cuda"):
        raw = Cache(_int32(n_pages, "n_pages"), _int32(page_size, "page_size"), _int32(n_kv_heads, "n_kv_heads"), _int32(head_dim, "head_dim"),
                    _int32(group, "group"), None)
        self._lay_out(raw, "mf_kv4_cache_bytes", n_pages, page_size, n_kv_heads, head_dim, int(group), device)


class KV8Cache(_KVCache):
    """A paged key/value cache in 8 bits, used as the one in 4 bits: n_pages pages of
    page_size tokens for n_kv_heads heads of head_dim values; 16 tokens of a head
    share a scale for their keys and one for their values.  A step that begins inside
    such a block needs the block's earlier tokens in the cache, or zeroed memory."""

    _APPEND, _READ, _WORKSPACE, _ATTENTION = "mf_kv8_append", "mf_kv8_read", "mf_kv8_workspace_size", "mf_kv8_attention"

    def __init__(self, n_pages, page_size, n_kv_heads, head_dim, device="cuda"):
        raw = Cache8(_int32(n_pages, "n_pages"), _int32(page_size, "page_size"), _int32(n_kv_heads, "n_kv_heads"), _int32(head_dim, "head_dim"), None)
        self._lay_out(raw, "mf_kv8_cache_bytes", n_pages, page_size, n_kv_heads, head_dim, "8-bit", device)
