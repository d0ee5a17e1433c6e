"""Binding of the stand-alone operators of a training step: layer norm and expert routing, forward and
backward (include/layer.h), and the orthogonalisation of a momentum (include/muon.h).

Argument checks and marshalling only, as in ``soap``: outputs and workspaces are allocated here
with torch, on the operands' device, and everything is computed by libsoap.so on the given stream
(the current one by default). A tensor that the caller made on another stream has to be ordered
before the call by the caller, as for any stream-ordered work; it may be dropped as soon as the call
returns, since the given stream is recorded on it. Results belong to the given stream, as tensors
made under ``torch.cuda.stream`` do: order their uses elsewhere after it.

The calls know nothing of autograd: a tensor that requires gradients is taken as its values, and results
are detached (the backward passes are calls of their own). ``status`` is optional everywhere: without it a
bounded device wait that gave up shows in the results alone, as NaN.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .soap import DTYPES, SOAP_OK, SoapError, load_library

# What every call asks torch for, without the Python objects around it (torch.cuda.current_stream(...) alone
# costs as much as half a launch): the cudaStream_t that is current on a device, and the current device. A
# torch without CUDA has neither, nor tensors that get as far as them.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current = getattr(torch._C, "_cuda_getDevice", None)
_F32, _I32 = torch.float32, torch.int32
_empty, _empty_like = torch.empty, torch.empty_like


def _refuse(name, t, dtype, device):
    """Raises for what _operand turned down."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype if dtype is not None else t.dtype not in DTYPES:
        raise TypeError(f"{name}: expected {dtype or 'float32, bfloat16 or float16'}, got {t.dtype}")
    raise ValueError(f"{name}: on {t.device}, expected {device}")


def _operand(name, t, dtype=None, device=None):
    """Checks a CUDA tensor of a supported (or the given) type on the given device; returns the device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(name, t, dtype, device)
    if t.dtype not in DTYPES if dtype is None else t.dtype != dtype:
        _refuse(name, t, dtype, device)
    if device is not None and t.device != device:
        _refuse(name, t, dtype, device)
    return t.device


def _elsewhere(index, stream, *operands):
    """The context in which a call has to run and allocate if that is not the present one: the given
    stream (outputs and workspaces then come from its memory pool; the operands' memory is not given out
    again before what that stream has of theirs to do), or the operands' device."""
    if stream is not None:
        if torch.device(stream.device).index != index:
            raise ValueError(f"stream of {stream.device} given for work on cuda:{index}")
        for t in operands:
            if isinstance(t, torch.Tensor) and t.is_cuda:
                t.record_stream(stream)
        return torch.cuda.stream(stream)
    return None if _current() == index else torch.cuda.device(index)


def _rows(t):
    """(tensor, rows, leading dimension) of [..., width] seen as rows; a copy only where no single leading
    dimension describes it."""
    shape = t.shape
    width = shape[-1]
    if not t.is_contiguous():
        rows, ld = 1, width
        for n, step in zip(reversed(shape[:-1]), reversed(t.stride()[:-1])):
            if n == 1:
                continue
            if rows == 1:
                ld = step
            elif step != rows * ld:
                ld = 0
            rows *= n
        if ld >= width and (t.stride(-1) == 1 or width == 1):
            return t, rows, ld
        t = t.contiguous()
    if len(shape) == 2:
        return t, shape[0], width
    return t, t.numel() // width if width else 0, width


def _done(code, name):
    if code != SOAP_OK:
        raise SoapError(code, name)


def _weights(name, x, width, *vectors):
    """Checks weight and bias (either may be None) and returns their soap_dtype_t."""
    index, wt = x.get_device(), None
    for t in vectors:
        if t is None:
            continue
        if not isinstance(t, torch.Tensor) or t.get_device() != index:
            _operand(name, t, None, x.device)
        dt = t.dtype
        if dt is not _F32 and dt is not x.dtype or wt is not None and dt is not wt:
            raise TypeError(f"{name}: weight and bias must both be float32 or both {x.dtype}")
        if t.shape != (width,) or not t.is_contiguous():
            raise ValueError(f"{name}: weight and bias need {width} contiguous elements")
        wt = dt
    return 0 if wt is None else DTYPES[wt]


def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                       eps: float = 1e-5, status: Optional[torch.Tensor] = None, stream=None):
    """Layer norm over x's last dimension: (y, mean, rstd), with y of x's shape and type and the fp32
    statistics of every row, which the backward pass takes. weight and bias: float32 or x's type.
    status: an int32 CUDA word that SOAP_STATUS_TIMEOUT is ORed into."""
    name = "layer_norm_forward"
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in DTYPES:
        _refuse(name, x, None, None)
    index = x.get_device()
    if stream is not None or index != _current():
        with _elsewhere(index, stream, x, weight, bias, status):
            return layer_norm_forward(x, weight, bias, eps, status)
    if status is not None:
        _operand(name, status, _I32, x.device)
    shape = x.shape
    if not shape or shape[-1] < 1:
        raise ValueError(f"{name}: the normalised dimension is empty")
    x, rows, ld = _rows(x)
    width = shape[-1]
    wt = _weights(name, x, width, weight, bias)
    y = _empty_like(x) if x.is_contiguous() else _empty(shape, dtype=x.dtype, device=x.device)
    mean = _empty(shape[:-1], dtype=_F32, device=x.device)
    rstd = _empty_like(mean)
    _done(load_library().layer_norm_forward(
        rows, width, x.data_ptr(), ld, DTYPES[x.dtype], None if weight is None else weight.data_ptr(),
        None if bias is None else bias.data_ptr(), wt, eps, y.data_ptr(), width, mean.data_ptr(),
        rstd.data_ptr(), None if status is None else status.data_ptr(), _raw_stream(index)), name)
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: Optional[torch.Tensor] = None, params: bool = True,
                        status: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight, dbias) of layer_norm_forward from dy and its mean and rstd. dx has x's type;
    dweight and dbias are float32 (the optimizer's gradient type), or None without ``params``."""
    name = "layer_norm_backward"
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in DTYPES:
        _refuse(name, x, None, None)
    index = x.get_device()
    if stream is not None or index != _current():
        with _elsewhere(index, stream, dy, x, mean, rstd, weight, status):
            return layer_norm_backward(dy, x, mean, rstd, weight, params, status)
    dev = x.device
    _operand(name, dy, x.dtype, dev)
    if status is not None:
        _operand(name, status, _I32, dev)
    shape = x.shape
    if dy.shape != shape:
        raise ValueError(f"{name}: dy and x have different shapes")
    if not shape or shape[-1] < 1:
        raise ValueError(f"{name}: the normalised dimension is empty")
    x, rows, ld = _rows(x)
    dy, _, ld_dy = _rows(dy)
    width = shape[-1]
    for t in (mean, rstd):
        _operand(name, t, _F32, dev)
        if t.numel() != rows or not t.is_contiguous():
            raise ValueError(f"{name}: mean and rstd do not match x's rows")
    wt = _weights(name, x, width, weight)
    lib = load_library()
    dx = _empty_like(x) if x.is_contiguous() else _empty(shape, dtype=x.dtype, device=x.device)
    dw = db = ws = None
    ws_bytes = 0
    if params:
        ws_bytes = lib.layer_norm_workspace_bytes(rows, width)
        dw = _empty(width, dtype=_F32, device=dev)
        db = _empty_like(dw)
        ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    _done(lib.layer_norm_backward(
        rows, width, dy.data_ptr(), ld_dy, x.data_ptr(), ld, DTYPES[x.dtype], mean.data_ptr(), rstd.data_ptr(),
        None if weight is None else weight.data_ptr(), wt, dx.data_ptr(), width, dw.data_ptr() if params else None,
        db.data_ptr() if params else None, ws.data_ptr() if params else None, ws_bytes,
        None if status is None else status.data_ptr(), _raw_stream(index)), name)
    return dx, dw, db


class Routing(NamedTuple):
    """What route_forward decided: int32 indices and fp32 gates [..., k], int32 counts [experts], fp32
    mean_probs [experts], the fp32 scalar loss and the int32 scalar number of tokens counted (live);
    for route_backward, each row's softmax statistics, and mask, normalize and coef as given."""
    indices: torch.Tensor
    gates: torch.Tensor
    counts: torch.Tensor
    mean_probs: torch.Tensor
    loss: torch.Tensor
    live: torch.Tensor
    stats: torch.Tensor
    mask: Optional[torch.Tensor]
    normalize: bool
    coef: float


def route_forward(logits: torch.Tensor, k: int, mask: Optional[torch.Tensor] = None, normalize: bool = True,
                  coef: float = 0.01, status: Optional[torch.Tensor] = None, stream=None) -> Routing:
    """A router's choice of k experts per token from logits [..., experts], with per-expert counts and the
    balance loss (include/layer.h). mask: bool per token, False = left out. status: an int32 CUDA word that
    SOAP_STATUS_NONFINITE is ORed into."""
    name = "route_forward"
    dev = _operand(name, logits)
    if stream is not None or dev.index != _current():
        with _elsewhere(dev.index, stream, logits, mask, status):
            return route_forward(logits, k, mask, normalize, coef, status)
    if logits.dim() < 1:
        raise ValueError(f"{name}: needs at least one dimension")
    z, tokens, ld = _rows(logits)
    lead, experts = z.shape[:-1], z.shape[-1]
    if mask is not None:
        _operand(name, mask, torch.bool, dev)
        if mask.shape != lead:
            raise ValueError(f"{name}: the mask needs one value per token")
        mask = mask.contiguous()
    if status is not None:
        _operand(name, status, _I32, dev)
    lib = load_library()
    k = int(k)
    ws_bytes = lib.layer_route_workspace_bytes(tokens, experts)
    if ws_bytes == 0 or not 1 <= k <= min(experts, 32):
        raise ValueError(f"{name}: needs 1 to 1024 experts and k of 1 to min(experts, 32)")
    chosen = lead + (k,)
    gates, indices = _empty(chosen, dtype=_F32, device=dev), _empty(chosen, dtype=_I32, device=dev)
    stats = _empty(lead + (2,), dtype=_F32, device=dev)
    mean_probs, counts = _empty(experts, dtype=_F32, device=dev), _empty(experts, dtype=_I32, device=dev)
    loss, live = _empty((), dtype=_F32, device=dev), _empty((), dtype=_I32, device=dev)
    ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    _done(lib.layer_route_forward(
        tokens, experts, k, z.data_ptr(), ld, DTYPES[z.dtype], None if mask is None else mask.data_ptr(),
        int(normalize), coef, indices.data_ptr(), gates.data_ptr(), stats.data_ptr(), counts.data_ptr(),
        live.data_ptr(), mean_probs.data_ptr(), loss.data_ptr(), None if status is None else status.data_ptr(),
        ws.data_ptr(), ws_bytes, _raw_stream(dev.index)), name)
    return Routing(indices, gates, counts, mean_probs, loss, live, stats, mask, bool(normalize), float(coef))


def route_backward(logits: torch.Tensor, routing: Routing, dgates: Optional[torch.Tensor] = None, dloss: float = 1.0,
                   stream=None) -> torch.Tensor:
    """dlogits (logits' shape and type) from the gates' gradient (fp32, None for zero) and the loss's (dloss, a
    host number). It is linear in both: a scale of the two that is on the device multiplies the result."""
    name = "route_backward"
    dev = _operand(name, logits)
    if stream is not None or dev.index != _current():
        with _elsewhere(dev.index, stream, logits, dgates, *routing):
            return route_backward(logits, routing, dgates, dloss)
    shape, shape_k = logits.shape, routing.indices.shape
    if logits.dim() < 1 or shape_k[:-1] != shape[:-1] or routing.counts.shape[0] != shape[-1]:
        raise ValueError(f"{name}: the routing is of other logits")
    if routing.indices.device != dev:
        raise ValueError(f"{name}: the routing is on {routing.indices.device}, the logits on {dev}")
    if dgates is not None:
        _operand(name, dgates, torch.float32, dev)
        if dgates.shape != shape_k:
            raise ValueError(f"{name}: dgates needs the gates' shape")
        dgates = dgates.contiguous()
    z, tokens, ld = _rows(logits)
    dz = _empty_like(z, memory_format=torch.contiguous_format)
    _done(load_library().layer_route_backward(
        tokens, shape[-1], shape_k[-1], z.data_ptr(), ld, DTYPES[z.dtype],
        None if routing.mask is None else routing.mask.data_ptr(), int(routing.normalize), routing.coef, dloss,
        routing.indices.data_ptr(), routing.stats.data_ptr(), routing.counts.data_ptr(), routing.live.data_ptr(),
        None if dgates is None else dgates.data_ptr(), dz.data_ptr(), shape[-1], _raw_stream(dev.index)), name)
    return dz


def _matrices(name, M):
    """(tensor, batch, rows, cols, ld, batch stride, transposed) of [..., m, n]: row-major matrices, or
    column-major ones seen as their transposes; a copy where neither describes it."""
    if M.dim() < 2:
        raise ValueError(f"{name}: needs matrices")
    m, n = M.shape[-2:]
    for _ in range(2):
        T = M if M.dim() == 3 else M.unsqueeze(0) if M.dim() == 2 else None
        if T is None and M.is_contiguous():
            T = M.view(-1, m, n)
        if T is None and M.mT.is_contiguous():
            T = M.mT.view(-1, n, m).mT
        if T is not None:
            b, sb, sr, sc = T.shape[0], *T.stride()
            if (sc == 1 or n == 1) and (sr >= n or m == 1):
                ld = sr if m > 1 else n
                if b == 1 or sb >= (m - 1) * ld + n:
                    return M, b, m, n, ld, sb, False
            if (sr == 1 or m == 1) and (sc >= m or n == 1):
                ld = sc if n > 1 else m
                if b == 1 or sb >= (n - 1) * ld + m:
                    return M, b, n, m, ld, sb, True
        M = M.contiguous()
    raise ValueError(f"{name}: no layout for strides {M.stride()}")


def muon_orthogonalize(M: torch.Tensor, coeffs=None, ns_steps: int = 16, eps: float = 1e-7,
                       status: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """X_n of Muon's Newton-Schulz iterations for matrices [..., m, n] (float32, bfloat16 or float16, row- or
    column-major): a new dense tensor of M's shape, type and order. coeffs: a list of (a_i, b_i, c_i)
    (its length is the number of steps), None: the library's quintic polynomial, ns_steps times.
    status: an int32 CUDA word that SOAP_STATUS_* bits are ORed into."""
    name = "muon_orthogonalize"
    dev = _operand(name, M)
    if stream is not None or dev.index != _current():
        with _elsewhere(dev.index, stream, M, status):
            return muon_orthogonalize(M, coeffs, ns_steps, eps, status)
    if status is not None:
        _operand(name, status, _I32, dev)
    flat = None
    if coeffs is not None:
        ns_steps = len(coeffs)
        flat = (ctypes.c_float * (3 * ns_steps))(*[float(x) for abc in coeffs for x in abc])
    M, batch, rows, cols, ld, stride, swapped = _matrices(name, M)
    if M.numel() == 0:
        return _empty_like(M)
    out = _empty(M.shape[:-2] + (rows, cols), dtype=M.dtype, device=dev)
    lib = load_library()
    ws_bytes = lib.muon_orthogonalize_workspace_bytes(batch, rows, cols, DTYPES[M.dtype])
    if ws_bytes == 0:
        raise ValueError(f"{name}: sides of 1 to 65536, fewer than 2^31 elements and 65536 matrices")
    ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    _done(lib.muon_orthogonalize(batch, rows, cols, M.data_ptr(), ld, stride, DTYPES[M.dtype], flat, ns_steps, eps,
                                 out.data_ptr(), cols, rows * cols, ws.data_ptr(), ws_bytes,
                                 None if status is None else status.data_ptr(), _raw_stream(dev.index)), name)
    return out.mT if swapped else out
