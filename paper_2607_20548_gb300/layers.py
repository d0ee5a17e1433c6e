"""Binding of the stand-alone operators of a training step: layer norm, expert routing, the gated feed-forward
block, and queries' and keys' norms with their rotation, forward and backward (include/layer.h), and the
orthogonalisation of a momentum (include/muon.h).

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
import functools
import math
from typing import NamedTuple, Optional

import torch

from .soap import DTYPES, SOAP_OK, SoapError, layer_heads, layer_matrix, load_library

# What every call asks torch for, without the Python objects around it (torch.cuda.current_stream(...) alone
# costs as much as half a launch): the cudaStream_t that is current on a device, and the current device. A
# torch without CUDA has neither, nor tensors that get as far as them.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current = getattr(torch._C, "_cuda_getDevice", None)
_F32, _I32 = torch.float32, torch.int32
_empty, _empty_like = torch.empty, torch.empty_like


@functools.lru_cache(4096)
def _size(function, *args):
    """What one of the library's functions of sizes alone gives (asked through ctypes, 1 us each time)."""
    return getattr(load_library(), function)(*args)


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


def _heads(name, t, dtype, index):
    """(layer_heads, lead shape, batch, length, heads, dim) of [..., heads, dim] (and what has to live until the call
    where that is a copy): [heads, dim], [length, heads, dim] or [batch, length, heads, dim] where it lies; a copy of more
    leading dimensions that do not merge, or of heads whose elements lie apart."""
    if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype is not dtype:
        _operand(name, t, dtype, torch.device("cuda", index))
    shape, step, made = t.shape, t.stride(), None
    n = len(shape)
    if n < 2:
        raise ValueError(f"{name}: needs [..., heads, dim]")
    lead = shape[:-2]
    if n > 4 or step[-1] != 1:
        if step[-1] != 1 and shape[-1] > 1:
            t = t.contiguous()
        made = t = t if n <= 4 else t.reshape(math.prod(lead[:-1]), *shape[-3:])
        shape, step = t.shape, t.stride()
        n = len(shape)
    if n == 3:
        return layer_heads(t.data_ptr(), 0, step[0], step[1]), lead, 1, *shape, made
    if n == 4:
        return layer_heads(t.data_ptr(), step[0], step[1], step[2]), lead, *shape, made
    return layer_heads(t.data_ptr(), 0, 0, step[0]), lead, 1, 1, *shape, made


def _qk_common(name, q, k, cos, sin, positions, q_weight, k_weight, status):
    """Checks what both passes take; the arguments of the C calls from the sizes to the positions in four pieces, and
    what has to live until the call."""
    index, dtype = q.get_device(), q.dtype
    hq, lead, batch, length, heads, dim, made_q = _heads(name, q, dtype, index)
    hk, lead_k, _, _, kv_heads, dim_k, made_k = _heads(name, k, dtype, index)
    if lead_k != lead or dim_k != dim:
        raise ValueError(f"{name}: q and k need the same tokens and the same size of a head")
    if dim % 2 or not 2 <= dim <= 512 or heads > 32768 or kv_heads > 32768:
        raise ValueError(f"{name}: heads need an even size of 2 to 512, and there are 32768 at most")
    if (cos is None) != (sin is None):
        raise ValueError(f"{name}: cos and sin come together")
    table = (None, None, 0, None, 0)
    rotary = 0
    if cos is not None:
        for t in (cos, sin):
            if not isinstance(t, torch.Tensor) or t.get_device() != index or t.dtype is not _F32:
                _operand(name, t, _F32, q.device)
            if t.dim() != 2 or t.shape != cos.shape or not t.is_contiguous():
                raise ValueError(f"{name}: cos and sin need contiguous [places, rotary / 2] elements")
        places, rotary = cos.shape
        rotary *= 2
        if rotary > dim:
            raise ValueError(f"{name}: {rotary} elements to rotate in heads of {dim}")
        table = (cos.data_ptr(), sin.data_ptr(), places, None, 0)
    if positions is not None:
        wide = isinstance(positions, torch.Tensor) and positions.dtype is torch.int64
        if not wide and (not isinstance(positions, torch.Tensor) or positions.dtype is not _I32):
            raise TypeError(f"{name}: positions are int32 or int64")
        if positions.get_device() != index:
            _operand(name, positions, positions.dtype, q.device)
        if positions.shape != lead:
            if positions.shape != lead[-1:]:
                raise ValueError(f"{name}: needs one position per token, or per token of a sequence")
            positions = positions.expand(lead)
        if not positions.is_contiguous():
            positions = positions.contiguous()
        table = (*table[:3], positions.data_ptr(), int(wide))
    weights = (None, None, 0)
    if q_weight is not None or k_weight is not None:
        weights = (None if q_weight is None else q_weight.data_ptr(), None if k_weight is None else k_weight.data_ptr(),
                   _weights(name, q, dim, q_weight, k_weight))
    if status is not None:
        _operand(name, status, _I32, q.device)
    return (batch, length, heads, kv_heads, dim, rotary), (hq, hk), weights, table, (made_q, made_k, positions)


def _dense_like(t, dev):
    return _empty_like(t) if t.is_contiguous() else _empty(t.shape, dtype=t.dtype, device=dev)


def _dense_heads(t, sizes, heads):
    dim = sizes[4]
    return layer_heads(t.data_ptr(), sizes[1] * heads * dim, heads * dim, dim)


def qk_rotary_forward(q: torch.Tensor, k: torch.Tensor, cos: Optional[torch.Tensor] = None,
                      sin: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                      q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                      eps: float = 1e-6, interleaved: bool = False, status: Optional[torch.Tensor] = None, stream=None):
    """Queries [..., heads, dim] and keys [..., kv_heads, dim] of the same tokens, each head divided by its root
    mean square, multiplied by its weight (float32 or q's type) and with its first elements rotated by the token's
    position (include/layer.h): (q, k) as new dense tensors. cos, sin: float32 [places, rotary / 2], None: no
    rotation. positions: int32 or int64, one per token or per token of a sequence, None: a token's place in its
    sequence (the dimension before the heads). Slices and transposes of heads and tokens are read where they lie.
    status: an int32 CUDA word that SOAP_STATUS_RANGE is ORed into where a position is not in the table; the
    token's results are NaN."""
    name = "qk_rotary_forward"
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dtype not in DTYPES:
        _refuse(name, q, None, None)
    index, dev = q.get_device(), q.device
    if stream is not None or index != _current():
        with _elsewhere(index, stream, q, k, cos, sin, positions, q_weight, k_weight, status):
            return qk_rotary_forward(q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, status)
    sizes, heads, w, table, held = _qk_common(name, q, k, cos, sin, positions, q_weight, k_weight, status)
    out_q, out_k = _dense_like(q, dev), _dense_like(k, dev)
    _done(load_library().layer_qk_forward(
        *sizes, int(interleaved), *heads, DTYPES[q.dtype], *w, eps, *table, _dense_heads(out_q, sizes, sizes[2]),
        _dense_heads(out_k, sizes, sizes[3]), None if status is None else status.data_ptr(), _raw_stream(index)), name)
    return out_q, out_k


def qk_rotary_backward(dq: torch.Tensor, dk: torch.Tensor, q: torch.Tensor, k: torch.Tensor,
                       cos: Optional[torch.Tensor] = None, sin: Optional[torch.Tensor] = None,
                       positions: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                       k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, interleaved: bool = False,
                       params: bool = True, status: Optional[torch.Tensor] = None, stream=None):
    """(q's gradient, k's, q_weight's, k_weight's) of qk_rotary_forward from its results' (dq, dk) and its operands.
    The first two have q's type, the weights' are float32 [dim] (of a weight that is None: as for one of ones), or
    None without ``params``."""
    name = "qk_rotary_backward"
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dtype not in DTYPES:
        _refuse(name, q, None, None)
    index, dev = q.get_device(), q.device
    if stream is not None or index != _current():
        with _elsewhere(index, stream, dq, dk, q, k, cos, sin, positions, q_weight, k_weight, status):
            return qk_rotary_backward(dq, dk, q, k, cos, sin, positions, q_weight, k_weight, eps, interleaved, params,
                                      status)
    sizes, heads, w, table, held = _qk_common(name, q, k, cos, sin, positions, q_weight, k_weight, status)
    grads = []
    for d, t in ((dq, q), (dk, k)):
        if isinstance(d, torch.Tensor) and d.shape != t.shape:
            raise ValueError(f"{name}: a gradient has another shape than its operand")
        found = _heads(name, d, q.dtype, index)
        grads.append((found[0], found[-1]))
    out_q, out_k = _dense_like(q, dev), _dense_like(k, dev)
    lib = load_library()
    dwq = dwk = ws = None
    ws_bytes = 0
    if params:
        ws_bytes = _size("layer_qk_workspace_bytes", *sizes[:5])
        dwq, dwk = _empty(sizes[4], dtype=_F32, device=dev), _empty(sizes[4], dtype=_F32, device=dev)
        ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    _done(lib.layer_qk_backward(
        *sizes, int(interleaved), grads[0][0], grads[1][0], *heads, DTYPES[q.dtype], *w, eps, *table,
        _dense_heads(out_q, sizes, sizes[2]), _dense_heads(out_k, sizes, sizes[3]), ptr(dwq), ptr(dwk), ptr(status),
        ptr(ws), ws_bytes, _raw_stream(index)), name)
    return out_q, out_k, dwq, dwk


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


_ACTS = {"silu": 0, "gelu": 1}


def _ffn_weight(name, w, size, groups):
    """(layer_matrix, what has to live until the call, transposed, rows, cols as stored, the bits of its 16-byte units)."""
    rows, cols = w.shape[-2:]
    if w.is_contiguous():
        swapped = False
    else:
        step = w.stride()
        if step[-2] != 1 or step[-1] != rows or (len(step) == 3 and step[0] != rows * cols):
            w, _, rows, cols, ld, stride, swapped = _matrices(name, w)
            at = w.data_ptr()
            return layer_matrix(at, ld, stride, swapped), w, swapped, rows, cols, at | ld * size | (groups > 1) * stride * size
        swapped, rows, cols = True, cols, rows
    at = w.data_ptr()
    return layer_matrix(at, cols, rows * cols, swapped), w, swapped, rows, cols, at | cols * size


def _ffn_common(name, x, weights, offsets, act, status):
    """Checks what both passes take: (rows, hidden, width, groups), x and its leading dimension, the weights as
    _ffn_weight finds them, which of them (gate: 0, up: 1) was copied into the other's order, offsets, the bits of the
    16-byte units of all of these."""
    index, dtype, size = x.get_device(), x.dtype, x.element_size()
    if act not in _ACTS:
        raise ValueError(f"{name}: act is one of {', '.join(_ACTS)}")
    if x.dim() < 1:
        raise ValueError(f"{name}: needs at least one dimension")
    hidden, groups, dims = x.shape[-1], 1, 2
    if offsets is not None:
        _operand(name, offsets, _I32, x.device)
        if offsets.dim() != 1 or offsets.numel() < 2:
            raise ValueError(f"{name}: offsets need groups + 1 elements")
        offsets = offsets.contiguous()
        groups, dims = offsets.numel() - 1, 3
    for w in weights:
        if not isinstance(w, torch.Tensor) or w.get_device() != index or w.dtype is not dtype:
            _operand(name, w, dtype, x.device)
        if w.dim() != dims or (dims == 3 and w.shape[0] != groups):
            raise ValueError(f"{name}: needs a matrix of each weight" + ("" if offsets is None else " for each group"))
    gate, up, down = weights
    shape = gate.shape
    width = shape[-1]
    if shape[-2] != hidden or up.shape != shape or down.shape[-2] != width or down.shape[-1] != hidden:
        raise ValueError(f"{name}: weights of shapes {tuple(shape)}, {tuple(up.shape)}, {tuple(down.shape)} do not "
                         f"fit rows of {hidden}")
    if not 1 <= hidden <= 65536 or not 1 <= width <= 65536 or groups > 1024:
        raise ValueError(f"{name}: hidden and width of 1 to 65536 and at most 1024 groups")
    found = [_ffn_weight(name, w, size, groups) for w in weights]
    turned = None
    if found[0][2] != found[1][2]:  # of two orders: a row-major copy of the other one, whose gradient is turned back
        turned = 0 if found[0][2] else 1
        found[turned] = _ffn_weight(name, weights[turned].contiguous(), size, groups)
    if status is not None:
        _operand(name, status, _I32, x.device)
    x, rows, ld = _rows(x)
    units = x.data_ptr() | ld * size | found[0][5] | found[1][5] | found[2][5]
    return (rows, hidden, width, groups), x, ld, found, turned, offsets, units


def ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                offsets: Optional[torch.Tensor] = None, act: str = "silu", keep: bool = False,
                status: Optional[torch.Tensor] = None, stream=None):
    """A gated feed-forward block act(x w_gate) * (x w_up) w_down of rows x [..., hidden]: (y, pre). Weights of x's
    type, row- or column-major (w_gate and w_up of different orders: the column-major one is copied in each call): w_gate
    and w_up [hidden, width], w_down [width, hidden]; with offsets (int32
    [groups + 1]) a matrix of each for every group, of which group g has the rows offsets[g] to offsets[g + 1] - 1,
    and rows of no group give 0 (include/layer.h). act: "silu" or "gelu". pre, with ``keep``: what ffn_backward takes of
    this call (float32, in the library's own order), else None. status: an int32 CUDA word that SOAP_STATUS_TIMEOUT
    and SOAP_STATUS_RANGE (offsets that fall or pass the rows) are ORed into."""
    name = "ffn_forward"
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in DTYPES:
        _refuse(name, x, None, None)
    index, dev = x.get_device(), x.device
    if stream is not None or index != _current():
        with _elsewhere(index, stream, x, w_gate, w_up, w_down, offsets, status):
            return ffn_forward(x, w_gate, w_up, w_down, offsets, act, keep, status)
    shape = x.shape
    sizes, x, ld, held, _, offsets, units = _ffn_common(name, x, (w_gate, w_up, w_down), offsets, act, status)
    lib, t = load_library(), DTYPES[x.dtype]
    y = _dense_like(x, dev)
    pre = _empty(_size("layer_ffn_pre_elems", sizes[0], sizes[2], sizes[3]), dtype=_F32, device=dev) if keep else None
    ws_bytes = _size("layer_ffn_workspace_bytes", *sizes, t, units % 16 == 0, 0)
    ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    _done(lib.layer_ffn_forward(
        *sizes, None if offsets is None else offsets.data_ptr(), x.data_ptr(), ld, t, held[0][0], held[1][0],
        held[2][0], _ACTS[act], y.data_ptr(), shape[-1], None if pre is None else pre.data_ptr(),
        None if status is None else status.data_ptr(), ws.data_ptr(), ws_bytes, _raw_stream(index)), name)
    return y, pre


def ffn_backward(dy: torch.Tensor, x: torch.Tensor, pre: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                 w_down: torch.Tensor, offsets: Optional[torch.Tensor] = None, act: str = "silu", params: bool = True,
                 status: Optional[torch.Tensor] = None, stream=None):
    """(dx, dw_gate, dw_up, dw_down) of ffn_forward from y's gradient, the call's operands and its pre. All have x's
    type, the weights' gradients their weights' shapes and orders (None without ``params``)."""
    name = "ffn_backward"
    if not isinstance(x, torch.Tensor) or not x.is_cuda or x.dtype not in DTYPES:
        _refuse(name, x, None, None)
    index, dev = x.get_device(), x.device
    if stream is not None or index != _current():
        with _elsewhere(index, stream, dy, x, pre, w_gate, w_up, w_down, offsets, status):
            return ffn_backward(dy, x, pre, w_gate, w_up, w_down, offsets, act, params, status)
    shape = x.shape
    sizes, x, ld, held, turned, offsets, units = _ffn_common(name, x, (w_gate, w_up, w_down), offsets, act, status)
    _operand(name, dy, x.dtype, dev)
    if dy.shape != shape:
        raise ValueError(f"{name}: dy and x have different shapes")
    dy, _, ld_dy = _rows(dy)
    lib, t = load_library(), DTYPES[x.dtype]
    _operand(name, pre, _F32, dev)
    if pre.numel() != _size("layer_ffn_pre_elems", sizes[0], sizes[2], sizes[3]) or not pre.is_contiguous():
        raise ValueError(f"{name}: pre is of another call")
    dx = _dense_like(x, dev)
    grads, out = [None] * 3, [None] * 3
    if params:
        # in the order in which its weight lies: stored [groups, rows, cols], seen transposed if that is column-major
        made = [_empty(((sizes[3],) if offsets is not None else ()) + f[3:5], dtype=x.dtype, device=dev) for f in held]
        grads = [layer_matrix(g.data_ptr(), f[4], f[3] * f[4], f[2]) for g, f in zip(made, held)]
        out = [g.mT if f[2] else g for g, f in zip(made, held)]
    units |= dy.data_ptr() | ld_dy * dy.element_size()
    ws_bytes = _size("layer_ffn_workspace_bytes", *sizes, t, units % 16 == 0, 1)
    ws = _empty(ws_bytes, dtype=torch.uint8, device=dev)
    _done(lib.layer_ffn_backward(
        *sizes, None if offsets is None else offsets.data_ptr(), dy.data_ptr(), ld_dy, x.data_ptr(), ld, t,
        held[0][0], held[1][0], held[2][0], _ACTS[act], pre.data_ptr(), dx.data_ptr(), shape[-1], *grads,
        None if status is None else status.data_ptr(), ws.data_ptr(), ws_bytes, _raw_stream(index)), name)
    if params and turned is not None:
        out[turned] = made[turned].mT.contiguous().mT
    return dx, *out
