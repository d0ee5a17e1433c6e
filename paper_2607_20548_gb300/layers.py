"""Binding of the stand-alone operators of a training step: layer norm and expert routing, forward and
backward (include/layer.h), and the orthogonalisation of a momentum (include/muon.h).

Argument checks and marshalling only, as in ``soap``: outputs and workspaces are allocated here
with torch, on the operands' device, and everything is computed by libsoap.so on the given stream
(the current one by default). A tensor that the caller made on another stream has to be ordered
before the call by the caller, as for any stream-ordered work.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import NamedTuple, Optional

import torch

from .soap import DTYPES, SOAP_OK, SoapError, _stream, load_library


def _operand(name, t, dtype=None, device=None):
    """Checks a CUDA tensor of a supported (or the given) type on the given device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA tensor")
    if t.dtype != dtype if dtype is not None else t.dtype not in DTYPES:
        raise TypeError(f"{name}: expected {dtype or 'float32, bfloat16 or float16'}, got {t.dtype}")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


def _rows(name, t):
    """(tensor, rows, width, leading dimension) of [..., width] seen as rows; a copy only where no
    single leading dimension describes it."""
    if t.dim() < 1:
        raise ValueError(f"{name}: needs at least one dimension")
    width = t.shape[-1]
    if t.is_contiguous():
        return t, t.numel() // max(1, width), width, width
    if t.dim() == 2 and (t.stride(1) == 1 or width == 1) and t.stride(0) >= width:
        return t, t.shape[0], width, t.stride(0)
    t = t.contiguous()
    return t, t.numel() // max(1, width), width, width


def _vector(name, t, n, device):
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name}: expected {n} contiguous elements")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on(dev, stream):
    """Where a call runs and allocates: the operands' device, and the given stream (outputs and workspaces
    then come from that stream's memory pool; None: the current stream)."""
    if stream is not None:
        if torch.device(stream.device).index != dev.index:
            raise ValueError(f"stream of {stream.device} given for work on {dev}")
        return torch.cuda.stream(stream)
    return contextlib.nullcontext() if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def _done(code, name):
    if code != SOAP_OK:
        raise SoapError(code, name)


def _weight_type(name, x, weight, bias, width):
    wt = None
    for what, t in (("weight", weight), ("bias", bias)):
        if t is None:
            continue
        _operand(f"{name} {what}", t)
        _vector(f"{name} {what}", t, width, x.device)
        if t.dtype not in (torch.float32, x.dtype) or (wt is not None and t.dtype != wt):
            raise TypeError(f"{name}: weight and bias must both be float32 or both {x.dtype}")
        wt = t.dtype
    return DTYPES[wt if wt is not None else torch.float32]


def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                       eps: float = 1e-5, stream=None):
    """Layer norm over x's last dimension: (y, mean, rstd), with y of x's shape and type and the fp32
    statistics of every row, which the backward pass takes. weight and bias: float32 or x's type."""
    name = "layer_norm_forward"
    _operand(name, x)
    with _on(x.device, stream):
        x, rows, width, ld = _rows(name, x)
        if width < 1:
            raise ValueError(f"{name}: the normalised dimension is empty")
        wt = _weight_type(name, x, weight, bias, width)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stats = torch.empty((2,) + x.shape[:-1], dtype=torch.float32, device=x.device)
        mean, rstd = stats[0], stats[1]
        _done(load_library().layer_norm_forward(rows, width, x.data_ptr(), ld, DTYPES[x.dtype], _ptr(weight), _ptr(bias),
                                                wt, eps, y.data_ptr(), width, mean.data_ptr(), rstd.data_ptr(),
                                                _stream(None, x.device)), name)
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        weight: Optional[torch.Tensor] = None, params: bool = True, stream=None):
    """(dx, dweight, dbias) of layer_norm_forward from dy and its mean and rstd. dx has x's type;
    dweight and dbias are float32 (the optimizer's gradient type), or None without ``params``."""
    name = "layer_norm_backward"
    _operand(name, x)
    dev = x.device
    _operand(f"{name} dy", dy, x.dtype, dev)
    if dy.shape != x.shape:
        raise ValueError(f"{name}: dy and x have different shapes")
    with _on(dev, stream):
        x, rows, width, ld = _rows(name, x)
        dy, _, _, ld_dy = _rows(name, dy)
        if width < 1:
            raise ValueError(f"{name}: the normalised dimension is empty")
        for what, t in (("mean", mean), ("rstd", rstd)):
            _operand(f"{name} {what}", t, torch.float32, dev)
            if t.numel() != rows or not t.is_contiguous():
                raise ValueError(f"{name}: {what} does not match x's rows")
        wt = _weight_type(name, x, weight, None, width)
        lib = load_library()
        dx = torch.empty(x.shape, dtype=x.dtype, device=dev)
        dw = db = ws = None
        ws_bytes = 0
        if params:
            dwb = torch.empty((2, width), dtype=torch.float32, device=dev)
            dw, db = dwb[0], dwb[1]
            ws_bytes = lib.layer_norm_workspace_bytes(rows, width)
            ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        _done(lib.layer_norm_backward(rows, width, dy.data_ptr(), ld_dy, x.data_ptr(), ld, DTYPES[x.dtype],
                                      mean.data_ptr(), rstd.data_ptr(), _ptr(weight), wt, dx.data_ptr(), width,
                                      _ptr(dw), _ptr(db), _ptr(ws), ws_bytes, _stream(None, dev)), name)
    return dx, dw, db


class Routing(NamedTuple):
    """What route_forward decided: int32 indices and fp32 gates [..., k], int32 counts [experts], fp32
    mean_probs [experts], the fp32 scalar loss and the int32 scalar number of tokens counted (live);
    mask, normalize and coef as given, for route_backward."""
    indices: torch.Tensor
    gates: torch.Tensor
    counts: torch.Tensor
    mean_probs: torch.Tensor
    loss: torch.Tensor
    live: torch.Tensor
    mask: Optional[torch.Tensor]
    normalize: bool
    coef: float


def _mask(name, mask, lead, dev):
    if mask is None:
        return None
    _operand(f"{name} mask", mask, torch.bool, dev)
    if mask.shape != lead:
        raise ValueError(f"{name}: the mask needs one value per token")
    return mask.contiguous()


def route_forward(logits: torch.Tensor, k: int, mask: Optional[torch.Tensor] = None, normalize: bool = True,
                  coef: float = 0.01, status: Optional[torch.Tensor] = None, stream=None) -> Routing:
    """A router's choice of k experts per token from logits [..., experts], with per-expert counts and the
    balance loss (include/layer.h). mask: bool per token, False = left out. status: an int32 CUDA word that
    SOAP_STATUS_NONFINITE is ORed into."""
    name = "route_forward"
    _operand(name, logits)
    lead, dev = logits.shape[:-1], logits.device
    if status is not None:
        _operand(f"{name} status", status, torch.int32, dev)
    lib = load_library()
    k = int(k)
    with _on(dev, stream):
        z, tokens, experts, ld = _rows(name, logits)
        mask = _mask(name, mask, lead, dev)
        ws_bytes = lib.layer_route_workspace_bytes(tokens, experts)
        if ws_bytes == 0 or not 1 <= k <= min(experts, 32):
            raise ValueError(f"{name}: needs 1 to 1024 experts and k of 1 to min(experts, 32)")
        n = tokens * k
        # one allocation for the fp32 outputs and one for the int32 ones
        out_f = torch.empty(n + experts + 1, dtype=torch.float32, device=dev)
        out_i = torch.empty(n + experts + 1, dtype=torch.int32, device=dev)
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        gates, indices = out_f[:n].view(lead + (k,)), out_i[:n].view(lead + (k,))
        mean_probs, loss = out_f[n:n + experts], out_f[n + experts]
        counts, live = out_i[n:n + experts], out_i[n + experts]
        _done(lib.layer_route_forward(tokens, experts, k, z.data_ptr(), ld, DTYPES[z.dtype], _ptr(mask),
                                      int(normalize), coef, indices.data_ptr(), gates.data_ptr(), counts.data_ptr(),
                                      live.data_ptr(), mean_probs.data_ptr(), loss.data_ptr(), _ptr(status),
                                      ws.data_ptr(), ws_bytes, _stream(None, dev)), name)
    return Routing(indices, gates, counts, mean_probs, loss, live, mask, bool(normalize), float(coef))


def route_backward(logits: torch.Tensor, routing: Routing, dgates: Optional[torch.Tensor] = None, dloss: float = 1.0,
                   stream=None) -> torch.Tensor:
    """dlogits (logits' shape and type) from the gates' gradient (fp32, None for zero) and the loss's."""
    name = "route_backward"
    _operand(name, logits)
    dev, k, experts = logits.device, routing.indices.shape[-1], logits.shape[-1]
    if routing.indices.shape[:-1] != logits.shape[:-1] or routing.counts.shape[0] != experts:
        raise ValueError(f"{name}: the routing is of other logits")
    if routing.indices.device != dev:
        raise ValueError(f"{name}: the routing is on {routing.indices.device}, the logits on {dev}")
    if dgates is not None:
        _operand(f"{name} dgates", dgates, torch.float32, dev)
        if dgates.shape != routing.gates.shape:
            raise ValueError(f"{name}: dgates needs the gates' shape")
    with _on(dev, stream):
        z, tokens, _, ld = _rows(name, logits)
        dgates = None if dgates is None else dgates.contiguous()
        dz = torch.empty(z.shape, dtype=z.dtype, device=dev)
        _done(load_library().layer_route_backward(
            tokens, experts, k, z.data_ptr(), ld, DTYPES[z.dtype], _ptr(routing.mask), int(routing.normalize),
            routing.coef, dloss, routing.indices.data_ptr(), routing.counts.data_ptr(), routing.live.data_ptr(),
            _ptr(dgates), dz.data_ptr(), experts, _stream(None, dev)), name)
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
    _operand(name, M)
    dev = M.device
    if status is not None:
        _operand(f"{name} status", status, torch.int32, dev)
    flat = None
    if coeffs is not None:
        ns_steps = len(coeffs)
        flat = (ctypes.c_float * (3 * ns_steps))(*[float(x) for abc in coeffs for x in abc])
    with _on(dev, stream):
        M, batch, rows, cols, ld, stride, swapped = _matrices(name, M)
        lead = M.shape[:-2]
        if M.numel() == 0:
            return torch.empty_like(M)
        out = torch.empty(lead + (rows, cols), dtype=M.dtype, device=dev)
        lib = load_library()
        ws_bytes = lib.muon_orthogonalize_workspace_bytes(batch, rows, cols, DTYPES[M.dtype])
        if ws_bytes == 0:
            raise ValueError(f"{name}: sides of 1 to 65536, fewer than 2^31 elements and 65536 matrices")
        ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev)
        _done(lib.muon_orthogonalize(batch, rows, cols, M.data_ptr(), ld, stride, DTYPES[M.dtype], flat, ns_steps, eps,
                                     out.data_ptr(), cols, rows * cols, ws.data_ptr(), ws_bytes, _ptr(status),
                                     _stream(None, dev)), name)
    return out.mT if swapped else out
