"""The operators for language models on PyTorch tensors: one function for each C entry point of include/netmax.h, with the same name.

Tensors live on one GPU, with the values of a row next to each other (any distance between rows and matrices); outputs that are not given
are allocated.  The work is enqueued on the tensors' device, on its current stream; workspaces come from torch's allocator on that stream.

Gradients are calls of their own (`netmax_linear_grad`; the losses return theirs), and nothing is recorded for torch's automatic differentiation: tensors
that require a gradient are refused while it records, rather than left without one.  Memory that a call writes counts as changed in place."""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from .binding import (NETMAX_ACT_GELU, NETMAX_ACT_NONE, NETMAX_ACT_RELU, NETMAX_ACT_SILU, NETMAX_BF16, NETMAX_EINVAL, NETMAX_F32, NETMAX_OK, NetmaxError,
                      _check, load, netmax_linear_shape, netmax_orth_shape)

ACTIVATIONS = {"none": NETMAX_ACT_NONE, "relu": NETMAX_ACT_RELU, "gelu": NETMAX_ACT_GELU, "silu": NETMAX_ACT_SILU}
_DTYPES = {torch.float32: NETMAX_F32, torch.bfloat16: NETMAX_BF16}


def _refuse(text: str):
    raise NetmaxError(NETMAX_EINVAL, text)


def _no_graph(name: str):
    if torch.is_grad_enabled():
        _refuse(f"{name} requires a gradient, which this call does not record: call it under torch.no_grad() or with a detached tensor")


def _check_tensor(name: str, t, like: torch.Tensor, shape: Tuple[int, ...], dtype: torch.dtype) -> torch.Tensor:
    # what is right takes one look; what is wrong is looked at closely
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == like.get_device() and t.shape == shape and (t.is_contiguous() or t.stride(-1) == 1 or t.shape[-1] <= 1):
        if t.requires_grad:
            _no_graph(name)
        return t
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} must be a tensor")
    if t.device != like.device:
        _refuse(f"{name} is on {t.device}, not on {like.device}")
    if t.dtype != dtype:
        _refuse(f"{name} is {t.dtype}, not {dtype}")
    if t.shape != shape:
        _refuse(f"{name} has the shape {tuple(t.shape)}, not {tuple(shape)}")
    _refuse(f"the values of a row of {name} must lie next to each other")


def _first(name: str, t, dims: Tuple[int, ...]):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a tensor on the GPU")
    if t.dim() not in dims:
        _refuse(f"{name} has {t.dim()} dimensions")
    if t.dtype not in _DTYPES:
        _refuse(f"{name} is {t.dtype}: float32 or bfloat16 is needed")
    if t.requires_grad:
        _no_graph(name)


def _changed(*outputs):
    """The caller's tensors that a call has written, for whoever saved them before."""
    for t in outputs:
        if t is not None:
            torch.autograd.graph.increment_version(t)


def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _strides(t: Optional[torch.Tensor]) -> Tuple[int, int]:
    """(distance of rows, distance of matrices) of a 2- or 3-dimensional tensor."""
    if t is None:
        return 0, 0
    s = t.stride()
    return (s[0], 0) if len(s) == 2 else (s[1], s[0])


try:
    _stream = torch._C._cuda_getCurrentRawStream                # the handle alone: a tenth of the time that a Stream object takes
except AttributeError:
    def _stream(index: int) -> int:
        return torch.cuda.current_stream(index).cuda_stream


def _call(f, device: torch.device, *args):
    """Calls a C entry point with the device's current stream as last argument, with the device current."""
    if device.index == torch.cuda.current_device():
        rc = f(*args, _stream(device.index))
    else:
        with torch.cuda.device(device):
            rc = f(*args, _stream(device.index))
    if rc != NETMAX_OK:
        _check(rc)


def _workspace(n: int, device: torch.device) -> Optional[torch.Tensor]:
    if n < 0:
        _check(NETMAX_EINVAL)
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _act(act: str) -> int:
    if act not in ACTIVATIONS:
        _refuse(f"unknown activation {act!r}: one of {', '.join(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def netmax_linear(x, w, bias=None, residual=None, *, act: str = "none", keep_preact: bool = False, y=None, z=None):
    """y = act(x w + bias) + residual.  x [rows, d_in] and w [d_in, d_out], or [batch, ...] with a layer each; bias [d_out] or [batch, d_out].
    Returns y, with keep_preact (y, z): z = x w + bias is what `netmax_linear_grad` needs unless act is "none"."""
    _first("x", x, (2, 3))
    kind, lead, (rows, d_in) = _act(act), tuple(x.shape[:-2]), x.shape[-2:]
    if not isinstance(w, torch.Tensor) or w.dim() != x.dim():
        _refuse("w must have as many dimensions as x")
    d_out, dt = w.shape[-1], x.dtype
    if not x.is_contiguous():
        _check_tensor("x", x, x, (*lead, rows, d_in), dt)
    _check_tensor("w", w, x, (*lead, d_in, d_out), dt)
    if bias is not None:
        _check_tensor("bias", bias, x, (*lead, d_out), dt)
    if residual is not None:
        _check_tensor("residual", residual, x, (*lead, rows, d_out), dt)
    given = (y, z)
    if y is None:
        y = torch.empty((*lead, rows, d_out), dtype=dt, device=x.device)
    else:
        _check_tensor("y", y, x, (*lead, rows, d_out), dt)
    if z is not None:
        _check_tensor("z", z, x, (*lead, rows, d_out), dt)
    elif keep_preact:
        z = torch.empty((*lead, rows, d_out), dtype=dt, device=x.device)
    ldx, sx = _strides(x)
    ldw, sw = _strides(w)
    ldr, sr = _strides(residual)
    ldy, sy = _strides(y)
    ldz, sz = _strides(z)
    sb = bias.stride(0) if bias is not None and lead else 0
    shape = netmax_linear_shape(lead[0] if lead else 1, rows, d_in, d_out, _DTYPES[dt], kind, ldx, ldw, ldr, ldy, ldz, sx, sw, sb, sr, sy, sz)
    lib, ref = load(), C.byref(shape)
    work = _workspace(lib.netmax_linear_workspace(ref, _p(x), _p(w)), x.device)
    _call(lib.netmax_linear, x.device, ref, _p(x), _p(w), _p(bias), _p(residual), _p(y), _p(z), _p(work), 0 if work is None else work.numel())
    _changed(*given)
    return (y, z) if keep_preact or z is not None else y


def netmax_linear_grad(dy, x, w, z=None, *, act: str = "none", need_input: bool = True, need_weight: bool = True, need_bias: bool = True, dx=None,
                       dw=None, db=None):
    """Gradients (dx, dw, db) of `netmax_linear` from dy, with None in the place of one that is not needed (dy is the residual's)."""
    _first("x", x, (2, 3))
    kind, lead, (rows, d_in) = _act(act), tuple(x.shape[:-2]), x.shape[-2:]
    if not isinstance(w, torch.Tensor) or w.dim() != x.dim():
        _refuse("w must have as many dimensions as x")
    d_out, dt, dev = w.shape[-1], x.dtype, x.device
    _check_tensor("x", x, x, (*lead, rows, d_in), dt)
    _check_tensor("w", w, x, (*lead, d_in, d_out), dt)
    _check_tensor("dy", dy, x, (*lead, rows, d_out), dt)
    if kind != NETMAX_ACT_NONE:
        _check_tensor("z", z, x, (*lead, rows, d_out), dt)
    else:
        z = None

    def output(name, t, needed, shape):
        if t is not None:
            _check_tensor(name, t, x, shape, dt)
            return t
        return torch.empty(shape, dtype=dt, device=dev) if needed else None

    given = (dx, dw, db)
    dx = output("dx", dx, need_input, (*lead, rows, d_in))
    dw = output("dw", dw, need_weight, (*lead, d_in, d_out))
    db = output("db", db, need_bias, (*lead, d_out))
    ldx, sx = _strides(x)
    ldw, sw = _strides(w)
    ldy, sy = _strides(dy)
    ldz, sz = _strides(z)
    lddx, sdx = _strides(dx)
    lddw, sdw = _strides(dw)
    sdb = db.stride(0) if db is not None and lead else 0
    shape = netmax_linear_shape(lead[0] if lead else 1, rows, d_in, d_out, _DTYPES[dt], kind, ldx, ldw, 0, ldy, ldz, sx, sw, 0, 0, sy, sz, lddx, lddw,
                                sdx, sdw, sdb)
    lib, ref = load(), C.byref(shape)
    work = _workspace(lib.netmax_linear_grad_workspace(ref, _p(dy), _p(x), _p(w)), dev)
    _call(lib.netmax_linear_grad, dev, ref, _p(dy), _p(x), _p(w), _p(z), _p(dx), _p(dw), _p(db), _p(work), 0 if work is None else work.numel())
    _changed(*given)
    return dx, dw, db


def netmax_orthogonalize(g, m=None, *, m_out=None, out=None, mu: float = 0.95, nesterov: bool = True, steps: int = 5,
                         coefficients: Tuple[float, float, float] = (3.4445, -4.7750, 2.0315), eps: float = 1e-7, scale: float = 1.0):
    """The orthogonalised momentum step of g [rows, cols] or [batch, rows, cols] (float32 or bfloat16); returns the update, of g's type.
    m: the momentum, float32, brought up to date in place unless m_out is given; None: no momentum."""
    _first("g", g, (2, 3))
    _check_tensor("g", g, g, g.shape, g.dtype)
    if m is not None:
        _check_tensor("m", m, g, g.shape, torch.float32)
        m_out = m if m_out is None else _check_tensor("m_out", m_out, g, g.shape, torch.float32)
        if m_out.stride() != m.stride():
            _refuse("m_out must have the strides of m")
    elif m_out is not None:
        _refuse("m_out without m")
    given = (out, m_out)
    if out is None:
        out = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    else:
        _check_tensor("out", out, g, g.shape, g.dtype)
    ldg, sg = _strides(g)
    ldm, sm = _strides(m)
    ldo, so = _strides(out)
    rows, cols = g.shape[-2:]
    shape = netmax_orth_shape(g.shape[0] if g.dim() == 3 else 1, rows, cols, _DTYPES[g.dtype], steps, int(bool(nesterov)), mu, *coefficients, eps, scale,
                              ldg, sg, ldm, sm, ldo, so)
    lib, ref = load(), C.byref(shape)
    work = _workspace(lib.netmax_orthogonalize_workspace(ref), g.device)
    _call(lib.netmax_orthogonalize, g.device, ref, _p(g), _p(m), _p(m_out), _p(out), _p(work), 0 if work is None else work.numel())
    _changed(*given)
    return out


def _token_rows(logits, labels, weight, grad, need_grad):
    given = grad
    _first("logits", logits, (2,))
    tokens, vocab = logits.shape
    dense = logits.is_contiguous()
    if not dense:
        _check_tensor("logits", logits, logits, logits.shape, logits.dtype)
    _check_tensor("labels", labels, logits, (tokens,), torch.int32)
    if weight is not None:
        _check_tensor("weight", weight, logits, (tokens,), torch.float32)
    if grad is not None:
        _check_tensor("grad", grad, logits, logits.shape, logits.dtype)
    elif need_grad:
        grad = torch.empty_like(logits) if dense else torch.empty((tokens, vocab), dtype=logits.dtype, device=logits.device)
    return tokens, vocab, grad, given


def netmax_policy_loss(logits, labels, old_logp, advantage, weight=None, *, ref_logp=None, clip_low: float = 0.2, clip_high: float = 0.2, kl: float = 0.0,
                       need_grad: bool = True, grad=None):
    """The clipped policy loss of sampled tokens: (loss [tokens], log probabilities [tokens], gradient of the sum of all losses by the logits or None)."""
    tokens, vocab, grad, given = _token_rows(logits, labels, weight, grad, need_grad)
    dev = logits.device
    for name, t in (("old_logp", old_logp), ("advantage", advantage), ("ref_logp", ref_logp)):
        if t is not None or name != "ref_logp":
            _check_tensor(name, t, logits, (tokens,), torch.float32)
    loss, logp = torch.empty_like(old_logp), torch.empty_like(old_logp)
    _call(load().netmax_policy_loss, dev, tokens, vocab, _DTYPES[logits.dtype], _p(logits), logits.stride(0), _p(labels), _p(old_logp), _p(ref_logp),
          _p(advantage), _p(weight), clip_low, clip_high, kl, _p(loss), _p(logp), _p(grad), 0 if grad is None else grad.stride(0))
    _changed(given)
    return loss, logp, grad


def netmax_preference_loss(logits, labels, offsets, weight=None, ref_logp=None, *, beta: float = 0.1, smoothing: float = 0.0,
                           scale: Optional[float] = None, need_grad: bool = True, grad=None):
    """The loss of paired log ratios: (loss [pairs], log ratios [2 pairs], gradient of the sum of all losses by the logits or None).
    offsets: int32 [2 pairs + 1], chosen and rejected sequences in turn; scale defaults to 1 / pairs."""
    tokens, vocab, grad, given = _token_rows(logits, labels, weight, grad, need_grad)
    dev = logits.device
    if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 3 or offsets.shape[0] % 2 == 0:
        _refuse("offsets must hold 2 pairs + 1 numbers, for at least one pair")
    _check_tensor("offsets", offsets, logits, offsets.shape, torch.int32)
    _check_tensor("ref_logp", ref_logp, logits, (tokens,), torch.float32)
    pairs = offsets.shape[0] // 2
    both = torch.empty(3 * pairs, dtype=torch.float32, device=dev)
    loss, ratio = both[:pairs], both[pairs:]
    lib = load()
    work = _workspace(lib.netmax_preference_workspace(tokens, pairs), dev)
    _call(lib.netmax_preference_loss, dev, tokens, vocab, _DTYPES[logits.dtype], _p(logits), logits.stride(0), _p(labels), pairs, _p(offsets), _p(ref_logp),
          _p(weight), beta, smoothing, 1.0 / pairs if scale is None else scale, _p(loss), _p(ratio), _p(grad), 0 if grad is None else grad.stride(0),
          _p(work), 0 if work is None else work.numel())
    _changed(given)
    return loss, ratio, grad
