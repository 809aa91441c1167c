"""The operators around the layers of a language model on PyTorch tensors: embedding, norms of a block, clipping by the norm of all gradients.

The manner is that of lm_ops.py: one function for each C entry point of include/netmax.h, with the same name; tensors on one GPU, outputs that are not given are allocated, work on the
tensors' device and its current stream, nothing recorded for automatic differentiation."""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional, Sequence

import torch

from .binding import (NETMAX_GATE_NONE, NETMAX_GATE_SIGMOID, NETMAX_GATE_TANH, NETMAX_NORM_LAYER, NETMAX_NORM_RMS, load, netmax_block_norm_data, netmax_block_norm_grads,
                      netmax_block_norm_shape, netmax_embed_shape, netmax_gradient)
from .lm_ops import _DTYPES, _call, _changed, _check_tensor, _first, _no_graph, _p, _refuse, _strides, _workspace

NORMS = {"rms": NETMAX_NORM_RMS, "layer": NETMAX_NORM_LAYER}
GATES = {"none": NETMAX_GATE_NONE, "sigmoid": NETMAX_GATE_SIGMOID, "tanh": NETMAX_GATE_TANH}


def _one_of(name: str, value: str, known: dict) -> int:
    if value not in known:
        _refuse(f"unknown {name} {value!r}: one of {', '.join(known)}")
    return known[value]


# ---- embedding ---------------------------------------------------------------------------------------------------------

def _ids(tokens, like: torch.Tensor):
    """(tokens of each table, distance of the batch's)."""
    lead = like.dim() - 2
    if not isinstance(tokens, torch.Tensor) or tokens.dim() != 1 + lead:
        _refuse("tokens must have one dimension for one table, two for a batch of them")
    shape = (*like.shape[:lead], tokens.shape[-1])
    _check_tensor("tokens", tokens, like, shape, torch.int32)
    return shape[-1], tokens.stride(0) if lead else 0


def netmax_embed(tokens, table, *, scale: float = 1.0, y=None):
    """y = scale table[tokens].  table [vocab, width] and tokens int32 [n], or [batch, vocab, width] and [batch, n] with a table each; tokens outside of the
    vocabulary are padding, with rows of zeros."""
    _first("table", table, (2, 3))
    n, s_ids = _ids(tokens, table)
    lead, (vocab, width) = tuple(table.shape[:-2]), table.shape[-2:]
    if not table.is_contiguous():
        _check_tensor("table", table, table, table.shape, table.dtype)
    given = y
    if y is None:
        y = torch.empty((*lead, n, width), dtype=table.dtype, device=table.device)
    else:
        _check_tensor("y", y, table, (*lead, n, width), table.dtype)
    ldt, st = _strides(table)
    ldy, sy = _strides(y)
    shape = netmax_embed_shape(lead[0] if lead else 1, n, vocab, width, _DTYPES[table.dtype], 0, scale, s_ids, ldt, st, ldy, sy)
    _call(load().netmax_embed, table.device, C.byref(shape), _p(tokens), _p(table), _p(y))
    _changed(given)
    return y


def netmax_embed_grad(dy, tokens, vocab: Optional[int] = None, *, scale: float = 1.0, accumulate: bool = False, dtable=None):
    """The gradient of `netmax_embed`'s table from dy [n, width] or [batch, n, width]; vocab, or the memory dtable, says how many rows it has.  accumulate: added to
    what dtable holds, whose other rows are not touched."""
    _first("dy", dy, (2, 3))
    n, s_ids = _ids(tokens, dy)
    lead, width, given = tuple(dy.shape[:-2]), dy.shape[-1], dtable
    if dy.shape[-2] != n:
        _refuse(f"dy has {dy.shape[-2]} rows for {n} tokens")
    if not dy.is_contiguous():
        _check_tensor("dy", dy, dy, dy.shape, dy.dtype)
    if dtable is not None:
        if not isinstance(dtable, torch.Tensor) or dtable.dim() != dy.dim():
            _refuse("dtable must have as many dimensions as dy")
        if vocab is None:
            vocab = dtable.shape[-2]
        _check_tensor("dtable", dtable, dy, (*lead, vocab, width), dy.dtype)
    elif accumulate:
        _refuse("accumulate needs dtable")
    elif vocab is None:
        _refuse("vocab or dtable is needed")
    else:
        dtable = torch.empty((*lead, vocab, width), dtype=dy.dtype, device=dy.device)
    ldt, st = _strides(dtable)
    ldy, sy = _strides(dy)
    shape = netmax_embed_shape(lead[0] if lead else 1, n, vocab, width, _DTYPES[dy.dtype], int(bool(accumulate)), scale, s_ids, ldt, st, ldy, sy)
    lib, ref = load(), C.byref(shape)
    work = _workspace(lib.netmax_embed_grad_workspace(ref), dy.device)
    _call(lib.netmax_embed_grad, dy.device, ref, _p(tokens), _p(dy), _p(dtable), _p(work), 0 if work is None else work.numel())
    _changed(given)
    return dtable


# ---- norms of a block ----------------------------------------------------------------------------------------------------

class BlockNormGrads(NamedTuple):
    """The gradients that `netmax_block_norm_grad` returns, None for what is not there or not needed."""
    dx: Optional[torch.Tensor]
    df: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost_gain: Optional[torch.Tensor]
    dpost_bias: Optional[torch.Tensor]
    dpre_gain: Optional[torch.Tensor]
    dpre_bias: Optional[torch.Tensor]


_NOTHING = (0, 0, 0)


def _rows(name, t, x, shape, dtype):
    if t is None:
        return _NOTHING
    _check_tensor(name, t, x, shape, dtype)
    s = t.stride()
    return (t.data_ptr(), s[0], 0) if len(s) == 2 else (t.data_ptr(), s[1], s[0])


def _vector(name, t, x, shape, dtype):
    if t is None:
        return _NOTHING
    _check_tensor(name, t, x, shape, dtype)
    return t.data_ptr(), 0, t.stride(0) if len(shape) == 2 else 0


def _operands(x, f, gate, post_gain, post_bias, pre_gain, pre_bias):
    """Their spans, whether the gate has rows of its own, and the shapes of rows and vectors."""
    _first("x", x, (2, 3))
    rows, dt = x.shape, x.dtype
    vector = (*rows[:-2], rows[-1])
    gate_rows = isinstance(gate, torch.Tensor) and gate.dim() == x.dim()
    return ((*_rows("x", x, x, rows, dt), *_rows("f", f, x, rows, dt), *(_rows if gate_rows else _vector)("gate", gate, x, rows if gate_rows else vector, dt),
             *_vector("post_gain", post_gain, x, vector, dt), *_vector("post_bias", post_bias, x, vector, dt), *_vector("pre_gain", pre_gain, x, vector, dt),
             *_vector("pre_bias", pre_bias, x, vector, dt)), gate_rows, rows, vector)


def _norm_shape(x, norm, gate_act, gate_rows, post, pre, x_scale, f_scale, eps):
    return netmax_block_norm_shape(x.shape[0] if x.dim() == 3 else 1, x.shape[-2], x.shape[-1], _DTYPES[x.dtype], _one_of("norm", norm, NORMS), _one_of("gate_act", gate_act, GATES),
                                   gate_rows, bool(post), bool(pre), x_scale, f_scale, eps)


def netmax_block_norm(x, f=None, gate=None, post_gain=None, post_bias=None, pre_gain=None, pre_bias=None, *, norm: str = "rms", post: bool = True, pre: bool = True,
                      gate_act: str = "none", x_scale: float = 1.0, f_scale: float = 1.0, eps: float = 1e-6, need_h: bool = True, h=None, y=None):
    """(h, y) with h = x_scale x + f_scale act(gate) (N(f) post_gain + post_bias), y = N(h) pre_gain + pre_bias; N: "rms" or "layer".
    x and f [rows, width], or [batch, rows, width] with vectors of their own each; gate [rows, width] or, the same for all rows, [width]; gains and biases [width].
    Without f, y = N(x_scale x) pre_gain + pre_bias, and h is None unless memory for it is given.  post=False: f is not normed; pre=False: y is None."""
    spans, gate_rows, rows, _ = _operands(x, f, gate, post_gain, post_bias, pre_gain, pre_bias)
    shape, given = _norm_shape(x, norm, gate_act, gate_rows, post, pre, x_scale, f_scale, eps), (h, y)
    if h is None and f is not None and need_h:
        h = torch.empty(rows, dtype=x.dtype, device=x.device)
    if y is None and pre:
        y = torch.empty(rows, dtype=x.dtype, device=x.device)
    data = netmax_block_norm_data(*spans, *_rows("h", h, x, rows, x.dtype), *_rows("y", y, x, rows, x.dtype))
    _call(load().netmax_block_norm, x.device, C.byref(shape), data)
    _changed(*given)
    return h, y


def netmax_block_norm_grad(dy, dh, x, f=None, gate=None, post_gain=None, post_bias=None, pre_gain=None, pre_bias=None, *, norm: str = "rms", post: bool = True,
                           pre: bool = True, gate_act: str = "none", x_scale: float = 1.0, f_scale: float = 1.0, eps: float = 1e-6, need_input: bool = True,
                           need_params: bool = True, dx=None, df=None, dgate=None, dpost_gain=None, dpost_bias=None, dpre_gain=None, dpre_bias=None) -> BlockNormGrads:
    """The gradients of `netmax_block_norm`, called with the same operands and options, from dy and dh (None: nothing reaches h but through y).  need_input: dx, df and the
    gradient of a gate of rows; need_params: those of gains, biases and a gate that is the same for all rows, summed over the rows."""
    spans, gate_rows, rows, vector = _operands(x, f, gate, post_gain, post_bias, pre_gain, pre_bias)
    shape, dt, dev = _norm_shape(x, norm, gate_act, gate_rows, post, pre, x_scale, f_scale, eps), x.dtype, x.device
    given = (dx, df, dgate, dpost_gain, dpost_bias, dpre_gain, dpre_bias)

    def output(t, of, needed, like):
        return torch.empty(like, dtype=dt, device=dev) if t is None and of is not None and needed else t

    dx, df = output(dx, x, need_input, rows), output(df, f, need_input, rows)
    dgate = output(dgate, gate, need_input, rows) if gate_rows else output(dgate, gate, need_params, vector)
    dpost_gain, dpost_bias, dpre_gain, dpre_bias = (output(t, of, need_params, vector) for t, of in ((dpost_gain, post_gain), (dpost_bias, post_bias), (dpre_gain, pre_gain), (dpre_bias, pre_bias)))
    data = netmax_block_norm_data(*spans, *_NOTHING, *_NOTHING)
    grads = netmax_block_norm_grads(*_rows("dy", dy, x, rows, dt), *_rows("dh", dh, x, rows, dt), *_rows("dx", dx, x, rows, dt), *_rows("df", df, x, rows, dt),
                                    *(_rows if gate_rows else _vector)("dgate", dgate, x, rows if gate_rows else vector, dt), *_vector("dpost_gain", dpost_gain, x, vector, dt),
                                    *_vector("dpost_bias", dpost_bias, x, vector, dt), *_vector("dpre_gain", dpre_gain, x, vector, dt), *_vector("dpre_bias", dpre_bias, x, vector, dt))
    lib, ref = load(), C.byref(shape)
    work = _workspace(lib.netmax_block_norm_grad_workspace(ref, data, grads), dev)
    _call(lib.netmax_block_norm_grad, dev, ref, data, grads, _p(work), 0 if work is None else work.numel())
    _changed(*given)
    return BlockNormGrads(dx, df, dgate, dpost_gain, dpost_bias, dpre_gain, dpre_bias)


# ---- clipping ------------------------------------------------------------------------------------------------------------

class Gradients:
    """Where a model's gradients lie, for `netmax_grad_norm` and `netmax_clip_grads`: a program whose gradients stay in the same memory lays the list out once.

    tensors: float32 or bfloat16, of any shapes, rows at one distance, on one GPU; batch: their first dimension counts models (workers), which have a norm each.  out: where the scaled
    gradients go, of the same shapes and types; None: in place.  The tensors are kept alive; one that is moved to other memory is noticed and refused."""

    def __init__(self, tensors: Sequence[torch.Tensor], *, out: Optional[Sequence[torch.Tensor]] = None, batch: bool = False):
        self.tensors = list(tensors)
        self.out = self.tensors if out is None else list(out)
        if not self.tensors:
            _refuse("there are no gradients")
        if len(self.out) != len(self.tensors):
            _refuse(f"{len(self.out)} outputs for {len(self.tensors)} gradients")
        first = self.tensors[0]
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            _refuse("gradients must be tensors on the GPU")
        self.device, self.batch = first.device, bool(batch)
        if batch and first.dim() == 0:
            _refuse("gradients of a batch need a first dimension")
        self.models = first.shape[0] if batch else 1
        self.entries = (netmax_gradient * len(self.tensors))()
        for e, g, o in zip(self.entries, self.tensors, self.out):
            rows, cols, e.ldg, e.sg = self._place(g, "a gradient")
            if o is not g:
                if not isinstance(o, torch.Tensor) or o.shape != g.shape or o.dtype != g.dtype:
                    _refuse("an output must be a tensor of its gradient's shape and type")
            e.ldo, e.so = self._place(o, "an output")[2:]
            e.g, e.out, e.rows, e.cols, e.dtype = g.data_ptr(), o.data_ptr(), rows, cols, _DTYPES[g.dtype]
        self._all = self.tensors if out is None else self.tensors + self.out
        self._at = [t.data_ptr() for t in self._all]

    def _place(self, t, name):
        """(rows, columns, distance of rows, distance of models)."""
        if not isinstance(t, torch.Tensor) or t.device != self.device:
            _refuse(f"{name} must be a tensor on {self.device}")
        if t.dtype not in _DTYPES:
            _refuse(f"{name} is {t.dtype}: float32 or bfloat16 is needed")
        shape, strides, step = list(t.shape), list(t.stride()), 0
        if self.batch:
            if not shape or shape[0] != self.models:
                _refuse(f"{name} has the shape {tuple(t.shape)} in a batch of {self.models}")
            step = strides[0]
            shape, strides = shape[1:], strides[1:]
        if not shape:
            return 1, 1, 1, step
        if 0 in shape:
            return 0, 0, 0, step
        if strides[-1] != 1 and shape[-1] > 1:
            _refuse(f"the values of a row of {name} must lie next to each other")
        rows, ld = 1, shape[-1]
        for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):      # from the last dimension on: rows at one distance
            if n == 1:
                continue
            if rows == 1:
                ld = s
            elif s != rows * ld:
                _refuse(f"the rows of {name} must lie at one distance")
            rows *= n
        return rows, shape[-1], ld, step

    def _ready(self):
        if [t.data_ptr() for t in self._all] != self._at:
            _refuse("a gradient has moved since the list was laid out")
        if torch.is_grad_enabled() and any(t.requires_grad for t in self._all):
            _no_graph("a gradient")

    def _run(self, max_norm: Optional[float]):
        self._ready()
        lib, dev, n = load(), self.device, len(self.tensors)
        norm = torch.empty(self.models if self.batch else (), dtype=torch.float32, device=dev)
        work = _workspace(lib.netmax_grad_norm_workspace(self.models, n, self.entries), dev)
        size = 0 if work is None else work.numel()
        if max_norm is None:
            _call(lib.netmax_grad_norm, dev, self.models, n, self.entries, _p(norm), _p(work), size)
        else:
            _call(lib.netmax_clip_grads, dev, self.models, n, self.entries, max_norm, _p(norm), _p(work), size)
            torch.autograd.graph.increment_version(self.out)
        return norm


def _gradients(gradients, out, batch) -> Gradients:
    if not isinstance(gradients, Gradients):
        return Gradients(gradients, out=out, batch=batch)
    if out is not None or batch:
        _refuse("out and batch are given to Gradients")
    return gradients


def netmax_grad_norm(gradients, *, batch: bool = False):
    """The norm of all gradients together, a tensor of float32 (one number; with batch one for each model).  gradients: a `Gradients` or a sequence of tensors."""
    return _gradients(gradients, None, batch)._run(None)


def netmax_clip_grads(gradients, max_norm: float, *, out: Optional[Sequence[torch.Tensor]] = None, batch: bool = False):
    """Scales the gradients down to max_norm where their norm is larger, in place or into out, and returns the norm that they had."""
    return _gradients(gradients, out, batch)._run(max_norm)
