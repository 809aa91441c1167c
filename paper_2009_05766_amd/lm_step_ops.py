"""The operators around the layers of a language model on PyTorch tensors: embedding, norms of a block, clipping by the norm of all gradients.

The manner is that of lm_ops.py: one function for each C entry point of include/netmax.h, with the same name; tensors on one GPU, outputs that are not given are allocated, work on the
tensors' device and its current stream, nothing recorded for automatic differentiation."""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from array import array
from typing import NamedTuple, Optional, Sequence

import torch

from .binding import (NETMAX_GATE_NONE, NETMAX_GATE_SIGMOID, NETMAX_GATE_TANH, NETMAX_NORM_LAYER, NETMAX_NORM_RMS, NetmaxError, load, netmax_gradient)
from .lm_ops import _DTYPES, _refuse, _stream

NORMS = {"rms": NETMAX_NORM_RMS, "layer": NETMAX_NORM_LAYER}
GATES = {"none": NETMAX_GATE_NONE, "sigmoid": NETMAX_GATE_SIGMOID, "tanh": NETMAX_GATE_TANH}
_ENTRIES = ("netmax_last_error", "netmax_embed", "netmax_embed_grad_workspace", "netmax_embed_grad", "netmax_block_norm", "netmax_block_norm_grad_workspace", "netmax_block_norm_grad",
            "netmax_grad_norm_workspace", "netmax_grad_norm", "netmax_clip_grads")
_calls = None


def _load_calls():
    """The extension module that checks tensors, allocates outputs and calls the C entry points (csrc/lm_calls.cpp); built first only if it is absent."""
    global _calls
    from .build import CALLS, build_calls
    lib = load()
    if not os.path.exists(CALLS):
        build_calls()
    spec = importlib.util.spec_from_file_location("_lm_calls", CALLS)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    module.setup(NetmaxError, _stream, tuple(C.cast(getattr(lib, n), C.c_void_p).value for n in _ENTRIES))
    _calls = module
    return module


def _one_of(name: str, value: str, known: dict) -> int:
    if value not in known:
        _refuse(f"unknown {name} {value!r}: one of {', '.join(known)}")
    return known[value]


def netmax_embed(tokens, table, *, scale: float = 1.0, y=None):
    """y = scale table[tokens].  table [vocab, width] and tokens int32 [n], or [batch, vocab, width] and [batch, n] with a table each; tokens outside of the
    vocabulary are padding, with rows of zeros."""
    return (_calls or _load_calls()).embed(tokens, table, scale, y)


def netmax_embed_grad(dy, tokens, vocab: Optional[int] = None, *, scale: float = 1.0, accumulate: bool = False, dtable=None):
    """The gradient of `netmax_embed`'s table from dy [n, width] or [batch, n, width]; vocab, or the memory dtable, says how many rows it has.  accumulate: added to
    what dtable holds, whose other rows are not touched."""
    return (_calls or _load_calls()).embed_grad(dy, tokens, vocab, scale, accumulate, dtable)


class BlockNormGrads(NamedTuple):
    """The gradients that `netmax_block_norm_grad` returns, None for what is not there or not needed."""
    dx: Optional[torch.Tensor]
    df: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dpost_gain: Optional[torch.Tensor]
    dpost_bias: Optional[torch.Tensor]
    dpre_gain: Optional[torch.Tensor]
    dpre_bias: Optional[torch.Tensor]


def netmax_block_norm(x, f=None, gate=None, post_gain=None, post_bias=None, pre_gain=None, pre_bias=None, *, norm: str = "rms", post: bool = True, pre: bool = True,
                      gate_act: str = "none", x_scale: float = 1.0, f_scale: float = 1.0, eps: float = 1e-6, need_h: bool = True, h=None, y=None):
    """(h, y) with h = x_scale x + f_scale act(gate) (N(f) post_gain + post_bias), y = N(h) pre_gain + pre_bias; N: "rms" or "layer".
    x and f [rows, width], or [batch, rows, width] with vectors of their own each; gate [rows, width] or, the same for all rows, [width]; gains and biases [width].
    Without f, y = N(x_scale x) pre_gain + pre_bias, and h is None unless memory for it is given.  post=False: f is not normed; pre=False: y is None."""
    return (_calls or _load_calls()).block_norm(x, f, gate, post_gain, post_bias, pre_gain, pre_bias, _one_of("norm", norm, NORMS), post, pre, _one_of("gate_act", gate_act, GATES), x_scale,
                                                f_scale, eps, need_h, h, y)


def netmax_block_norm_grad(dy, dh, x, f=None, gate=None, post_gain=None, post_bias=None, pre_gain=None, pre_bias=None, *, norm: str = "rms", post: bool = True,
                           pre: bool = True, gate_act: str = "none", x_scale: float = 1.0, f_scale: float = 1.0, eps: float = 1e-6, need_input: bool = True,
                           need_params: bool = True, dx=None, df=None, dgate=None, dpost_gain=None, dpost_bias=None, dpre_gain=None, dpre_bias=None) -> BlockNormGrads:
    """The gradients of `netmax_block_norm`, called with the same operands and options, from dy and dh (None: nothing reaches h but through y).  need_input: dx, df and the
    gradient of a gate of rows; need_params: those of gains, biases and a gate that is the same for all rows, summed over the rows."""
    return BlockNormGrads._make((_calls or _load_calls()).block_norm_grad(dy, dh, x, f, gate, post_gain, post_bias, pre_gain, pre_bias, _one_of("norm", norm, NORMS), post, pre,
                                                                          _one_of("gate_act", gate_act, GATES), x_scale, f_scale, eps, need_input, need_params, dx, df, dgate, dpost_gain,
                                                                          dpost_bias, dpre_gain, dpre_bias))


# ---- clipping ------------------------------------------------------------------------------------------------------------

def _laid_out(tensors) -> bytes:
    """Address, type, dimensions, sizes and strides of each tensor, for the extension module to compare with."""
    return array("q", [n for t in tensors for n in (t.data_ptr(), _DTYPES[t.dtype], t.dim(), *t.shape, *t.stride())]).tobytes()


class Gradients:
    """Where a model's gradients lie, for `netmax_grad_norm` and `netmax_clip_grads`: a program whose gradients stay in the same memory lays the list out once (a sequence of tensors is laid out
    in every call, 3 us for each: 96 small ones 300 us a call, laid out before 16).

    tensors: float32 or bfloat16, of any shapes, rows at one distance, on one GPU; batch: their first dimension counts models (workers), which have a norm each.  out: where the scaled
    gradients go, of the same shapes and types; None: in place.  The tensors are kept alive; one that has other memory, sizes, strides or
    another type than when the list was laid out is refused."""

    def __init__(self, tensors: Sequence[torch.Tensor], *, out: Optional[Sequence[torch.Tensor]] = None, batch: bool = False):
        self.tensors = tuple(tensors)
        self.out = self.tensors if out is None else tuple(out)
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
        self._laid = _laid_out(self.tensors + self.out)
        self._entries_at = C.addressof(self.entries)

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

    def _run(self, max_norm: Optional[float]):
        return (_calls or _load_calls()).clip(self.tensors, self.out, self._laid, self._entries_at, self.models, self.batch, max_norm)


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
