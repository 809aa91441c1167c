"""Argument checks and workspaces of the operators for language models through the C entry points: refused calls launch nothing, so no GPU is needed.
Addresses are numbers that are never followed."""
import ctypes as C

import pytest

import paper_2009_05766_amd as nm
from paper_2009_05766_amd.binding import netmax_linear_shape, netmax_orth_shape

A, B, D = 1 << 20, 1 << 21, 1 << 22          # aligned addresses


def linear_shape(**kw):
    v = dict(batch=1, rows=8, d_in=16, d_out=24, dtype=nm.NETMAX_F32, act=nm.NETMAX_ACT_NONE, ldx=16, ldw=24, ldr=24, ldy=24, ldz=24, lddx=16, lddw=24)
    v.update(kw)
    return netmax_linear_shape(**v)


def refused(rc, text):
    assert rc == nm.NETMAX_EINVAL
    assert text in nm.load().netmax_last_error(None).decode(), nm.load().netmax_last_error(None)


@pytest.mark.parametrize("kw,text", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(rows=-1), "rows"), (dict(d_in=0), "d_in"), (dict(d_out=0), "d_out"), (dict(d_in=1 << 22), "d_in"),
    (dict(rows=1 << 40), "too large"), (dict(rows=65535 * 64 + 1), "too large"), (dict(dtype=7), "dtype"), (dict(act=9), "activation"), (dict(act=-1), "activation"),
    (dict(batch=2, sx=128, sr=192, sz=192), "y:"), (dict(batch=2, sy=192), "z:"), (dict(ldx=15), "x:"), (dict(ldw=23), "w:"), (dict(ldy=23), "y:"), (dict(ldr=1), "residual:"), (dict(ldz=0), "z:"), (dict(batch=2, sx=-8), "x:"), (dict(ldx=-16), "x:"),
])
def test_linear_refuses(kw, text):
    lib, s = nm.load(), linear_shape(**kw)
    refused(lib.netmax_linear(C.byref(s), A, A, A, A, A, A, None, 0, None), text)


@pytest.mark.parametrize("kw", [dict(batch=1000, rows=1 << 21), dict(batch=65535, rows=8, d_in=1 << 15), dict(batch=65535, rows=1, d_out=1 << 15)])
def test_more_blocks_than_a_launch_can_have(kw):
    lib, s = nm.load(), linear_shape(**kw)
    refused(lib.netmax_linear(C.byref(s), A, A, A, A, A, A, None, 0, None), "too large")


def test_linear_refuses_pointers():
    lib, s = nm.load(), linear_shape()
    for k, name in ((1, "x is NULL"), (2, "w is NULL"), (5, "y is NULL")):
        args = [C.byref(s), A, A, None, None, A, None, None, 0, None]
        args[k] = None
        refused(lib.netmax_linear(*args), name)
    refused(lib.netmax_linear(C.byref(s), A + 2, A, None, None, A, None, None, 0, None), "x: misaligned")
    refused(lib.netmax_linear(None, A, A, None, None, A, None, None, 0, None), "shape is NULL")
    half = linear_shape(dtype=nm.NETMAX_BF16, d_in=17, ldx=17)                    # rows at odd places: a new layout needs space
    need = lib.netmax_linear_workspace(C.byref(half), A, A)
    assert need > 0
    refused(lib.netmax_linear(C.byref(half), A, A, None, None, A, None, None, 0, None), "workspace")
    refused(lib.netmax_linear(C.byref(half), A, A, None, None, A, None, D, need - 1, None), "workspace")
    refused(lib.netmax_linear(C.byref(half), A, A, None, None, A, None, D + 16, need, None), "workspace")
    g = linear_shape(act=nm.NETMAX_ACT_GELU)
    refused(lib.netmax_linear_grad(C.byref(g), A, A, A, None, A, A, A, D, 1 << 30, None), "z is NULL")
    refused(lib.netmax_linear_grad(C.byref(g), None, A, A, A, A, A, A, D, 1 << 30, None), "dy is NULL")
    refused(lib.netmax_linear_grad(C.byref(g), A, None, A, A, A, A, A, D, 1 << 30, None), "x is NULL")
    refused(lib.netmax_linear_grad(C.byref(g), A, A, None, A, A, A, A, D, 1 << 30, None), "w is NULL")
    refused(lib.netmax_linear_grad(C.byref(g), A, A, A, A, A, A, A, D, 8, None), "workspace")


def test_workspaces():
    lib = nm.load()
    assert lib.netmax_linear_workspace(C.byref(linear_shape()), A, A) == 0
    assert lib.netmax_linear_workspace(C.byref(linear_shape(d_in=0)), A, A) == -1
    aligned = linear_shape(dtype=nm.NETMAX_BF16)
    assert lib.netmax_linear_workspace(C.byref(aligned), A, B) == 0
    assert lib.netmax_linear_workspace(C.byref(aligned), A + 2, B) >= 8 * 16 * 2        # x alone
    assert lib.netmax_linear_workspace(C.byref(aligned), A + 2, B + 2) >= 8 * 16 * 2 + 16 * 24 * 2
    assert lib.netmax_linear_grad_workspace(C.byref(linear_shape(act=nm.NETMAX_ACT_SILU)), A, A, A) >= 8 * 24 * 4
    o = netmax_orth_shape(batch=2, rows=30, cols=20, dtype=nm.NETMAX_F32, steps=5, nesterov=1, mu=0.9, a=3.0, b=-4.0, c=2.0, eps=1e-7, scale=1.0, ldg=20, sg=600, ldm=20,
                          sm=600, ldo=20, so=600)
    assert lib.netmax_orthogonalize_workspace(C.byref(o)) > 2 * 30 * 24 * 2 * 4
    assert lib.netmax_preference_workspace(100, 4) >= 1600 + 32 and lib.netmax_preference_workspace(-1, 4) == -1 and lib.netmax_preference_workspace(4, 0) == -1
    refused(lib.netmax_orthogonalize(C.byref(o), A, B, B, A, D, 64, None), "workspace")
    refused(lib.netmax_orthogonalize(C.byref(o), A, None, B, A, D, 1 << 30, None), "m is NULL")
    refused(lib.netmax_orthogonalize(C.byref(o), A, B, None, A, D, 1 << 30, None), "m_out is NULL")
    refused(lib.netmax_orthogonalize(C.byref(o), None, B, B, A, D, 1 << 30, None), "g is NULL")
    for kw, text in ((dict(steps=0), "steps"), (dict(steps=65), "steps"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(rows=0), "rows"), (dict(cols=1 << 22), "cols"),
                     (dict(dtype=3), "dtype"), (dict(ldg=19), "g:"), (dict(so=-1), "out:")):
        v = {n: getattr(o, n) for n, _ in o._fields_}
        v.update(kw)
        refused(lib.netmax_orthogonalize(C.byref(netmax_orth_shape(**v)), A, B, B, A, D, 1 << 30, None), text)


def test_losses_refuse():
    lib = nm.load()

    def policy(tokens=4, vocab=10, dtype=0, logits=A, ld=10, labels=A, old=A, ref=None, adv=A, weight=None, low=0.2, high=0.2, kl=0.0, loss=A, logp=None, grad=None, ldg=0):
        return lib.netmax_policy_loss(tokens, vocab, dtype, logits, ld, labels, old, ref, adv, weight, low, high, kl, loss, logp, grad, ldg, None)

    for kw, text in ((dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(vocab=0), "vocab"), (dict(dtype=5), "dtype"), (dict(logits=None), "logits is NULL"),
                     (dict(ld=9), "logits:"), (dict(labels=None), "labels"), (dict(old=None), "NULL"), (dict(adv=None), "NULL"), (dict(loss=None), "NULL"), (dict(low=-0.1), "clip_low"),
                     (dict(low=1.1), "clip_low"), (dict(high=-0.1), "clip_high"), (dict(high=float("nan")), "clip_high"), (dict(kl=0.1), "ref_logp"), (dict(grad=B, ldg=9), "grad:"),
                     (dict(grad=A, ldg=11), "distance")):
        refused(policy(**kw), text)
    assert policy(tokens=0, logits=None, labels=None, old=None, adv=None, loss=None) == nm.NETMAX_OK

    def preference(tokens=4, pairs=1, offsets=A, ref=A, smoothing=0.0, loss=A, ratio=A, work=D, size=1 << 20):
        return lib.netmax_preference_loss(tokens, 10, 0, A, 10, A, pairs, offsets, ref, None, 0.1, smoothing, 1.0, loss, ratio, None, 0, work, size, None)

    for kw, text in ((dict(pairs=0), "pairs"), (dict(smoothing=1.5), "smoothing"), (dict(smoothing=float("nan")), "smoothing"), (dict(offsets=None), "NULL"), (dict(ref=None), "NULL"),
                     (dict(loss=None), "NULL"), (dict(ratio=None), "NULL"), (dict(work=None), "workspace"), (dict(size=16), "workspace")):
        refused(preference(**kw), text)
