"""Argument checks and workspaces of the operators around a language model's layers through the C entry points: refused calls launch nothing, so no GPU is needed.
Addresses are numbers that are never followed."""
import ctypes as C

import pytest

import paper_2009_05766_amd as nm

A = 1 << 36
SPANS = ("x", "f", "gate", "post_gain", "post_bias", "pre_gain", "pre_bias", "h", "y")
GRADS = ("dy", "dh", "dx", "df", "dgate", "dpost_gain", "dpost_bias", "dpre_gain", "dpre_bias")


def at(k, elements=0, size=4):
    """An address of its own for every k, aligned, with 64 GiB of room."""
    return (k + 1) * A + elements * size


def refused(rc, text):
    assert rc == nm.NETMAX_EINVAL
    assert text in nm.load().netmax_last_error(None).decode(), nm.load().netmax_last_error(None)


def embed_shape(**kw):
    v = dict(batch=1, tokens=8, vocab=10, width=16, dtype=nm.NETMAX_F32, accumulate=0, scale=1.0, s_ids=8, ldt=16, st=160, ldy=16, sy=128)
    v.update(kw)
    return nm.netmax_embed_shape(**v)


@pytest.mark.parametrize("kw,text", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(tokens=-1), "tokens"), (dict(tokens=1 << 31), "tokens"), (dict(vocab=0), "vocab"), (dict(vocab=1 << 22), "vocab"),
    (dict(width=0), "width"), (dict(width=1 << 22), "width"), (dict(dtype=2), "dtype"), (dict(batch=65535, vocab=1 << 21, width=1 << 21), "too large"), (dict(tokens=1 << 30, width=1 << 20), "too large"),
    (dict(ldt=15), "table:"), (dict(ldt=-16), "table:"), (dict(ldy=15), "y:"), (dict(batch=2, sy=0), "y:"), (dict(batch=2, sy=100), "y:"), (dict(batch=2, s_ids=-1), "ids:"), (dict(batch=2, st=-1), "table:")])
def test_embed_refuses(kw, text):
    lib, s = nm.load(), embed_shape(**kw)
    refused(lib.netmax_embed(C.byref(s), at(0), at(1), at(2), None), text)
    if text.endswith("large") or kw.get("dtype"):
        assert lib.netmax_embed_grad_workspace(C.byref(s)) == -1


def test_embed_refuses_pointers():
    lib, s = nm.load(), embed_shape()
    for k, name in ((1, "ids is NULL"), (2, "table is NULL"), (3, "y is NULL")):
        args = [C.byref(s), at(0), at(1), at(2), None]
        args[k] = None
        refused(lib.netmax_embed(*args), name)
    refused(lib.netmax_embed(None, at(0), at(1), at(2), None), "shape is NULL")
    refused(lib.netmax_embed(C.byref(s), at(0) + 2, at(1), at(2), None), "ids: misaligned")
    refused(lib.netmax_embed(C.byref(s), at(0), at(1) + 2, at(2), None), "table: misaligned")
    refused(lib.netmax_embed(C.byref(s), at(0), at(1), at(1, 150), None), "y and table share")
    refused(lib.netmax_embed(C.byref(s), at(0), at(1), at(0, 7), None), "y and ids share")
    refused(lib.netmax_embed_grad(C.byref(s), at(0), at(1), None, None, 0, None), "dtable is NULL")
    refused(lib.netmax_embed_grad(C.byref(s), at(0), None, at(2), None, 0, None), "dy is NULL")
    refused(lib.netmax_embed_grad(C.byref(s), at(0), at(1), at(1, 127), None, 0, None), "dtable and dy share")
    refused(lib.netmax_embed_grad(C.byref(s), at(0), at(1), at(0, 7), None, 0, None), "dtable and ids share")
    refused(lib.netmax_embed_grad(C.byref(embed_shape(batch=2, st=100)), at(0), at(1), at(2), None, 0, None), "dtable:")
    many = embed_shape(tokens=5000)
    need = lib.netmax_embed_grad_workspace(C.byref(many))
    assert need > 5000 * 8 and lib.netmax_embed_grad_workspace(C.byref(s)) == 0
    refused(lib.netmax_embed_grad(C.byref(many), at(0), at(1), at(2), None, 0, None), "workspace")
    refused(lib.netmax_embed_grad(C.byref(many), at(0), at(1), at(2), at(3), need - 1, None), "workspace")
    refused(lib.netmax_embed_grad(C.byref(many), at(0), at(1), at(2), at(3) + 128, need, None), "workspace")
    refused(lib.netmax_embed_grad(C.byref(many), at(0), at(1), at(2), at(1), need, None), "the workspace and dy share")
    assert lib.netmax_embed(C.byref(embed_shape(tokens=0)), None, None, None, None) == nm.NETMAX_OK
    assert lib.netmax_embed_grad(C.byref(embed_shape(batch=0)), None, None, None, None, 0, None) == nm.NETMAX_OK


def norm_shape(**kw):
    v = dict(batch=1, rows=8, width=16, dtype=nm.NETMAX_F32, norm=nm.NETMAX_NORM_RMS, gate_act=nm.NETMAX_GATE_NONE, gate_rows=0, post=1, pre=1, x_scale=1.0, f_scale=1.0, eps=1e-6)
    v.update(kw)
    return nm.netmax_block_norm_shape(**v)


def spans(names, first, there, **kw):
    """Each of `there` in memory of its own, 16 wide; kw: an address, or (address, ld, s)."""
    out = []
    for k, n in enumerate(names):
        v = kw.get(n, at(first + k) if n in there else 0)
        out += list(v) if isinstance(v, tuple) else [v, 16, 128]
    return (C.c_int64 * 27)(*out)


def data(there=SPANS, **kw):
    return spans(SPANS, 0, there, **kw)


def grads(there=GRADS, **kw):
    return spans(GRADS, 10, there, **kw)


@pytest.mark.parametrize("kw,text", [
    (dict(batch=-1), "batch"), (dict(batch=65536), "batch"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(width=0), "width"), (dict(width=1 << 22), "width"), (dict(dtype=9), "dtype"),
    (dict(norm=2), "norm"), (dict(norm=-1), "norm"), (dict(gate_act=3), "gate_act"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(rows=1 << 30, width=1 << 20), "too large"),
    (dict(post=0), "post_gain"), (dict(pre=0), "pre_gain"), (dict(width=17), "x:")])
def test_norm_refuses(kw, text):
    lib, s = nm.load(), norm_shape(**kw)
    refused(lib.netmax_block_norm(C.byref(s), data(), None), text)
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), at(30), 1 << 30, None), text if text != "x:" else "dy:")


@pytest.mark.parametrize("d,text", [
    (data(x=0), "x is NULL"), (data(x=at(0) + 2), "x: misaligned"), (data(f=0), "without f"), (data(h=0, y=0), "h and y are NULL"), (data(h=(at(7), 15, 0)), "h:"), (data(y=(at(8), -16, 0)), "y:"),
    (data(h=at(8)), "h and y share"), (data(h=at(0, 16)), "h and x share"), (data(y=at(1, 8)), "y and f share"), (data(y=at(2, 15)), "y and gate share"), (data(h=at(3)), "h and post_gain share"),
    (data(h=at(4)), "post_bias share"), (data(y=at(5)), "y and pre_gain share"), (data(y=at(6)), "pre_bias share"), (data(h=(at(0), 20, 0)), "h and x share"), (data(h=at(2)), "h and gate share")])
def test_norm_refuses_operands(d, text):
    refused(nm.load().netmax_block_norm(C.byref(norm_shape()), d, None), text)


@pytest.mark.parametrize("g,d,text", [
    (grads(dy=0), data(), "dy is NULL"), (grads(dx=at(11, 5)), data(), "dx and dh share"), (grads(df=at(12)), data(), "dx and df share"), (grads(dgate=at(12, 3)), data(), "dx and dgate share"),
    (grads(dpost_gain=at(10)), data(), "dpost_gain and dy share"), (grads(dpre_gain=at(18)), data(), "dpre_gain and dpre_bias share"), (grads(dpre_gain=at(5)), data(), "dpre_gain and pre_gain share"),
    (grads(), data(f=0, gate=0, post_gain=0, post_bias=0), "without f"), (grads(), data(gate=0), "dgate without a gate"), (grads(dx=(at(12), 8, 0)), data(), "dx:"), (grads(), None, "data is NULL"),
    (None, data(), "grads is NULL")])
def test_norm_grad_refuses_operands(g, d, text):
    refused(nm.load().netmax_block_norm_grad(C.byref(norm_shape()), d, g, at(30), 1 << 30, None), text)


def test_norm_workspaces_and_nothing():
    lib, s = nm.load(), norm_shape()
    need = lib.netmax_block_norm_grad_workspace(C.byref(s), data(), grads())
    assert need >= 5 * 16 * 4 and lib.netmax_block_norm_grad_workspace(C.byref(s), data(("x",)), grads(("dy", "dx"))) == 0
    assert lib.netmax_block_norm_grad_workspace(C.byref(norm_shape(batch=0)), data(), grads()) == 0 and lib.netmax_block_norm_grad_workspace(C.byref(norm_shape(rows=0)), data(), grads()) == 0
    assert lib.netmax_embed_grad_workspace(C.byref(embed_shape(batch=0, tokens=9999))) == 0 and lib.netmax_embed_grad_workspace(C.byref(embed_shape(tokens=0))) == 0
    assert lib.netmax_block_norm_grad_workspace(C.byref(norm_shape(width=0)), data(), grads()) == -1 and lib.netmax_block_norm_grad_workspace(C.byref(s), data(), None) == -1 and lib.netmax_block_norm_grad_workspace(C.byref(s), None, grads()) == -1
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), None, 0, None), "workspace")
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), at(30), need - 1, None), "workspace")
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), at(30) + 4, need, None), "workspace")
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), at(1), need, None), "the workspace and f share")
    refused(lib.netmax_block_norm_grad(C.byref(s), data(), grads(), at(18), need, None), "the workspace and dpre_bias share")
    refused(lib.netmax_block_norm(C.byref(norm_shape(batch=2)), data(h=(at(7), 16, 0)), None), "h:")
    refused(lib.netmax_block_norm_grad(C.byref(norm_shape(batch=2)), data(), grads(dpre_gain=(at(17), 0, 0)), at(30), 1 << 20, None), "dpre_gain:")
    for kw in (dict(batch=0), dict(rows=0)):
        assert lib.netmax_block_norm(C.byref(norm_shape(**kw)), data(()), None) == nm.NETMAX_OK
    assert lib.netmax_block_norm_grad(C.byref(norm_shape(batch=0)), data(()), grads(()), None, 0, None) == nm.NETMAX_OK


def gradient_list(*entries):
    """Entries as dicts; what is not named is a matrix of 4 rows of 8 in memory of its own."""
    out = (nm.netmax_gradient * max(len(entries), 1))()
    for k, e in enumerate(entries):
        v = dict(g=at(2 * k), out=at(2 * k + 1), rows=4, cols=8, ldg=8, sg=32, ldo=8, so=32, dtype=nm.NETMAX_F32)
        v.update(e)
        for name, value in v.items():
            setattr(out[k], name, value)
    return len(entries), out


WORK = dict(norm=at(100), work=at(101), size=1 << 30)


def clip(entries, batch=1, max_norm=1.0, **kw):
    v = dict(WORK, **kw)
    n, g = gradient_list(*entries)
    return nm.load().netmax_clip_grads(batch, n, g, max_norm, v["norm"], v["work"], v["size"], None)


@pytest.mark.parametrize("entries,kw,text", [
    ([{}], dict(max_norm=0.0), "max_norm"), ([{}], dict(max_norm=float("nan")), "max_norm"), ([{}], dict(batch=-1), "batch"), ([{}], dict(batch=65536), "batch"), ([dict(dtype=4)], {}, "dtype"),
    ([dict(rows=-1)], {}, "too large"), ([dict(cols=-1)], {}, "too large"), ([dict(rows=1 << 41)], {}, "too large"), ([dict(rows=1 << 40, cols=1, ldg=1, ldo=1)], {}, "too large"),
    ([dict(g=None)], {}, "g is NULL"), ([dict(out=None)], {}, "out is NULL"), ([dict(ldg=7)], {}, "g:"), ([dict(ldo=7)], {}, "out:"), ([dict(g=at(0) + 2)], {}, "g: misaligned"), ([{}], dict(batch=2, norm=at(100) + 1), "norm:"),
    ([dict(so=0)], dict(batch=2), "out:"), ([dict(so=16)], dict(batch=2), "out:"), ([{}], dict(work=None), "workspace"), ([{}], dict(size=8), "workspace"), ([{}], dict(work=at(101) + 8), "workspace"),
    ([dict(out=at(0, 8))], {}, "g 0 and out 0 share"), ([{}, dict(out=at(1))], {}, "share"), ([{}, dict(out=at(0))], {}, "share"), ([dict(out=at(0)), dict(g=at(0), out=at(7))], {}, "share"),
    ([dict(out=at(0), ldo=9)], {}, "share"), ([{}], dict(norm=at(0, 3)), "norm and g share"), ([{}], dict(norm=at(1)), "norm and out share"), ([{}], dict(work=at(1)), "the workspace and out share"),
    ([dict(sg=100, so=100, out=at(0)), dict(g=at(0, 31), out=at(0, 31), sg=100, so=100)], dict(batch=3), "share")])
def test_clip_refuses(entries, kw, text):
    refused(clip(entries, **kw), text)


def test_clip_workspaces_and_norms():
    lib = nm.load()
    n, g = gradient_list({}, {})
    need = lib.netmax_grad_norm_workspace(3, n, g)
    assert need >= 8 * 3 and lib.netmax_grad_norm_workspace(-1, n, g) == -1 and lib.netmax_grad_norm_workspace(1, 65536, g) == -1 and lib.netmax_grad_norm_workspace(1, 2, None) == -1
    assert lib.netmax_grad_norm_workspace(0, n, g) == 0
    refused(lib.netmax_grad_norm(1, n, g, None, at(101), need, None), "norm is NULL")
    refused(lib.netmax_grad_norm(1, n, g, at(0), at(101), need, None), "norm and g share")
    refused(lib.netmax_grad_norm(1, n, g, at(100), at(2), need, None), "the workspace and g share")
    refused(lib.netmax_grad_norm(1, n, g, at(100), at(101), 0, None), "workspace")
    assert lib.netmax_grad_norm(0, n, g, None, None, 0, None) == nm.NETMAX_OK
