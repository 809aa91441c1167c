"""Lists of gradients whose tensors have changed.  Sums over no rows.  Rows of an embedding's gradient that are added to.  Gradients of a block's norms of which only some are wanted, or that are written over what is read, in batches of rows of every kind of kernel: the same bits as all of them in memory of
their own.  (Where their kernels work is looked at without a GPU: test_lm_step_places.py.)"""
import pytest
import torch

import paper_2009_05766_amd as nm
import test_gpu_lm_step_ops as ops

pytestmark = pytest.mark.gpu

SIZES = [(3, 5, 40), (2, 33, 300), (2, 64, 700), (2, 20, 1500), (3, 7, 6000), (2, 10, 8200), (2, 64, 9000), (4, 64, 12000), (8, 20, 16384), (2, 6, 20000)]


def operands(g, batch, rows, width, dtype, block=True, gate=None):
    x, f, q, dy, dh = (ops.normal(g, batch, rows, width, dtype=dtype) for _ in range(5))
    v = [ops.normal(g, batch, width, dtype=dtype, mean=1.0) for _ in range(5)]
    if not block:
        return dy, dh, [x, None, None, None, None, v[0], v[1]]
    return dy, dh, [x, f, {"rows": q, "channel": v[4], None: None}[gate], v[0], v[1], v[2], v[3]]


@ops.BOTH
@pytest.mark.parametrize("batch,rows,width", SIZES)
def test_some_results(batch, rows, width, dtype):
    g = ops.gen(width)
    for form in (dict(block=False), dict(gate="channel"), dict(gate="rows")):
        dy, dh, t = operands(g, batch, rows, width, dtype, **form)
        options = dict(norm="layer", gate_act="sigmoid")
        want = nm.netmax_block_norm_grad(dy, dh, *t, **options)
        same = lambda got, names: all((torch.equal(a, b) if n in names else a is None) for n, a, b in zip(want._fields, got, want) if b is not None)  # noqa: E731
        of_rows = [n for n, w in want._asdict().items() if w is not None and w.dim() == 3]
        others = [n for n, w in want._asdict().items() if w is not None and w.dim() == 2]
        assert same(nm.netmax_block_norm_grad(dy, dh, *t, need_input=False, **options), others), form
        assert same(nm.netmax_block_norm_grad(dy, dh, *t, need_params=False, **options), of_rows), form
        for n in of_rows:
            got = nm.netmax_block_norm_grad(dy, dh, *t, need_input=False, **options, **{n: torch.empty_like(dy)})
            assert same(got, [n, *others]), (form, n)


@ops.BOTH
@pytest.mark.parametrize("batch,rows,width", SIZES)
def test_results_over_what_is_read(batch, rows, width, dtype):
    g = ops.gen(width + 1)
    for gate in (None, "rows"):
        dy, dh, t = operands(g, batch, rows, width, dtype, gate=gate)
        want = nm.netmax_block_norm_grad(dy, dh, *t)
        for order in (dict(dx=0, df=1), dict(dx=1, df=3), dict(dx=3), dict(df=2)):
            c = [v if v is None else v.clone() for v in t]
            rows_of = [dy.clone(), dh.clone(), *c[:3]]
            got = nm.netmax_block_norm_grad(rows_of[0], rows_of[1], *c, **{n: rows_of[k] for n, k in order.items()})
            assert all(torch.equal(a, b) for a, b in zip(got, want) if b is not None), (gate, order)


def test_rows_of_other_tokens_are_kept_by_the_widest_calls():
    """A launch of more workgroups than go along one dimension, to which its shape adds some: they clear nothing of what is added to, and what they should of what is not."""
    n, vocab, width = 513, 12, (1 << 22) - 4
    dy = torch.ones(n, width, device="cuda")
    tokens = (torch.arange(n, device="cuda") % 3 * 4).to(torch.int32)                   # 0, 4 and 8, 171 times each
    table = torch.full((vocab, width), 5.0, device="cuda")
    nm.netmax_embed_grad(dy, tokens, accumulate=True, dtable=table)
    want = torch.full((vocab,), 5.0, device="cuda")
    want[::4] += 171.0
    assert torch.equal(table, want[:, None].expand(vocab, width))
    nm.netmax_embed_grad(dy, tokens, dtable=table)
    assert torch.equal(table, (want - 5.0)[:, None].expand(vocab, width))


@ops.BOTH
@pytest.mark.parametrize("batch,width", [(300, 16384), (3000, 3), (5000, 8200), (2, 20000)])
def test_sums_over_no_rows(batch, width, dtype):
    x, v = torch.empty(batch, 0, width, device="cuda", dtype=dtype), torch.ones(batch, width, device="cuda", dtype=dtype)
    for _ in range(2):
        memory = torch.full((1 << 28,), float("nan"), device="cuda")                    # what workspaces may come from
        del memory
        got = nm.netmax_block_norm_grad(x, x, x, x, v, v, v, v, v)
        assert all(t.shape == (batch, width) and not bool(t.any()) for t in got[2:])


def test_a_list_whose_tensors_have_changed():
    """Neither read nor written by the sizes that a tensor had, whichever of the two sides it is on; what has changed back, or only its values, is fine."""
    g = ops.gen(2)
    room, out = ops.normal(g, 50, 40), torch.full((50, 40), 5.0, device="cuda")
    laid = nm.Gradients([room], out=[out])
    want = nm.netmax_clip_grads(laid, 1.0)
    for t in (room, out):
        for change in (lambda: t.resize_(20, 40), lambda: t.resize_(40, 50), lambda: t.as_strided_((50, 30), (40, 1))):
            change()
            for call in (lambda: nm.netmax_grad_norm(laid), lambda: nm.netmax_clip_grads(laid, 1.0)):
                with pytest.raises(nm.NetmaxError, match="has changed") as e:
                    call()
                assert e.value.code == nm.NETMAX_EINVAL
            t.as_strided_((50, 40), (40, 1))
    room.mul_(2.0)
    assert torch.equal(nm.netmax_clip_grads(laid, 1.0), 2 * want) and float(nm.netmax_grad_norm([out])) == pytest.approx(1.0, rel=1e-5)
