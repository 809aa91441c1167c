"""Sizes of the operators for language models that reach kernels which no other test of results does (test_lm_routes.py looks whether all are reached)."""
import pytest

import paper_2009_05766_amd as nm
import test_gpu_lm_ops as ops

pytestmark = pytest.mark.gpu

F32, BF16 = ops.F32, ops.BF16


@pytest.mark.parametrize("rows,d_in,d_out,batch,dtype", [
    (42, 533, 2501, 0, BF16), (1, 408, 1560, 12, BF16), (1009, 9, 2057, 4, BF16), (2445, 336, 8, 9, BF16), (232, 2032, 351, 16, BF16), (2126, 653, 2057, 0, BF16), (1300, 2100, 1200, 0, BF16),
    (2100, 1200, 1300, 0, BF16), (70, 1000, 1100, 0, BF16), (520, 130, 140, 40, BF16), (384, 390, 400, 60, BF16), (4096, 72, 1168, 9, BF16), (1152, 4104, 1200, 0, BF16), (1152, 1200, 4104, 0, BF16), (4104, 1150, 1200, 0, BF16),
    (280, 1944, 1976, 0, F32), (3535, 1165, 359, 0, F32), (130, 200, 190, 30, F32), (2370, 443, 259, 12, F32)])
def test_layers(rows, d_in, d_out, batch, dtype):
    ops.check_linear(rows, d_in, d_out, dtype, "gelu", batch=batch, seed=rows)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(1, 33, 70), (100, 260, 300), (200, 1100, 120), (700, 1500, 700), (1500, 1300, 1400), (2100, 1030, 2050)])
@pytest.mark.parametrize("which", ["dx", "dw", "db"])
def test_one_gradient_alone(which, rows, d_in, d_out, dtype):
    g = ops.gen(rows)
    x, w, dy = ops.normal(g, rows, d_in, dtype=dtype), ops.normal(g, d_in, d_out, dtype=dtype, scale=d_in ** -0.5), ops.normal(g, rows, d_out, dtype=dtype)
    got = dict(zip(("dx", "dw", "db"), nm.netmax_linear_grad(dy, x, w, need_input=which == "dx", need_weight=which == "dw", need_bias=which == "db")))
    assert [n for n, t in got.items() if t is not None] == [which]
    X, W, DY = x.double(), w.double(), dy.double()
    want, size, terms = {"dx": lambda: (DY @ W.t(), DY.abs() @ W.abs().t(), d_out), "dw": lambda: (X.t() @ DY, X.abs().t() @ DY.abs(), rows), "db": lambda: (DY.sum(0), DY.abs().sum(0), rows)}[which]()
    ops.within(got[which], want, (terms + 4) * 2.0 ** -24 * size + ops.ULP[dtype] * want.abs(), which)


@pytest.mark.parametrize("batch,rows,cols,dtype", [
    (1, 538, 526, F32), (1, 530, 537, F32), (1, 512, 642, BF16), (1, 723, 531, BF16), (132, 72, 434, F32), (242, 69, 273, BF16), (44, 1821, 65, BF16), (260, 313, 67, F32), (46, 65, 293, BF16), (48, 293, 65, F32), (142, 69, 78, F32), (140, 78, 69, BF16),
    (86, 384, 400, F32), (86, 400, 384, F32), (86, 384, 400, BF16), (86, 400, 384, BF16)])
def test_updates(batch, rows, cols, dtype):
    ops.test_orthogonalize_many_matrices(batch, rows, cols, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab", [(7, 3001), (5, 4096), (6, 9001), (5, 12289), (4, 16385), (3, 20000)])
def test_lengths_of_rows(tokens, vocab, dtype):
    ops.test_policy_loss_sizes(tokens, vocab, dtype)
    ops.test_preference_loss_sizes([tokens, 2], vocab, dtype)
