"""Values at which the operators around a language model's layers went wrong once: infinities that nothing norms, products beside the middle of two bfloat16 values, outputs made in inference
mode.  Tolerances as in test_gpu_lm_step_ops.py, where they are not bits."""
import pytest
import torch

import paper_2009_05766_amd as nm
import test_gpu_lm_step_ops as ops

pytestmark = pytest.mark.gpu

BF16, E, ULP = ops.BF16, ops.E, ops.ULP


@ops.BOTH
@pytest.mark.parametrize("gate", [None, "channel", "rows"])
@pytest.mark.parametrize("width", [3, 40, 130, 300, 700, 1500, 3000, 5000, 8192, 9000, 12000, 16384, 20000])
def test_infinities_of_a_block_without_norms(width, gate, dtype):
    """df = f_scale gate dh does not depend on f: it is finite where f is not."""
    g = ops.gen(width)
    x, f, dh, q = (ops.normal(g, 7, width, dtype=dtype) for _ in range(4))
    f[2], f[4, width // 2] = float("inf"), -float("inf")
    f[5, 0] = float("nan")
    gates = {None: None, "channel": q[0], "rows": q}[gate]
    for norm in ("rms", "layer"):
        got = nm.netmax_block_norm_grad(None, dh, x, f, gates, norm=norm, post=False, pre=False, f_scale=1.5, x_scale=0.5)
        want = 1.5 * dh.double() * (1.0 if gates is None else gates.double())
        ops.within(got.df, want, (3 * E + ULP[dtype]) * want.abs() + 1e-37, f"df {norm}")
        ops.within(got.dx, 0.5 * dh.double(), (E + ULP[dtype]) * dh.double().abs(), f"dx {norm}")
