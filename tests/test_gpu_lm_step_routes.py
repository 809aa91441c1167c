"""Sizes of the operators around a language model's layers that reach kernels which no other test of results does (test_lm_step_routes.py looks whether all are reached)."""
import pytest
import torch

import test_gpu_lm_step_ops as ops

pytestmark = pytest.mark.gpu

FORMS = [dict(block=False), dict(gate="channel"), dict(gate="channel", bias=True), dict(gate="rows", act="tanh"), dict(gate="rows", bias=True)]


@ops.BOTH
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("rows,width", [(60, 30), (35, 100), (70, 300), (9, 600), (11, 900), (8, 1400), (6, 1800), (7, 2500), (5, 3500), (5, 6000), (4, 7000), (3, 11000), (3, 13000)])
def test_norms(rows, width, norm, dtype):
    for k, form in enumerate(FORMS):
        ops.check_norm(rows, width, dtype, norm, seed=k + width, **form)


@ops.BOTH
@pytest.mark.parametrize("n", [700, 2500])
@pytest.mark.parametrize("width", [30, 50, 100, 120, 250, 300, 500, 800, 1500, 2500])
def test_embeddings(n, width, dtype):
    ops.check_embed(n, 600, width, dtype, seed=width)


@ops.BOTH
def test_clipping(dtype):
    g = ops.gen(1)
    for tensors in ([ops.strided(ops.normal(g, 9, 30, dtype=dtype), 2)], [ops.strided(ops.normal(g, 300, 101, dtype=dtype), 2), ops.normal(g, 70000, dtype=dtype)],
                    [ops.normal(g, 40000 + k, dtype=dtype) for k in range(130)], [ops.strided(ops.normal(g, 30 + k, 41, dtype=dtype), 1) for k in range(60)],
                    [ops.normal(g, 1 << 24, dtype=dtype), *(ops.normal(g, 3000, dtype=dtype) for _ in range(200))]):
        ops.check_clip([t.clone() if t.is_contiguous() else ops.strided(t.clone(), t.stride(0) - t.shape[1]) for t in tensors], 5.0)
        ops.check_clip(tensors, 5.0, out=[torch.empty_like(t) for t in tensors])
