"""The kernels that the operators for language models launch, on the host code of the built library (lm_calls.py): every kernel is reached by a test that compares
its results on a GPU, so that a rule that moves cannot leave one untested."""
import itertools
import os
import shutil

import pytest

import test_gpu_lm_ops as ops
import test_gpu_lm_routes as routes
import test_gpu_lm_values as values
from lm_calls import BF16, F32, GELU, NONE, RELU, SILU, compiled, grad, linear, orth, policy, preference

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs g++ and the HIP headers")

ACT = {"none": NONE, "relu": RELU, "gelu": GELU, "silu": SILU}
OURS = {"lay_out_kernel", "join_parts_kernel", "gemm16_kernel", "gemm16_pair_kernel", "few_rows_kernel", "gemm_f32_kernel", "gemm_f32_pair_kernel", "slope_kernel", "bias_sum_kernel",
        "momentum_kernel", "normalise_kernel", "policy_loss_kernel", "preference_rows_kernel", "preference_pairs_kernel", "preference_gradient_kernel"}


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    return compiled(tmp_path_factory.mktemp("routes"))


def cases(test):
    """The parameters of a parametrised test, as dicts."""
    parts = []
    for mark in getattr(test, "pytestmark", []):
        if mark.name == "parametrize":
            names = [n.strip() for n in mark.args[0].split(",")]
            parts.append([dict(zip(names, v if len(names) > 1 else (v,))) for v in mark.args[1]])
    return [{k: v for part in combo for k, v in part.items()} for combo in itertools.product(*parts)]


def kind(dtype):
    return BF16 if dtype is ops.BF16 else F32


def layer(rows, d_in, d_out, dtype, act, batch=0, pad=0, bias=1, residual=1, grads=True):
    """What check_linear calls."""
    lds = dict(ldx=d_in + pad, ldw=d_out + pad, ldr=d_out + pad, ldy=d_out, ldz=d_out)
    out = [linear(rows, d_in, d_out, batch or 1, kind(dtype), ACT[act], bias=bias and (20 << 36), residual=residual and (21 << 36), z=22 << 36, **lds)]
    if grads:
        out.append(grad(rows, d_in, d_out, batch or 1, kind(dtype), ACT[act], ldx=d_in + pad, ldw=d_out + pad, ldy=d_out + pad, ldz=d_out))
    return out


def calls_of_tests():
    """The calls of the tests that compare with 64 bits on a GPU."""
    c = []
    for k in cases(ops.test_linear_sizes):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "gelu")
    for k in cases(ops.test_linear_batches):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "silu", k["batch"])
    for k in cases(ops.test_linear_large_batches_of_small_layers):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "gelu", k["batch"])
    for k in cases(ops.test_linear_distances_of_rows):
        c += layer(70, 264, 200, k["dtype"], "gelu", k["batch"], k["pad"])
    for k in cases(ops.test_linear_long):
        c += layer(k["rows"], 512, 768, k["dtype"], "gelu") + layer(k["rows"], 96, 80, k["dtype"], "none")
    for k in cases(ops.test_linear_many_blocks):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "silu")
    for k in cases(ops.test_linear_large_in_float):
        c += layer(k["rows"], k["d_in"], k["d_out"], ops.F32, "gelu", k["batch"])
    for k in cases(ops.test_linear_few_rows):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "gelu") + layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "none", 3, 8)
    for k in cases(routes.test_layers):
        c += layer(k["rows"], k["d_in"], k["d_out"], k["dtype"], "gelu", k["batch"])
    for k in cases(routes.test_one_gradient_alone):
        c.append(grad(k["rows"], k["d_in"], k["d_out"], 1, kind(k["dtype"]), **{n: 0 for n in ("dx", "dw", "db") if n != k["which"]}))
    for test in (ops.test_orthogonalize_sizes, ops.test_orthogonalize_many_matrices, ops.test_orthogonalize_many_matrices_that_fill_their_blocks, routes.test_updates):
        c += [orth(k["rows"], k["cols"], k["batch"], kind(k["dtype"])) for k in cases(test)]
    for k in cases(ops.test_policy_loss_sizes):
        c.append(policy(k["tokens"], k["vocab"], kind(k["dtype"])))
    for k in cases(ops.test_preference_loss_sizes):
        c.append(preference(sum(k["lengths"]) + 5, k["vocab"], len(k["lengths"]) // 2, kind(k["dtype"])))
    for k in cases(routes.test_lengths_of_rows):
        c += [policy(k["tokens"], k["vocab"], kind(k["dtype"])), preference(k["tokens"] + 7, k["vocab"], 1, kind(k["dtype"]))]
    for k in cases(values.test_log_probability_of_a_peak):
        c += [policy(6, k["vocab"], kind(k["dtype"]), grad=0), preference(6, k["vocab"], 1, kind(k["dtype"]), grad=0)]
    return c


def test_every_kernel_is_reached(call):
    (_, _, all_kernels), *answers = call(("kernels", {}), *calls_of_tests())
    mine = {k for k, _ in all_kernels if k.split("<")[0] in OURS}
    assert len(mine) > 100 and {k.split("<")[0] for k in mine} == OURS
    for k, (status, error, launches) in enumerate(answers):
        assert status == 0 and launches, (calls_of_tests()[k], error)
    assert sorted(mine - {k for _, _, launches in answers for k, _ in launches}) == []
