"""The kernels that the operators around a language model's layers launch, on the host code of the built library: every kernel is reached by a test that compares its results on a GPU, and
operands that lie apart, or where they may be shared, are launched."""
import os
import shutil
import subprocess

import pytest

import paper_2009_05766_amd as nm
import test_gpu_lm_step_ops as ops
import test_gpu_lm_step_routes as routes
from lm_calls import BF16, F32, ROOT, at
from paper_2009_05766_amd.build import LIB, build
from test_lm_routes import cases

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs g++ and the HIP headers")

OURS = {"embed_kernel", "embed_grad_narrow_kernel", "embed_grad_few_kernel", "embed_count_kernel", "embed_sort_kernel", "embed_sum_kernel", "embed_join_kernel", "long_norm_kernel", "norm_kernel",
        "long_norm_grad_kernel", "norm_grad_kernel", "norm_columns_kernel", "join_sums_kernel", "squares_kernel", "total_kernel", "scale_kernel", "clip_small_kernel"}


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("step") / "drive")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "lm_step_calls_driver.cpp"), "-rdynamic", "-ldl", "-o", exe], check=True)
    lib = LIB if os.path.exists(LIB) else build()

    def run(*calls):
        lines = "\n".join(" ".join([op] + [f"{k}={n!r}" for k, n in v.items()]) for op, v in calls)
        r = subprocess.run([exe, lib], input=lines, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line in r.stdout.splitlines():
            status, text, launches = line.split("|")
            out.append((int(status), text, [(k.rsplit("@", 1)[0], int(k.rsplit("@", 1)[1])) for k in launches.split()]))
        return out
    return run


def kind(dtype):
    return BF16 if dtype is ops.BF16 else F32


def embed(n, vocab, width, batch=0, dtype=F32, **kw):
    v = dict(batch=batch or 1, tokens=n, vocab=vocab, width=width, dtype=dtype, s_ids=n, ldt=width, st=vocab * width, ldy=width, sy=n * width, ids=at(0), table=at(1), y=at(2), work=at(3))
    v.update(kw)
    return [("embed", v), ("embed_grad", v), ("embed_grad", dict(v, accumulate=1))]


SPANS = ("x", "f", "gate", "post_gain", "post_bias", "pre_gain", "pre_bias", "h", "y")


def norm(rows, width, dtype=F32, norm="rms", block=True, gate=None, act="none", gains=True, bias=False, post=True, pre=True, dh=True, batch=0, **kw):
    """What check_norm calls."""
    there = {"x": True, "f": block, "gate": block and gate, "post_gain": block and post and gains, "post_bias": block and post and bias, "pre_gain": pre and gains, "pre_bias": pre and bias}
    v = dict(batch=batch or 1, rows=rows, width=width, dtype=dtype, norm=int(norm == "layer"), gate_act=["none", "sigmoid", "tanh"].index(act), gate_rows=int(gate == "rows"), post=int(post), pre=int(pre),
             x_scale=1.0, f_scale=1.0, eps=1e-6, work=at(40))
    names = [n for n in SPANS[:7] if there[n]]
    for k, n in enumerate(names + ["h"] * block + ["y"] * pre + ["dy"] * pre + ["dh"] * (dh or not pre) + ["d" + n for n in names]):
        rows_of = n in ("x", "f", "h", "y", "dy", "dh", "dx", "df") or (n in ("gate", "dgate") and gate == "rows")
        v.update({n: at(k), n + ".ld": width, n + ".s": rows * width if rows_of else width})
    v.update({k: n for k, n in kw.items() if k in v or "." in k or k in SPANS})
    return [("norm", v), ("norm_grad", v)]


def clip(tensors, batch=1, out=True):
    """tensors: (rows, columns, distance of rows, type)."""
    v = dict(batch=batch, n=len(tensors), norm=at(1000), work=at(1001))
    for k, (rows, cols, ld, dtype) in enumerate(tensors):
        v.update({f"g{k}": at(2 * k), f"out{k}": at(2 * k + out), f"rows{k}": rows, f"cols{k}": cols, f"ldg{k}": ld, f"sg{k}": rows * ld, f"ldo{k}": ld, f"so{k}": rows * ld, f"dtype{k}": dtype})
    return [("clip", v), ("grad_norm", v)]


def calls_of_tests():
    """The calls of the tests that compare with 64 bits on a GPU."""
    c = []
    for k in cases(ops.test_embed_sizes):
        c += embed(k["n"], k["vocab"], k["width"], dtype=kind(k["dtype"]))
    for k in cases(ops.test_embed_batches):
        c += embed(k["n"], k["vocab"], k["width"], k["batch"], kind(k["dtype"]))
    for k in cases(routes.test_embeddings):
        c += embed(k["n"], 600, k["width"], dtype=kind(k["dtype"]))
    for k in cases(ops.test_norm_sizes):
        c += norm(k["rows"], k["width"], kind(k["dtype"]), k["norm"], gate="channel", act="sigmoid", bias=k["norm"] == "layer")
    for k in cases(routes.test_norms):
        for form in routes.FORMS:
            c += norm(k["rows"], k["width"], kind(k["dtype"]), k["norm"], **form)
    for k in cases(ops.test_norm_forms):
        for form in (dict(block=False), dict(gate="rows", act="sigmoid"), dict(gate="rows", act="tanh", bias=True), dict(gate="channel"), dict(bias=True)):
            c += norm(k["rows"], k["width"], kind(k["dtype"]), k["norm"], **form)
    for dtype in (F32, BF16):
        for tensors in ops.CLIP_SIZES:
            c += clip([(1, n, n, dtype) for n in (int(__import__("math").prod(s)) for s in tensors)])
        c += clip([(9, 30, 32, dtype)]) + clip([(300, 101, 103, dtype), (1, 70000, 70000, dtype)]) + clip([(1, 1 << 24, 1 << 24, dtype)] + [(1, 3000, 3000, dtype)] * 200)
    return c


def test_every_kernel_is_reached(call):
    (_, _, all_kernels), *answers = call(("kernels", {}), *calls_of_tests())
    mine = {k for k, _ in all_kernels if k.split("<")[0] in OURS}
    assert len(mine) > 200 and {k.split("<")[0] for k in mine} == OURS
    for (status, error, launches), c in zip(answers, calls_of_tests()):
        assert status == 0 and (launches or c[1].get("tokens") == 0), (c, error)
    assert sorted(mine - {k for _, _, launches in answers for k, _ in launches}) == []


def slices(batch, apart, sizes, out):
    """Slices of models' rows of gradients, in place or into rows of their own."""
    v, first = dict(batch=batch, n=len(sizes), norm=at(1000), work=at(1001)), 0
    for k, n in enumerate(sizes):
        v.update({f"g{k}": at(0, first), f"out{k}": at(0 if out is None else out, first), f"rows{k}": 1, f"cols{k}": n, f"ldg{k}": n, f"ldo{k}": n, f"sg{k}": apart, f"so{k}": apart, f"dtype{k}": F32})
        first += n
    return v


def test_operands_that_may_be_shared_are_launched(call):
    lds = {n + ".ld": 200 for n in ("x", "f", "h", "y", "dy", "dh", "dx", "df")}
    calls = [norm(50, 100, h=at(0), y=at(1))[0], norm(50, 100, gate="rows", h=at(2), y=at(0))[0], norm(50, 96, x=at(0), f=at(0, 96), **lds)[0],
             ("clip", slices(7, 1000, [10, 500, 490], None)), ("clip", slices(7, 1001, [10, 500, 490], 3)), ("clip", slices(1, 0, [3, 5, 1 << 20], None))]
    g = norm(5, 9000, gate="rows")[1]
    v = g[1]
    calls += [("norm_grad", dict(v, dx=v["dy"], df=v["dh"], dgate=v["x"])), ("norm_grad", dict(v, dx=v["dh"], df=v["f"], dgate=v["gate"]))]
    for (status, error, launches), c in zip(call(*calls), calls):
        assert status == nm.NETMAX_OK and launches, (c, error)
    # wide rows written over what is read: the rows' kernel runs before the columns' for the means alone, and behind it for the results
    (_, _, apart), (_, _, over) = call(g, calls[-1])
    names = lambda launches: [k.split("<")[0] for k, _ in launches]  # noqa: E731
    assert names(apart) == ["norm_grad_kernel", "norm_columns_kernel", "join_sums_kernel"] and names(over) == names(apart) + ["norm_grad_kernel"]


def test_shared_slices_are_refused(call):
    bad = [slices(7, 1000, [10, 500, 491], None), slices(7, 1000, [500, 500], 3), slices(3, 100, [60, 30], None)]
    bad[1]["out1"] = at(3, 499)
    bad[2]["g1"] = bad[2]["out1"] = at(0, 59)
    for (status, error, launches), v in zip(call(*(("clip", v) for v in bad)), bad):
        assert status == nm.NETMAX_EINVAL and ("share" in error or "same place" in error) and launches == [], v


def test_more_tensors_than_a_launch_holds(call):
    many, padded = clip([(1, 3000 + k, 3000 + k, F32) for k in range(400)]), clip([(7, 30, 40, BF16)] * 60)
    (_, _, a), (_, _, b), (_, _, c), _ = call(*many, *padded)
    names = lambda launches: [k for k, _ in launches]  # noqa: E731
    assert names(a) == ["squares_kernel<true>"] * 4 + ["scale_kernel<true>"] * 4 and names(b) == ["squares_kernel<true>"] * 4 + ["total_kernel"] and names(c) == ["squares_kernel<false>"] * 2 + ["scale_kernel<false>"] * 2
