"""Memory that calls of the operators for language models share: what would race is refused before anything is launched, what only interleaves is not.
Calls run on the host code alone, with a stand-in for the runtime, so that none of them, refused or not, reaches a GPU."""
import os
import shutil
import subprocess

import pytest

import paper_2009_05766_amd as nm
from lm_calls import BF16, GELU, ROOT, at, compiled, grad, linear, orth, policy, preference

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    return compiled(tmp_path_factory.mktemp("calls"))


def test_places_against_sets_of_bytes(tmp_path):
    exe = str(tmp_path / "places")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", os.path.join(ROOT, "tests", "places_driver.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    pairs, sharing = map(int, r.stdout.split())
    assert pairs == 200000 and 0.1 * pairs < sharing < 0.9 * pairs


SHARED = [
    (linear(64, 128, 128, y=at(0)), "y and x"), (linear(64, 128, 128, y=at(1)), "y and w"), (linear(64, 128, 128, z=at(2)), "y and z"),
    (linear(64, 128, 128, y=at(0, 64 * 128 - 1)), "y and x"), (linear(64, 128, 128, batch=3, y=at(0, 2 * 64 * 128)), "y and x"),
    (linear(64, 128, 128, bias=at(2, 5)), "y and bias"), (linear(64, 128, 128, residual=at(2, 4)), "y and residual"),
    (linear(64, 128, 128, residual=at(2), ldr=132), "y and residual"), (linear(64, 128, 128, batch=2, residual=at(2), sr=0), "y and residual"),
    (linear(64, 128, 128, z=at(1)), "z and w"), (linear(64, 128, 128, residual=at(3), z=at(3)), "z and residual"),
    (linear(64, 128, 130, dtype=BF16, work=at(0)), "the workspace and x"), (linear(64, 130, 128, dtype=BF16, work=at(2)), "the workspace and y"),
    # dx and dw may come from one launch, and both products read dy
    (grad(64, 128, 128, dx=at(2)), "dx and dy"), (grad(64, 128, 128, dtype=BF16, dx=at(2)), "dx and dy"), (grad(64, 128, 128, dw=at(2)), "dw and dy"),
    (grad(64, 128, 128, db=at(2, 7)), "db and dy"), (grad(64, 128, 128, dx=at(0)), "dx and x"), (grad(64, 128, 128, act=GELU, dx=at(0)), "dx and x"),
    (grad(64, 128, 128, act=GELU, dw=at(1)), "dw and w"), (grad(64, 128, 128, dw=at(0), act=GELU), "dw and x"), (grad(64, 128, 128, dx=at(5)), "dx and dw"),
    (grad(64, 128, 128, db=at(5, 64 * 128)), "dw and db"), (grad(64, 128, 128, db=at(4)), "dx and db"), (grad(64, 128, 128, act=GELU, work=at(3)), "the workspace and z"),
    (orth(96, 64, m_out=at(1, 4)), "m_out and m"), (orth(96, 64, m_out=at(0), m=at(1)), "m_out and g"), (orth(96, 64, out=at(1)), "m_out and out"), (orth(96, 64, work=at(1)), "the workspace and m"),
    (policy(100, 1000, grad=at(0, 1000)), "grad and logits"), (policy(100, 1000, dtype=BF16, grad=at(0, 8, 2)), "grad and logits"), (policy(100, 1000, loss=at(2)), "loss and old_logp"),
    (policy(100, 1000, logp=at(4, 99)), "logp and advantage"), (policy(100, 1000, grad=at(1)), "grad and labels"), (policy(100, 1000, loss=at(7)), "loss and logp"),
    (policy(100, 1000, loss=at(0, 99999)), "loss and logits"), (policy(100, 1000, logp=at(8, 5)), "logp and grad"),
    (preference(100, 1000, 4, grad=at(0, 1000)), "grad and logits"), (preference(100, 1000, 4, loss=at(2)), "loss and offsets"), (preference(100, 1000, 4, ratio=at(5)), "loss and ratio"),
    (preference(100, 1000, 4, ratio=at(4)), "ratio and weight"), (preference(100, 1000, 4, work=at(3)), "the workspace and ref_logp"), (preference(100, 1000, 4, work=at(7)), "the workspace and grad"),
    # rows that interleave and touch; a batch that interleaves with another
    (linear(64, 96, 128, ldx=200, ldy=200, y=at(0, 95)), "y and x"), (linear(64, 100, 128, ldx=200, ldy=200, y=at(0, 73)), "y and x"),
    (linear(64, 40, 56, batch=3, x=at(0), sx=10000, w=at(0, 2560), sw=10000, y=at(0, 2560 + 40 * 56 - 1), sy=10000), "y and w"),
]


@pytest.mark.parametrize("k", range(len(SHARED)), ids=[f"{c[0]}-{text.replace(' ', '_')}-{k}" for k, (c, text) in enumerate(SHARED)])
def test_shared_memory_is_refused(call, k):
    c, text = SHARED[k]
    (status, error, launches), = call(c)
    assert status == nm.NETMAX_EINVAL and error == text + " share memory" and launches == []


APART = [
    linear(64, 128, 128), linear(64, 128, 128, bias=at(4), residual=at(5), z=at(6)), linear(64, 128, 130, dtype=BF16), linear(64, 128, 128, x=at(0), w=at(0)),
    linear(64, 128, 128, residual=at(2)), linear(64, 128, 128, batch=3, residual=at(2)), linear(64, 128, 128, residual=at(2), ldr=140, ldy=140), linear(1, 128, 128, residual=at(2), ldr=999),
    # columns of one wide matrix; several workers' rows of parameters; a batch along the columns
    linear(64, 96, 104, ldx=200, ldy=200, y=at(0, 96)), linear(64, 96, 60, ldx=220, ldy=220, ldz=220, y=at(0, 96), z=at(0, 156)),
    linear(64, 40, 56, batch=3, x=at(0), sx=10000, w=at(0, 2560), sw=10000, y=at(0, 2560 + 40 * 56), sy=10000),
    linear(64, 32, 32, batch=4, ldx=256, sx=64, ldy=256, sy=64, y=at(0, 32)),
    grad(64, 128, 128), grad(64, 128, 128, dtype=BF16, act=GELU), grad(64, 128, 128, act=GELU, dx=at(2)), grad(64, 128, 128, act=GELU, dx=at(3), dw=at(2)), grad(64, 128, 128, act=GELU, db=at(2)),
    grad(64, 128, 128, dw=0, dx=at(0)), grad(64, 128, 128, dx=0, dw=at(1)), grad(64, 128, 128, dx=0, dw=0, db=at(2)), grad(0, 128, 128, dy=0, x=0, dw=at(2)),
    grad(50, 40, 56, batch=3, dw=at(5, 7), sdw=2309, db=at(5, 7 + 40 * 56), sdb=2309),
    orth(96, 64), orth(96, 64, out=at(0)), orth(96, 64, out=at(0, 12)), orth(96, 64, m=0, m_out=0, out=at(0)), orth(96, 64, m_out=at(4), out=at(1)),
    policy(100, 1000), policy(100, 1000, grad=at(0)), policy(100, 1000, ld=3000, grad=at(0, 1500), ldg=3000), policy(100, 1000, grad=0, logp=0), policy(1, 1000, grad=at(0), ldg=1000),
    preference(100, 1000, 4), preference(100, 1000, 4, grad=at(0)), preference(0, 1000, 4, logits=0, labels=0, ref_logp=0, weight=0),
]


@pytest.mark.parametrize("k", range(len(APART)), ids=[f"{c[0]}-{k}" for k, c in enumerate(APART)])
def test_what_lies_apart_is_launched(call, k):
    (status, error, launches), = call(APART[k])
    assert status == nm.NETMAX_OK and error == "" and len(launches) >= 1


OVERLAPPING = [
    (linear(64, 128, 128, batch=3, sy=1), "y"), (linear(64, 128, 128, batch=3, sy=64 * 128 - 1), "y"), (linear(64, 128, 128, batch=3, z=at(3), sz=100), "z"),
    (linear(64, 32, 32, batch=4, ldy=128, sy=31), "y"), (linear(64, 32, 32, batch=5, ldy=128, sy=32), "y"),
    (grad(64, 128, 128, batch=3, sdx=128), "dx"), (grad(64, 128, 128, batch=3, sdw=4), "dw"), (grad(64, 128, 128, batch=3, sdb=127), "db"),
    (orth(96, 64, batch=2, so=64), "out"), (orth(96, 64, batch=2, sm=64, m_out=at(5)), "m_out"),
]


@pytest.mark.parametrize("k", range(len(OVERLAPPING)), ids=[f"{c[0]}-{name}-{k}" for k, (c, name) in enumerate(OVERLAPPING)])
def test_results_of_a_batch_that_overlap_are_refused(call, k):
    c, name = OVERLAPPING[k]
    (status, error, launches), = call(c)
    assert status == nm.NETMAX_EINVAL and error.startswith(name + ":") and error.endswith("results in the same place") and launches == []


@pytest.mark.parametrize("c", [linear(64, 32, 32, batch=4, ldy=128, sy=32), linear(1, 32, 32, batch=4, ldy=1, sy=32), linear(64, 32, 32, batch=4, ldy=32, sy=64 * 32, ldx=128, sx=0),
                               grad(64, 32, 32, batch=3, lddw=96, sdw=32, sdb=32), orth(8, 4, batch=3, ldo=12, so=4)], ids=lambda c: c[0])
def test_results_of_a_batch_that_interleave_are_written(call, c):
    (status, error, launches), = call(c)
    assert status == nm.NETMAX_OK and len(launches) >= 1
