"""Where the kernels around a language model's layers work, on the host code of the built library with a stand-in for the runtime (lm_step_places_driver.cpp): no GPU follows an address."""
import os
import shutil
import subprocess

import pytest

import paper_2009_05766_amd as nm
from lm_calls import BF16, F32, ROOT
from paper_2009_05766_amd.build import LIB, build
from test_lm_step_routes import embed, norm

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"), reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def call(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("places") / "drive")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "lm_step_places_driver.cpp"), "-rdynamic", "-ldl", "-o", exe], check=True)
    lib = LIB if os.path.exists(LIB) else build()

    def run(*calls):
        """-> for each call: launches and what is wrong with them as (name, number)."""
        lines = "\n".join(" ".join([op] + [f"{k}={n!r}" for k, n in v.items()]) for op, v in calls)
        r = subprocess.run([exe, lib], input=lines, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line, c in zip(r.stdout.splitlines(), calls):
            status, text, launches = line.split("|")
            assert int(status) == nm.NETMAX_OK, (c, text)
            out.append([(k.rsplit("@", 1)[0], int(k.rsplit("@", 1)[1])) for k in launches.split()])
        return out
    return run


WRONG = ("behind_the_workspace", "sums_of_no_rows", "clears_kept_rows", "clears_behind_the_table")


def wrong(call, calls):
    """What is wrong with launches, with the call."""
    return [(c, k, n) for c, launches in zip(calls, call(*calls)) for k, n in launches if k in WRONG]


FORMS = [dict(block=False), dict(block=False, bias=True), dict(gate="channel"), dict(gate="channel", bias=True), dict(gate="rows"), dict(gate="rows", bias=True), dict(gate="rows", pre=False)]


@pytest.mark.parametrize("batch", [1, 2, 4, 8, 300])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_norms_stay_in_their_workspace(call, dtype, batch):
    """Whatever of the results is wanted, or written over what is read."""
    calls = []
    for rows in (1, 2, 10, 64, 512, 5000):
        for width in (2, 40, 64, 130, 300, 700, 1500, 3000, 5000, 6000, 8192, 8200, 9000, 12000, 13000, 16384, 20000):
            if batch * rows * width * 4 >= 60 << 30:                # operands lie 64 GiB apart
                continue
            for form in FORMS:
                v = norm(rows, width, dtype, batch=batch, **form)[1][1]
                outs = [n for n in ("dx", "df", "dgate") if n in v and (n != "dgate" or v["gate_rows"])]
                sums = [n for n in v if n.startswith("d") and n.split("_")[0] in ("dpost", "dpre") and "." not in n] + ["dgate"] * (not v["gate_rows"] and "dgate" in v)
                calls.append(("norm_grad", v))
                for missing in ([outs] + [[n] for n in outs] if len(outs) > 1 else [outs]):
                    calls.append(("norm_grad", dict(v, **{n: 0 for n in missing})))
                    calls.append(("norm_grad", dict(v, **{n: 0 for n in [*missing, *sums]})))
                calls.append(("norm_grad", dict(v, dx=v["x"])))
                if "df" in v:
                    calls.append(("norm_grad", dict(v, dx=v["dh"], df=v["x"])))
    assert wrong(call, calls) == []


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_no_rows_join_nothing(call, dtype):
    calls = [norm(0, width, dtype, batch=batch, **form, **{n + ".s": width for n in ("dx", "df", "dgate")})[1] for batch in (1, 2, 300, 3000, 65535) for width in (3, 100, 5000, 9000, 16384, 40000) for form in FORMS]
    assert wrong(call, calls) == [] and all(launches for launches in call(*calls))


def test_results_without_rows_have_any_distance(call):
    """Matrices of no rows lie 0 apart where they lie next to each other: they share no memory, and the sums over their rows are 0."""
    calls = [norm(0, 40, batch=3, **form)[1] for form in FORMS]
    assert all(c[1]["dx.s"] == 0 for c in calls) and all(launches for launches in call(*calls))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_embeddings_clear_what_they_may(call, dtype):
    """Launches of more workgroups than go along one dimension are rounded up: what is added clears nothing."""
    sizes = [(1, 10, 8), (300, 90, 100), (2048, 33, 2000), (2049, 17, 40), (5000, 6000, 100), (40000, 131072, 64)]
    wide = ((1 << 22) - 4) // (1 + dtype)
    sizes += [(513 * (1 + 3 * dtype), 20, wide), (2048, 20, wide), (2048, 60000, wide // 8), (1 << 24, 100, 16384), (1 << 25, 1000, 8200), (1 << 30, 5, 7)]
    calls = [c for n, vocab, width in sizes for c in embed(n, vocab, width, dtype=dtype, table=1 << 47, y=1 << 48, work=1 << 49)]
    assert all(launches for launches in call(*calls))
    assert wrong(call, calls) == []
