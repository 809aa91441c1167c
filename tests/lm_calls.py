"""Calls of the operators for language models on the host code of the built library, without a GPU: tests/lm_calls_driver.cpp stands in for the runtime."""
import os
import subprocess

from paper_2009_05766_amd.build import LIB, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1
NONE, RELU, GELU, SILU = range(4)


def at(k, elements=0, size=4):
    """An address of its own for every k, aligned, with 64 GiB of room."""
    return (k + 1) * (1 << 36) + elements * size


def linear(rows, d_in, d_out, batch=1, dtype=F32, act=NONE, **kw):
    v = dict(batch=batch, rows=rows, d_in=d_in, d_out=d_out, dtype=dtype, act=act, ldx=d_in, ldw=d_out, ldr=d_out, ldy=d_out, ldz=d_out, x=at(0), w=at(1), y=at(2), work=at(9))
    v.update(kw)
    for s, n, ld in (("sx", rows, "ldx"), ("sw", d_in, "ldw"), ("sr", rows, "ldr"), ("sy", rows, "ldy"), ("sz", rows, "ldz")):
        v.setdefault(s, n * v[ld])
    v.setdefault("sb", d_out)
    return "linear", v


def grad(rows, d_in, d_out, batch=1, dtype=F32, act=NONE, **kw):
    v = dict(lddx=d_in, lddw=d_out, dy=at(2), z=at(3) if act else 0, dx=at(4), dw=at(5), db=at(6))
    v.update(kw)
    v = linear(rows, d_in, d_out, batch, dtype, act, **v)[1]
    v.setdefault("sdx", rows * v["lddx"])
    v.setdefault("sdw", d_in * v["lddw"])
    v.setdefault("sdb", d_out)
    return "grad", v


def orth(rows, cols, batch=1, dtype=F32, **kw):
    v = dict(batch=batch, rows=rows, cols=cols, dtype=dtype, steps=5, nesterov=1, mu=0.95, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, scale=1.0, ldg=cols, ldm=cols, ldo=cols, sg=rows * cols,
             sm=rows * cols, so=rows * cols, g=at(0), m=at(1), m_out=at(1), out=at(2), work=at(9))
    v.update(kw)
    return "orth", v


def policy(tokens, vocab, dtype=F32, **kw):
    v = dict(tokens=tokens, vocab=vocab, dtype=dtype, logits=at(0), ld=vocab, labels=at(1), old_logp=at(2), ref_logp=at(3), advantage=at(4), weight=at(5), low=0.2, high=0.2, kl=0.1, loss=at(6),
             logp=at(7), grad=at(8), ldg=vocab)
    v.update(kw)
    return "policy", v


def preference(tokens, vocab, pairs, dtype=F32, **kw):
    v = dict(tokens=tokens, vocab=vocab, pairs=pairs, dtype=dtype, logits=at(0), ld=vocab, labels=at(1), offsets=at(2), ref_logp=at(3), weight=at(4), beta=0.1, smoothing=0.0, scale=1.0, loss=at(5),
             ratio=at(6), grad=at(7), ldg=vocab, work=at(9))
    v.update(kw)
    return "preference", v


def compiled(folder):
    exe = str(folder / "drive")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", os.path.join(ROOT, "tests", "lm_calls_driver.cpp"), "-rdynamic", "-ldl", "-o", exe],
                   check=True)
    lib = LIB if os.path.exists(LIB) else build()

    def run(*calls):
        """-> for each call: status, text of the error, launches as (kernel, workgroups)."""
        lines = "\n".join(" ".join([op] + [f"{k}={n!r}" for k, n in v.items()]) for op, v in calls)
        r = subprocess.run([exe, lib], input=lines, capture_output=True, text=True, timeout=120)
        assert r.returncode == 0, r.stderr
        out = []
        for line in r.stdout.splitlines():
            status, text, launches = line.split("|")
            out.append((int(status), text, [(k.rsplit("@", 1)[0], int(k.rsplit("@", 1)[1])) for k in launches.split()]))
        return out
    return run
