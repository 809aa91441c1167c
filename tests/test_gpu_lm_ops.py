"""The operators for language models against plain implementations in 64 bits.

Tolerances.  Linear layers: a float sum of K products differs from the exact one by at most (K + 4) 2^-24 times the sum of the products'
magnitudes; a result in bfloat16 is off by 2^-8 of itself more, half a unit in the last of its 8 bits (2^-24 for float); through an activation an error grows by at most 1.2 (the
largest slope of GELU and SiLU is below that), through its slope by at most 1.0 (their second derivatives stay below).  What goes into a product as bfloat16 (dz, and
z in memory) brings its own 2^-8.  These bounds are propagated element by element.
Losses: log probabilities are exact to a few 2^-24 of their terms; a probability's exponential to 2^-21 plus 2^-22 for each unit of its argument.
Orthogonalised updates: the norm of the difference.  Float: every one of the 3 x 5 products is exact to about 2^-22, which the polynomial
(slope up to 3.4 per step, falling with the singular values it lifts) carries to below 1e-5 of the result.  bfloat16 results: 2^-9 / sqrt(3) = 1.1e-3 to
2^-8 / sqrt(3) = 2.3e-3 by their own rounding, and less than that again by operands of 11 bits in the products: 4e-3."""
import math

import pytest
import torch

import paper_2009_05766_amd as nm

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def strided(t, pad):
    """The same values with rows `pad` further apart, and something that must not be touched between them."""
    wide = torch.full((*t.shape[:-1], t.shape[-1] + pad), float("nan"), device=t.device, dtype=t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z / math.sqrt(2)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def within(got, want, tol, what):
    d = (got.double() - want).abs()
    bad = ~(d <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((d / tol.clamp(min=1e-300)).max()):.3g} of the bound"


def check_linear(rows, d_in, d_out, dtype, act, batch=0, bias=True, residual=True, pad=0, grad=True, seed=0):
    g = gen(seed)
    lead = (batch,) if batch else ()
    put = (lambda t: strided(t, pad)) if pad else (lambda t: t)
    x, w = put(normal(g, *lead, rows, d_in, dtype=dtype)), put(normal(g, *lead, d_in, d_out, dtype=dtype, scale=d_in ** -0.5))
    b = normal(g, *lead, d_out, dtype=dtype) if bias else None
    r = put(normal(g, *lead, rows, d_out, dtype=dtype)) if residual else None
    y, z = nm.netmax_linear(x, w, b, r, act=act, keep_preact=True)
    X, W = x.double(), w.double()
    Z, mag = X @ W, X.abs() @ W.abs()
    if bias:
        Z, mag = Z + b.double().unsqueeze(-2), mag + b.double().abs().unsqueeze(-2)
    u, e = ULP[dtype], (d_in + 4) * 2.0 ** -24
    within(z, Z, e * mag + u * Z.abs(), "z")
    Y = act64(Z, act) + (r.double() if residual else 0)
    within(y, Y, 1.2 * e * mag + (u + 2.0 ** -21) * (Y.abs() + (Z.abs() + 1e-6 if act != "none" else 0) * 2.0 ** -12) + 2.0 ** -22 * (Z.abs() + (r.double().abs() if residual else 0)), "y")
    if not grad:
        return
    dy = put(normal(g, *lead, rows, d_out, dtype=dtype))
    dx, dw, db = nm.netmax_linear_grad(dy, x, w, z if act != "none" else None, act=act)
    used = z.double()                                  # the derivative is taken where the forward pass left z
    DY = dy.double()
    dz = DY * slope64(used, act)
    tz = DY.abs() * 2.0 ** -20 * (1 + used.abs()) + (u if dtype == BF16 and act != "none" else 0) * dz.abs() + 1e-30
    at = lambda t: t.transpose(-1, -2)  # noqa: E731
    for got, want, tol, m, k, name in (
            (dx, dz @ at(W), tz @ at(W).abs(), dz.abs() @ at(W).abs(), d_out, "dx"),
            (dw, at(X) @ dz, at(X).abs() @ tz, at(X).abs() @ dz.abs(), rows, "dw"),
            (db, dz.sum(-2), (DY.abs() * 2.0 ** -20 * (1 + used.abs())).sum(-2) + 1e-30, dz.abs().sum(-2), rows, "db")):
        within(got, want, tol + (k + 4) * 2.0 ** -24 * m + u * want.abs(), name)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(1, 1, 1), (1, 64, 64), (1, 1000, 333), (2, 77, 1030), (17, 33, 65), (64, 784, 512), (65, 128, 136), (128, 256, 256), (129, 257, 255),
                                             (255, 1000, 264), (300, 72, 700), (1000, 40, 24), (513, 520, 1032)])
def test_linear_sizes(rows, d_in, d_out, dtype):
    check_linear(rows, d_in, d_out, dtype, "gelu", seed=rows)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("rows", [1, 96])
def test_linear_activations(act, dtype, rows):
    check_linear(rows, 192, 320, dtype, act, bias=False, residual=False, seed=1)
    check_linear(rows, 192, 320, dtype, act, bias=True, residual=False, seed=2)
    check_linear(rows, 192, 320, dtype, act, bias=False, residual=True, seed=3)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,d_in,d_out", [(1, 5, 40, 48), (3, 1, 136, 200), (16, 64, 784, 512), (5, 33, 129, 67), (2, 300, 256, 520)])
def test_linear_batches(batch, rows, d_in, d_out, dtype):
    check_linear(rows, d_in, d_out, dtype, "silu", batch=batch, seed=batch)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,d_in,d_out", [(100, 250, 250, 500), (300, 200, 72, 64), (200, 100, 96, 80), (40, 500, 120, 33), (40, 70, 40, 600), (300, 70, 300, 20)])
def test_linear_large_batches_of_small_layers(batch, rows, d_in, d_out, dtype):
    check_linear(rows, d_in, d_out, dtype, "gelu", batch=batch, seed=batch + rows)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 3, 8, 24])
@pytest.mark.parametrize("batch", [0, 3])
def test_linear_distances_of_rows(pad, batch, dtype):
    check_linear(70, 264, 200, dtype, "gelu", batch=batch, pad=pad, seed=pad)
    check_linear(1, 264, 200, dtype, "gelu", batch=batch, pad=pad, seed=pad + 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [2048, 4099])
def test_linear_long(rows, dtype):
    check_linear(rows, 512, 768, dtype, "gelu", seed=rows)
    check_linear(rows, 96, 80, dtype, "none", seed=rows + 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,d_in,d_out", [(4100, 72, 3080), (72, 3500, 4100), (3600, 4001, 99), (5000, 200, 10), (9000, 65, 127)])
def test_linear_many_blocks(rows, d_in, d_out, dtype):
    """Results wide enough for the largest blocks in the forward pass, in dw and in dx, with edges; long contractions onto few results."""
    check_linear(rows, d_in, d_out, dtype, "silu", seed=rows)


@pytest.mark.parametrize("rows,d_in,d_out,batch", [(1600, 1601, 1602, 0), (2048, 1024, 2048, 0), (700, 2304, 2305, 2), (3000, 1500, 1030, 0)])
def test_linear_large_in_float(rows, d_in, d_out, batch):
    """Products that are worth planes of halves."""
    check_linear(rows, d_in, d_out, F32, "gelu", batch=batch, seed=rows)
    check_linear(rows, d_in, d_out, F32, "none", batch=batch, pad=3, seed=rows + 1)


def test_linear_large_in_float_over_many_magnitudes():
    """Rows of x and columns of w from 1e-30 to 1e+6, an infinity in one row, a NaN in another: every other result as exact as its own magnitudes allow."""
    g = gen(12)
    n = 1664
    x = normal(g, n, n) * 10.0 ** (torch.rand(n, 1, generator=g, device="cuda") * 36 - 30)
    w = normal(g, n, n) * 10.0 ** (torch.rand(1, n, generator=g, device="cuda") * 16 - 10)
    x[5] = 0.0
    w[:, 9] = 0.0
    keep = x.clone()
    x[3, 7], x[4, 8], x[6, 0] = float("inf"), float("nan"), 3e38
    y = nm.netmax_linear(x, w)
    rows = torch.ones(n, dtype=torch.bool, device="cuda")
    rows[3] = rows[4] = rows[6] = False
    X, W = keep.double(), w.double()
    want, mag = X @ W, X.abs() @ W.abs()
    within(y[rows], want[rows], ((n + 4) * 2.0 ** -24 * mag + 2.0 ** -24 * want.abs() + 2.0 ** -149)[rows], "y")
    live = torch.ones(n, dtype=torch.bool, device="cuda")
    live[9] = False
    assert not bool(torch.isfinite(y[3:5][:, live]).any())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [31, 32, 33, 63, 64])
@pytest.mark.parametrize("d_in,d_out", [(40, 1000), (1000, 40), (4104, 72)])
def test_linear_few_rows(rows, d_in, d_out, dtype):
    check_linear(rows, d_in, d_out, dtype, "gelu", seed=rows)
    check_linear(rows, d_in, d_out, dtype, "none", batch=3, pad=8, seed=rows + 1)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_linear_into_given_memory(dtype):
    """Slices of a worker's row of parameters as w, b and their gradients; what lies beside them keeps its values.  In place onto the residual."""
    g = gen(5)
    M, rows, d_in, d_out = 3, 50, 40, 56
    D = 7 + d_in * d_out + d_out + 5
    params = normal(g, M, D, dtype=dtype, scale=0.1)
    grads = torch.full((M, D), 3.0, dtype=dtype, device="cuda")
    cut = lambda t: (t[:, 7:7 + d_in * d_out].view(M, d_in, d_out), t[:, 7 + d_in * d_out:7 + d_in * d_out + d_out])  # noqa: E731
    w, b = cut(params)
    x, r, dy = normal(g, M, rows, d_in, dtype=dtype), normal(g, M, rows, d_out, dtype=dtype), normal(g, M, rows, d_out, dtype=dtype)
    want = nm.netmax_linear(x, w.contiguous(), b.contiguous(), r)
    y = r.clone()
    assert nm.netmax_linear(x, w, b, y, y=y) is y
    assert torch.equal(y, want)
    dw, db = cut(grads)
    got = nm.netmax_linear_grad(dy, x, w, dw=dw, db=db)
    ref = nm.netmax_linear_grad(dy, x, w.contiguous())
    for a, c in zip(got, ref):
        assert torch.equal(a, c)
    left = torch.ones(D, dtype=torch.bool)
    left[7:7 + d_in * d_out + d_out] = False
    assert bool((grads[:, left.cuda()] == 3.0).all())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_linear_nothing(dtype):
    x, w = torch.empty(0, 24, dtype=dtype, device="cuda"), torch.ones(24, 40, dtype=dtype, device="cuda")
    assert nm.netmax_linear(x, w).shape == (0, 40)
    dx, dw, db = nm.netmax_linear_grad(torch.empty(0, 40, dtype=dtype, device="cuda"), x, w)
    assert dx.shape == (0, 24) and bool((dw == 0).all()) and bool((db == 0).all())
    assert nm.netmax_linear(torch.empty(0, 5, 24, dtype=dtype, device="cuda"), torch.empty(0, 24, 40, dtype=dtype, device="cuda")).shape == (0, 5, 40)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 70])
def test_linear_values_that_are_not_finite(rows, dtype):
    """A row that holds an infinity or a NaN reaches its own results only; infinite weights their own columns."""
    g = gen(6)
    x, w = normal(g, rows + 2, 136, dtype=dtype), normal(g, 136, 72, dtype=dtype)
    x[0, 3], x[1, 135] = float("nan"), float("inf")
    y = nm.netmax_linear(x, w)
    assert not bool(torch.isfinite(y[:2]).any())
    assert torch.equal(y[2:], nm.netmax_linear(x[2:], w)) or bool(torch.isfinite(y[2:]).all())
    w[:, 5] = float("inf")
    y = nm.netmax_linear(x[2:], w)
    assert not bool(torch.isfinite(y[:, 5]).any()) and bool(torch.isfinite(y[:, 6:]).all()) and bool(torch.isfinite(y[:, :5]).all())


def test_activations_far_out():
    z = torch.tensor([[-3e38, -1e30, -200.0, -90.0, -1e-40, 0.0, 1e-40, 90.0, 200.0, 1e30, 3e38]], device="cuda")
    one, eye = torch.ones(1, 11, device="cuda"), torch.eye(11, device="cuda")
    for act in ("relu", "gelu", "silu"):
        y = nm.netmax_linear(z, eye, act=act)
        assert torch.allclose(y.double(), act64(z.double(), act), rtol=1e-5, atol=1e-37), act
        dx, _, _ = nm.netmax_linear_grad(one, z, eye, z, act=act)
        assert torch.allclose(dx.double(), slope64(z.double(), act).nan_to_num(0.0), rtol=1e-5, atol=1e-30), act


def test_linear_gradient_against_differences():
    g = gen(7)
    x, w, b = normal(g, 6, 24), normal(g, 24, 16, scale=0.2), normal(g, 16)
    dy = normal(g, 6, 16)
    for act in ("gelu", "silu"):
        _, z = nm.netmax_linear(x, w, b, act=act, keep_preact=True)
        grads = nm.netmax_linear_grad(dy, x, w, z, act=act)
        for k, t in enumerate((x, w, b)):
            v, h = normal(g, *t.shape), 1e-2
            ends = []
            for s in (h, -h):
                a = [x, w, b]
                a[k] = t + s * v
                ends.append(float((nm.netmax_linear(*a, act=act).double() * dy.double()).sum()))
            want, got = (ends[0] - ends[1]) / (2 * h), float((grads[k].double() * v.double()).sum())
            # third differences are of order h^2 |v|^3, the sums' rounding 2^-24 of a few hundred over h
            assert abs(got - want) < 2e-2 * max(1.0, abs(want)), (act, k, got, want)


# ---- orthogonalised updates ------------------------------------------------------------------------------------------

def orth64(g, m, mu, nesterov, steps=5, co=(3.4445, -4.7750, 2.0315), eps=1e-7, scale=1.0):
    g = g.double()
    co = [float(torch.tensor(v, dtype=F32)) for v in co]
    mu = float(torch.tensor(mu, dtype=F32))
    if m is not None:
        m = mu * m.double() + g
        u = g + mu * m if nesterov else m
    else:
        u = g
    x = u / torch.linalg.matrix_norm(u).clamp(min=eps)[..., None, None]
    for _ in range(steps):
        if g.shape[-2] > g.shape[-1]:
            p = x.transpose(-1, -2) @ x
            x = co[0] * x + x @ (co[1] * p + co[2] * p @ p)
        else:
            p = x @ x.transpose(-1, -2)
            x = co[0] * x + (co[1] * p + co[2] * p @ p) @ x
    return scale * x, m


def gradient_like(g, b, m, n, dtype):
    r = max(1, min(m, n) // 8)
    return (torch.randn(b, m, r, generator=g, device="cuda") @ torch.randn(b, r, n, generator=g, device="cuda") * r ** -0.5
            + 0.5 * torch.randn(b, m, n, generator=g, device="cuda")).mul_(1e-3).to(dtype)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


ORTH_TOL = {F32: 1e-5, BF16: 4e-3}


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 300), (3, 300, 1), (4, 32, 32), (2, 33, 70), (16, 784, 512), (3, 129, 128), (2, 512, 10), (1, 700, 1501), (5, 128, 256), (2, 1000, 1000),
                                             (1, 1024, 2048), (1, 2050, 1030)])
def test_orthogonalize_sizes(batch, rows, cols, dtype):
    g = gen(rows + cols)
    a, m = gradient_like(g, batch, rows, cols, dtype), gradient_like(g, batch, rows, cols, F32) * 5
    want, m64 = orth64(a, m, 0.95, True)
    kept = m.clone()
    got = nm.netmax_orthogonalize(a, m, mu=0.95)
    assert got.dtype == dtype and off(m, m64) < 1e-7
    assert off(got, want) < ORTH_TOL[dtype]
    m2 = torch.empty_like(m)
    again = nm.netmax_orthogonalize(a, kept, m_out=m2, mu=0.95)
    assert torch.equal(again, got) and torch.equal(m2, m)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,cols", [(64, 300, 520), (66, 530, 290), (64, 264, 257), (200, 65, 140), (150, 200, 130)])
def test_orthogonalize_many_matrices(batch, rows, cols, dtype):
    """Enough blocks for every block shape, with edges."""
    g = gen(batch)
    a = gradient_like(g, batch, rows, cols, dtype)
    want, _ = orth64(a, None, 0.0, False)
    got = nm.netmax_orthogonalize(a)
    assert max(off(got[k], want[k]) for k in range(batch)) < ORTH_TOL[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("batch,rows,cols", [(200, 250, 500), (200, 500, 250), (300, 60, 70), (600, 33, 120), (150, 128, 100)])
def test_orthogonalize_many_matrices_that_fill_their_blocks(batch, rows, cols, dtype):
    """As above; blocks are chosen by what lies behind the edges, too."""
    test_orthogonalize_many_matrices(batch, rows, cols, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_orthogonalize_forms(dtype):
    g = gen(3)
    a, m = gradient_like(g, 2, 96, 160, dtype), gradient_like(g, 2, 96, 160, F32)
    for kw, mom in ((dict(nesterov=False, mu=0.9), m), (dict(), None), (dict(steps=1), m), (dict(steps=8, coefficients=(2.0, -1.5, 0.5)), m), (dict(scale=0.25), m)):
        want, _ = orth64(a, mom, kw.get("mu", 0.95), kw.get("nesterov", True), kw.get("steps", 5), kw.get("coefficients", (3.4445, -4.7750, 2.0315)), scale=kw.get("scale", 1.0))
        got = nm.netmax_orthogonalize(a, None if mom is None else mom.clone(), **kw)
        assert off(got, want) < ORTH_TOL[dtype], kw
    one = nm.netmax_orthogonalize(a[0], m[0].clone())
    assert off(one, orth64(a, m, 0.95, True)[0][0]) < ORTH_TOL[dtype]


def test_orthogonalize_singular_values():
    """By definition: the singular vectors stay, each singular value goes through the polynomial."""
    g = gen(4)
    a = gradient_like(g, 1, 120, 200, F32)[0]
    u, s, v = torch.linalg.svd(a.double().cpu(), full_matrices=False)
    s = s / s.norm()
    co = [float(torch.tensor(c, dtype=F32)) for c in (3.4445, -4.7750, 2.0315)]
    for _ in range(5):
        s = co[0] * s + co[1] * s ** 3 + co[2] * s ** 5
    assert off(nm.netmax_orthogonalize(a).cpu(), u * s @ v) < ORTH_TOL[F32]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_orthogonalize_zero_tiny_and_not_finite(dtype):
    a = torch.zeros(4, 40, 72, dtype=dtype, device="cuda")
    g = gen(5)
    a[1] = gradient_like(g, 1, 40, 72, dtype)[0]
    a[2] = (gradient_like(g, 1, 40, 72, F32)[0] * 1e-3 * 2.0 ** -100).to(dtype)
    a[3] = a[1]
    a[3, 7, 9] = float("nan")
    got = nm.netmax_orthogonalize(a, eps=1e-37)
    assert bool((got[0] == 0).all()) and not bool(torch.isfinite(got[3]).all())
    for k in (1, 2):
        assert off(got[k], orth64(a, None, 0.0, False, eps=1e-37)[0][k]) < ORTH_TOL[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_orthogonalize_strides_and_in_place(dtype):
    """Weight slices of workers' parameter rows, an update into such rows, in place over the gradient."""
    g = gen(6)
    M, m, n = 3, 48, 40
    D = 11 + m * n + 6
    a = gradient_like(g, M, m, n, dtype)
    rows, moms = torch.full((M, D), 3.0, dtype=dtype, device="cuda"), torch.full((M, D), 3.0, device="cuda")
    cut = lambda t: t[:, 11:11 + m * n].view(M, m, n)  # noqa: E731
    cut(rows).copy_(a)
    cut(moms).copy_(gradient_like(g, M, m, n, F32))
    want = nm.netmax_orthogonalize(a, cut(moms).clone())
    assert torch.equal(nm.netmax_orthogonalize(cut(rows), cut(moms), out=cut(rows)), want)
    assert torch.equal(cut(rows), want)
    for t in (rows, moms):
        assert bool((t[:, :11] == 3.0).all()) and bool((t[:, 11 + m * n:] == 3.0).all())
    wide = strided(a, 5)
    assert torch.equal(nm.netmax_orthogonalize(wide), nm.netmax_orthogonalize(a))
    assert nm.netmax_orthogonalize(a[:0]).shape == (0, m, n)


# ---- losses ----------------------------------------------------------------------------------------------------------

def logits_and_labels(g, t, v, dtype, scale=3.0):
    z = normal(g, t, v, dtype=dtype, scale=scale)
    return z, torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)


def logp64(z, labels):
    q = torch.log_softmax(z.double(), 1)
    return q.gather(1, labels.long()[:, None])[:, 0], q


def grad64(q, labels, slope):
    s = slope.double()[:, None]
    return torch.zeros_like(q).scatter_(1, labels.long()[:, None], s) - s * q.exp()


def policy64(logp, old, ref, adv, w, low, high, kl):
    logp = logp.detach().clone().requires_grad_()
    r, a = torch.exp(logp - old.double()), adv.double()
    low, high, kl = (float(torch.tensor(v, dtype=F32)) for v in (low, high, kl))
    loss = -torch.minimum(r * a, r.clamp(1 - low, 1 + high) * a)
    if kl:
        d = ref.double() - logp
        loss = loss + kl * (torch.exp(d) - d - 1)
    loss = w.double() * loss
    return loss.detach(), torch.autograd.grad(loss.sum(), logp)[0], slope_terms(logp.detach(), old, ref, adv, w, kl)


def slope_terms(logp, old, ref, adv, w, kl):
    """Magnitudes of the terms that a token's slope is the sum of: they may cancel, their rounding does not."""
    terms = (torch.exp(logp - old.double()) * adv.double()).abs()
    return w.double().abs() * (terms + (kl * (1 + torch.exp(ref.double() - logp)) if kl else 0))


def check_grad(got, q, labels, slope, dtype, terms=None):
    want = grad64(q, labels, slope)
    p = q.exp()
    own = torch.zeros_like(slope) if terms is None else terms * 2.0 ** -20             # the slope's own error
    tol = own[:, None] * p + slope.double().abs()[:, None] * (p * (2.0 ** -21 + 2.0 ** -22 * q.abs().clamp(max=200)) + 2.0 ** -21 * (want != 0) * (p > 1e-3)) + (ULP[dtype] + 2.0 ** -20) * want.abs() + 1e-38
    at = labels.long()[:, None]
    tol.scatter_add_(1, at, (slope.double().abs() * 2.0 ** -20 + own)[:, None])
    within(got, want, tol, "gradient")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens,vocab", [(1, 1), (1, 2), (3, 7), (5, 255), (2, 257), (40, 1000), (300, 5001), (64, 16384), (33, 32001), (9, 50000), (7, 131072), (3, 131073), (2, 262150), (1, 300000)])
def test_policy_loss_sizes(tokens, vocab, dtype):
    g = gen(tokens + vocab)
    z, labels = logits_and_labels(g, tokens, vocab, dtype)
    lp, q = logp64(z, labels)
    old, ref = (lp - torch.round(normal(g, tokens, scale=10).double()) * 0.02 - 0.01).float(), (lp + normal(g, tokens, scale=0.3)).float()
    adv, w = normal(g, tokens), torch.rand(tokens, generator=g, device="cuda") + 0.1
    for kl in (0.0, 0.1):
        loss, logp, grad = nm.netmax_policy_loss(z, labels, old, adv, w, ref_logp=ref if kl else None, kl=kl)
        want, slope, terms = policy64(lp, old, ref, adv, w, 0.2, 0.2, kl)
        within(logp, lp, 2.0 ** -23 * lp.abs() + 2.0 ** -20, "log probability")
        within(loss, want, (want.abs() + w.double() * adv.double().abs() * 3 + 1) * 2.0 ** -18, "loss")
        check_grad(grad, q, labels, slope, dtype, terms)
        only, _, none = nm.netmax_policy_loss(z, labels, old, adv, w, ref_logp=ref if kl else None, kl=kl, need_grad=False)
        assert none is None and torch.equal(only, loss)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_policy_loss_rows_without_weight_and_masks(dtype):
    g = gen(8)
    t, v = 12, 1003
    z, labels = logits_and_labels(g, t, v, dtype)
    lowest = torch.finfo(dtype).min
    z[1] = float("nan")                                # no weight: not looked at
    z[2] = float("inf")
    labels[3], labels[4] = -100, v                     # labels that are no token
    z[5, 100:] = float("-inf")                         # masked vocabulary
    labels[5] = 17
    z[6, ::2] = lowest
    labels[6] = 1
    z[7] = lowest                                      # everything at the type's lowest value: uniform
    z[8] = float("-inf")                               # nothing left
    z[9, 5:] = float("-inf")
    labels[9] = 700                                    # a masked label
    w = torch.ones(t, device="cuda")
    w[1] = w[2] = 0.0
    old, adv = torch.full((t,), -5.0, device="cuda"), torch.ones(t, device="cuda")
    kept = z.clone()
    loss, logp, grad = nm.netmax_policy_loss(z, labels, old, adv, w)
    for k in (1, 2, 3, 4):
        assert float(loss[k]) == 0.0 and float(logp[k]) == 0.0 and bool((grad[k] == 0).all()), k
    assert float(logp[8]) == float("-inf") and float(loss[8]) == 0.0 and bool((grad[8] == 0).all())
    assert float(logp[9]) == float("-inf") and bool((grad[9] == 0).all())
    assert bool((grad[5, 100:] == 0).all()) and bool(torch.isfinite(grad[5:]).all())
    assert float(logp[7]) == pytest.approx(-math.log(v), rel=1e-6)
    for k in (0, 5, 6, 7, 10, 11):
        lp, q = logp64(z[k:k + 1], labels[k:k + 1])
        assert float(logp[k]) == pytest.approx(float(lp), rel=1e-6)
        want, slope, terms = policy64(lp, old[k:k + 1], old, adv[k:k + 1], w[k:k + 1], 0.2, 0.2, 0.0)
        check_grad(grad[k:k + 1], q.nan_to_num(neginf=-1e4), labels[k:k + 1], slope, dtype, terms)
    again = nm.netmax_policy_loss(z, labels, old, adv, w, grad=z)         # in the logits' place
    assert torch.equal(again[2], grad) and again[2].data_ptr() == z.data_ptr()
    wide = strided(kept, 3)
    assert torch.equal(nm.netmax_policy_loss(wide, labels, old, adv, w)[2], grad)
    out = strided(kept, 5)
    nm.netmax_policy_loss(kept, labels, old, adv, w, grad=out)
    assert torch.equal(out, grad) and bool(torch.isnan(out.as_strided((t, 5), (v + 5, 1), v)).all())
    z = kept.clone()
    z[0, 500] = float("nan")
    loss, logp, grad = nm.netmax_policy_loss(z, labels, old, adv, w)
    assert math.isnan(float(loss[0])) and math.isnan(float(logp[0])) and bool(torch.isnan(grad[0]).all()) and math.isfinite(float(loss[10]))


def test_policy_loss_clipping():
    """One logit decides: the ratios are set through old_logp, on both sides of both ends, for both signs of the advantage."""
    z = torch.tensor([[0.0, 0.0]] * 12, device="cuda")
    labels = torch.zeros(12, dtype=torch.int32, device="cuda")
    ratios = torch.tensor([0.5, 0.69, 0.71, 1.0, 1.09, 1.11, 0.5, 0.69, 0.71, 1.0, 1.09, 1.11], device="cuda")
    adv = torch.tensor([2.0] * 6 + [-2.0] * 6, device="cuda")
    old = math.log(0.5) - torch.log(ratios)
    loss, logp, grad = nm.netmax_policy_loss(z, labels, old, adv, clip_low=0.3, clip_high=0.1)
    kept = ratios.clamp(0.7, 1.1)
    assert torch.allclose(loss, -torch.minimum(ratios * adv, kept * adv), rtol=1e-5)
    active = torch.tensor([1, 1, 1, 1, 1, 0, 0, 0, 1, 1, 1, 1], device="cuda")
    assert torch.allclose(grad[:, 0], -0.5 * ratios * adv * active, rtol=1e-5) and torch.allclose(grad[:, 1], -grad[:, 0])


def test_policy_gradient_against_differences():
    g = gen(9)
    t, v = 4, 50
    z, labels = logits_and_labels(g, t, v, F32, 1.0)
    lp, _ = logp64(z, labels)
    old, ref, adv = (lp + 0.05).float(), (lp - 0.3).float(), normal(g, t)
    args = dict(ref_logp=ref, kl=0.2)
    _, _, grad = nm.netmax_policy_loss(z, labels, old, adv, **args)
    d, h = normal(g, t, v), 1e-3
    ends = [float(nm.netmax_policy_loss(z + s * d, labels, old, adv, **args)[0].double().sum()) for s in (h, -h)]
    # rounding: a few 2^-24 of losses of order one over 2 h
    assert (ends[0] - ends[1]) / (2 * h) == pytest.approx(float((grad.double() * d.double()).sum()), abs=2e-3)


def preference64(lp, ref, w, offsets, beta, e, scale):
    beta, e, scale = (float(torch.tensor(v, dtype=F32)) for v in (beta, e, scale))
    off = offsets.tolist()
    R = torch.stack([(w[a:b].double() * (lp[a:b] - ref[a:b].double())).sum() if b > a else torch.zeros((), dtype=torch.float64, device="cuda") for a, b in zip(off[:-1], off[1:])])
    h = beta * (R[0::2] - R[1::2])
    ls = torch.nn.functional.logsigmoid
    loss = scale * (-(1 - e) * ls(h) - e * ls(-h))
    dh = scale * beta * (torch.sigmoid(h) - (1 - e))
    slope = torch.zeros_like(lp)
    for q, (a, b) in enumerate(zip(off[:-1], off[1:])):
        slope[a:b] = w[a:b].double() * (dh[q // 2] if q % 2 == 0 else -dh[q // 2])
    return loss, R, slope


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lengths,vocab", [([1, 1], 5), ([0, 3], 17), ([0, 0, 4, 1], 1000), ([30, 0, 1, 12, 7, 7], 5001), ([100, 200, 300, 50], 257), ([6, 9], 40000), ([5, 4, 3, 8], 131072), ([2, 1], 262150)])
def test_preference_loss_sizes(lengths, vocab, dtype):
    g = gen(sum(lengths) + vocab)
    offsets = torch.tensor([2] + [2 + sum(lengths[:k + 1]) for k in range(len(lengths))], dtype=torch.int32, device="cuda")
    t = int(offsets[-1]) + 3                           # two tokens before and three behind all sequences
    z, labels = logits_and_labels(g, t, vocab, dtype)
    lp, q = logp64(z, labels)
    ref, w = (lp + normal(g, t, scale=0.3)).float(), (torch.rand(t, generator=g, device="cuda") < 0.8).float() * (0.5 + torch.rand(t, generator=g, device="cuda"))
    for e, scale in ((0.0, None), (0.1, 0.7)):
        loss, ratio, grad = nm.netmax_preference_loss(z, labels, offsets, w, ref, beta=0.3, smoothing=e, scale=scale)
        want, R, slope = preference64(lp, ref, w, offsets, 0.3, e, scale or 2.0 / len(lengths))
        terms = torch.stack([(w[a:b].double() * (lp[a:b].abs() + 1)).sum() for a, b in zip(offsets[:-1].tolist(), offsets[1:].tolist())])
        within(ratio, R, 2.0 ** -20 * terms + 2.0 ** -23 * R.abs(), "ratio")
        both = (terms[0::2] + terms[1::2]) * 2.0 ** -20
        within(loss, want, (scale or 1) * both + 2.0 ** -22 * want.abs(), "loss")
        terms = torch.zeros(t, dtype=torch.float64, device="cuda")      # sigma' <= 1/4: an error of h reaches the slopes as beta scale / 4 of it
        for k in range(len(lengths)):
            terms[int(offsets[k]):int(offsets[k + 1])] = (scale or 2.0 / len(lengths)) * 0.3 * 0.3 * (both[k // 2] * 2.0 ** 20 + 1)
        check_grad(grad, q, labels, slope, dtype, w.double() * terms)
        assert bool((grad[:2] == 0).all()) and bool((grad[-3:] == 0).all()) and bool((grad[w == 0] == 0).all())
        assert torch.equal(nm.netmax_preference_loss(z, labels, offsets, w, ref, beta=0.3, smoothing=e, scale=scale, need_grad=False)[0], loss)
    z[w == 0] = float("nan")                           # rows without weight are not looked at
    loss2, ratio2, grad2 = nm.netmax_preference_loss(z, labels, offsets, w, ref, beta=0.3, smoothing=0.1, scale=0.7, grad=z)
    assert torch.equal(loss2, loss) and torch.equal(ratio2, ratio) and torch.equal(grad2, grad)


def test_preference_loss_far_out():
    """Ratios that decide everything: the loss grows linearly, nothing overflows."""
    z = torch.tensor([[50.0, 0.0], [0.0, 50.0]] * 2, device="cuda")
    labels = torch.tensor([0, 0, 1, 1], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 1, 2, 3, 4], dtype=torch.int32, device="cuda")
    loss, ratio, grad = nm.netmax_preference_loss(z, labels, offsets, None, torch.zeros(4, device="cuda"), beta=100.0, scale=1.0)
    assert torch.equal(loss, torch.tensor([0.0, 5000.0], device="cuda"))
    assert torch.allclose(ratio, torch.tensor([0.0, -50.0, -50.0, 0.0], device="cuda"))
    assert bool(torch.isfinite(grad).all()) and float(grad[2, 1]) == pytest.approx(-100.0) and float(grad[2, 0]) == pytest.approx(100.0)


def test_losses_of_nothing():
    z, labels, f = torch.empty(0, 10, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    loss, logp, grad = nm.netmax_policy_loss(z, labels, f, f)
    assert loss.shape == (0,) and grad.shape == (0, 10)
    loss, ratio, grad = nm.netmax_preference_loss(z, labels, torch.zeros(3, dtype=torch.int32, device="cuda"), None, f)
    assert float(loss[0]) == pytest.approx(math.log(2)) and bool((ratio == 0).all()) and grad.shape == (0, 10)


# ---- far apart in memory -----------------------------------------------------------------------------------------------

def test_offsets_past_32_bits():
    """More than 2^32 bytes and 2^31 values in one operand: the last rows are as those of a call of their own."""
    g = gen(13)
    z = torch.randn(17000, 131072, generator=g, device="cuda", dtype=BF16)
    labels = torch.randint(0, 131072, (17000,), generator=g, device="cuda", dtype=torch.int32)
    old, adv, w = torch.full((17000,), -12.0, device="cuda"), torch.ones(17000, device="cuda"), torch.ones(17000, device="cuda")
    w[:-3] = 0.0
    last = nm.netmax_policy_loss(z[-3:].clone(), labels[-3:].clone(), old[-3:].clone(), adv[-3:].clone(), w[-3:].clone())
    loss, logp, grad = nm.netmax_policy_loss(z, labels, old, adv, w, grad=z)
    assert torch.equal(loss[-3:], last[0]) and torch.equal(logp[-3:], last[1]) and torch.equal(grad[-3:], last[2]) and not bool(grad[0].any())
    del z, grad
    x, wt = torch.randn(600_000, 4104, generator=g, device="cuda", dtype=BF16), normal(g, 4104, 72, dtype=BF16)
    y = nm.netmax_linear(x, wt)
    within(y[-300:], x[-300:].double() @ wt.double(), 4108 * 2.0 ** -24 * (x[-300:].double().abs() @ wt.double().abs()) + 2.0 ** -8 * y[-300:].double().abs() * 1.01, "y")
    dy = torch.zeros(600_000, 72, device="cuda", dtype=BF16)
    dy[-200:] = normal(g, 200, 72, dtype=BF16)
    dx, dw, db = nm.netmax_linear_grad(dy, x, wt)
    a, b = x[-200:].double(), dy[-200:].double()
    within(dw, a.t() @ b, 204 * 2.0 ** -24 * (a.abs().t() @ b.abs()) + 2.0 ** -8 * (a.t() @ b).abs(), "dw")
    within(dx[-200:], b @ wt.double().t(), 76 * 2.0 ** -24 * (b.abs() @ wt.double().abs().t()) + 2.0 ** -8 * (b @ wt.double().t()).abs(), "dx")
    assert not bool(dx[:-200].any())
    del x, y, dx
    m = torch.randn(520, 2056, 2056, generator=g, device="cuda", dtype=BF16)
    alone = nm.netmax_orthogonalize(m[-2:].clone())
    assert off(nm.netmax_orthogonalize(m, out=m)[-2:], alone.double()) < ORTH_TOL[BF16]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_many_tokens(dtype):
    """More rows than a launch has threads along one dimension for: parts of them give what calls of their own give."""
    g, n = gen(19), 16_800_002
    z, labels = normal(g, n, 3, dtype=dtype), torch.randint(0, 3, (n,), generator=g, device="cuda", dtype=torch.int32)
    old, adv, w = normal(g, n) - 1.0, normal(g, n), torch.ones(n, device="cuda")
    got = nm.netmax_policy_loss(z, labels, old, adv, w)
    parts = [slice(0, 1000), slice((1 << 21) - 500, (1 << 21) + 500), slice(n - 1000, n)]
    for p in parts:
        for a, b in zip(got, nm.netmax_policy_loss(*(v[p].clone() for v in (z, labels, old, adv, w)))):
            assert torch.equal(a[p], b)
    loss, ratio, grad = nm.netmax_preference_loss(z, labels, torch.arange(n + 1, device="cuda", dtype=torch.int32), w, old, scale=1.0)
    for p in parts:
        alone = nm.netmax_preference_loss(z[p].clone(), labels[p].clone(), torch.arange(1001, device="cuda", dtype=torch.int32), w[p].clone(), old[p].clone(), scale=1.0)
        assert torch.equal(loss[p.start // 2:p.stop // 2], alone[0]) and torch.equal(ratio[p], alone[1]) and torch.equal(grad[p], alone[2])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
def test_the_same_bits_every_time(dtype):
    g = gen(14)
    x, w, b, dy = normal(g, 5000, 300, dtype=dtype), normal(g, 300, 130, dtype=dtype), normal(g, 130, dtype=dtype), normal(g, 5000, 130, dtype=dtype)
    a = gradient_like(g, 3, 500, 333, dtype)
    z, labels = logits_and_labels(g, 600, 3001, dtype)
    offsets, ref = torch.tensor([0, 250, 600], dtype=torch.int32, device="cuda"), torch.full((600,), -8.0, device="cuda")

    def work():
        y, pre = nm.netmax_linear(x, w, b, act="gelu", keep_preact=True)
        return [y, *nm.netmax_linear_grad(dy, x, w, pre, act="gelu"), nm.netmax_orthogonalize(a), *nm.netmax_policy_loss(z, labels, ref, ref, ref_logp=ref, kl=0.1),
                *nm.netmax_preference_loss(z, labels, offsets, None, ref)]

    first = work()
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(first, work()))


# ---- streams and refusals --------------------------------------------------------------------------------------------

def test_operators_on_another_stream():
    g = gen(10)
    x, w, a = normal(g, 300, 264, dtype=BF16), normal(g, 264, 520, dtype=BF16), gradient_like(g, 2, 130, 200, F32)
    want = nm.netmax_linear(x, w, act="gelu"), nm.netmax_orthogonalize(a)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = nm.netmax_linear(x, w, act="gelu"), nm.netmax_orthogonalize(a)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_operators_in_a_graph():
    """Captured once, replayed on new inputs with other work between."""
    g = gen(11)
    x, w, b, dy = normal(g, 200, 136, dtype=BF16), normal(g, 136, 264, dtype=BF16), normal(g, 264, dtype=BF16), normal(g, 200, 264, dtype=BF16)
    a, m = gradient_like(g, 2, 70, 100, F32), torch.zeros(2, 70, 100, device="cuda")
    z, labels = logits_and_labels(g, 20, 1000, BF16)
    old, ref = torch.full((20,), -7.0, device="cuda"), torch.full((20,), -6.0, device="cuda")
    offsets = torch.tensor([0, 9, 20], dtype=torch.int32, device="cuda")

    def work():
        y, pre = nm.netmax_linear(x, w, b, act="silu", keep_preact=True)
        return [y, *nm.netmax_linear_grad(dy, x, w, pre, act="silu"), nm.netmax_orthogonalize(a, m, m_out=torch.empty_like(m)),
                *nm.netmax_policy_loss(z, labels, old, ref, ref_logp=ref, kl=0.1), *nm.netmax_preference_loss(z, labels, offsets, None, ref)]

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for k in range(4):
        for t in (x, dy, a, z):
            t.copy_(normal(g, *t.shape, dtype=t.dtype))
        graph.replay()
        torch.cuda.synchronize()
        for h, e in zip(held, work()):
            assert torch.equal(h, e), k
        torch.cuda.synchronize()


def test_refusals():
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, 6, device="cuda")
    f, labels = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    bad = [
        lambda: nm.netmax_linear(x.cpu(), w), lambda: nm.netmax_linear(x, w.cpu()), lambda: nm.netmax_linear(x.half(), w.half()),
        lambda: nm.netmax_linear(x, w.bfloat16()), lambda: nm.netmax_linear(x, w.t()), lambda: nm.netmax_linear(x, w[:7]),
        lambda: nm.netmax_linear(x, torch.ones(6, 8, device="cuda").t()), lambda: nm.netmax_linear(x, w, act="tanh"),
        lambda: nm.netmax_linear(x, w, torch.ones(5, device="cuda")), lambda: nm.netmax_linear(x, w, None, torch.ones(4, 5, device="cuda")),
        lambda: nm.netmax_linear(x[None], w), lambda: nm.netmax_linear(x[:, :0], w[:0]),
        lambda: nm.netmax_linear(x, w, y=torch.empty(6, device="cuda").expand(4, 6)),
        lambda: nm.netmax_linear_grad(torch.ones(4, 6, device="cuda"), x, w, act="gelu"),
        lambda: nm.netmax_linear_grad(torch.ones(4, 5, device="cuda"), x, w),
        lambda: nm.netmax_orthogonalize(x, f), lambda: nm.netmax_orthogonalize(x, x.bfloat16()), lambda: nm.netmax_orthogonalize(x, steps=0),
        lambda: nm.netmax_orthogonalize(x, eps=0.0), lambda: nm.netmax_orthogonalize(x, m_out=x), lambda: nm.netmax_orthogonalize(x[:0]),
        lambda: nm.netmax_policy_loss(x, labels.long(), f, f), lambda: nm.netmax_policy_loss(x, labels, f[:3], f), lambda: nm.netmax_policy_loss(x, labels, f, f, kl=0.1),
        lambda: nm.netmax_policy_loss(x, labels, f, f, clip_low=1.5), lambda: nm.netmax_policy_loss(x, labels, f, f, clip_high=-0.1),
        lambda: nm.netmax_policy_loss(x.half(), labels, f, f), lambda: nm.netmax_policy_loss(x[:, :0], labels, f, f),
        lambda: nm.netmax_preference_loss(x, labels, offsets[:2], None, f), lambda: nm.netmax_preference_loss(x, labels, offsets.long(), None, f),
        lambda: nm.netmax_preference_loss(x, labels, offsets, None, None), lambda: nm.netmax_preference_loss(x, labels, offsets, None, f, smoothing=2.0),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(nm.NetmaxError) as e:
            call()
        assert e.value.code == nm.NETMAX_EINVAL and str(e.value).split(": ", 1)[1], k
    nm.netmax_linear(x, w)
    torch.cuda.synchronize()
