"""The operators for language models beside torch's automatic differentiation, which they do not record."""
import pytest
import torch

import paper_2009_05766_amd as nm

pytestmark = pytest.mark.gpu


def inputs():
    x, w = torch.ones(4, 8, device="cuda"), torch.ones(8, 6, device="cuda")
    f, labels = torch.zeros(4, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    return x, w, torch.ones(4, 6, device="cuda"), f, labels, torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")


def test_tensors_that_require_gradients():
    x, w, dy, f, labels, offsets = inputs()
    need = lambda t: t.clone().requires_grad_()  # noqa: E731
    calls = [
        lambda k: nm.netmax_linear(k(x), w), lambda k: nm.netmax_linear(x, k(w)), lambda k: nm.netmax_linear(x, w, k(dy[0])), lambda k: nm.netmax_linear(x, w, None, k(dy)),
        lambda k: nm.netmax_linear_grad(k(dy), x, w), lambda k: nm.netmax_linear_grad(dy, k(x), w), lambda k: nm.netmax_linear_grad(dy, x, k(w)),
        lambda k: nm.netmax_linear_grad(dy, x, w, k(dy), act="silu"), lambda k: nm.netmax_linear_grad(dy, x, w, dw=k(w)),
        lambda k: nm.netmax_orthogonalize(k(x)), lambda k: nm.netmax_orthogonalize(x, k(x)), lambda k: nm.netmax_orthogonalize(x, out=k(x)),
        lambda k: nm.netmax_policy_loss(k(x), labels, f, f), lambda k: nm.netmax_policy_loss(x, labels, k(f), f), lambda k: nm.netmax_policy_loss(x, labels, f, k(f)),
        lambda k: nm.netmax_policy_loss(x, labels, f, f, k(f)), lambda k: nm.netmax_policy_loss(x, labels, f, f, ref_logp=k(f), kl=0.1),
        lambda k: nm.netmax_preference_loss(k(x), labels, offsets, None, f), lambda k: nm.netmax_preference_loss(x, labels, offsets, k(f), f),
        lambda k: nm.netmax_preference_loss(x, labels, offsets, None, k(f)),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(nm.NetmaxError) as e:
            call(need)
        assert e.value.code == nm.NETMAX_EINVAL and "requires a gradient" in str(e.value), i
        with torch.no_grad():
            got = call(need)
        want = call(lambda t: t.clone())
        for a, b in zip(got if isinstance(got, tuple) else (got,), want if isinstance(want, tuple) else (want,)):
            assert torch.equal(a, b), i


def test_memory_that_a_call_writes_has_changed():
    """A graph that saved such a tensor says so instead of using other values."""
    x, w, dy, f, labels, offsets = inputs()
    outputs = {n: torch.empty(s, device="cuda") for n, s in (("y", (4, 6)), ("z", (4, 6)), ("dx", (4, 8)), ("dw", (8, 6)), ("db", (6,)), ("out", (4, 8)), ("m", (4, 8)), ("m_out", (4, 8)), ("grad", (4, 8)))}
    before = {n: t._version for n, t in outputs.items()}
    v = outputs["m"].zero_()._version
    nm.netmax_linear(x, w, y=outputs["y"], z=outputs["z"])
    nm.netmax_linear_grad(dy, x, w, dx=outputs["dx"], dw=outputs["dw"], db=outputs["db"])
    nm.netmax_orthogonalize(x, outputs["m"], out=outputs["out"])
    assert outputs["m"]._version > v
    v = outputs["m"]._version
    nm.netmax_orthogonalize(x, outputs["m"], m_out=outputs["m_out"])
    assert outputs["m"]._version == v
    nm.netmax_policy_loss(x, labels, f, f, grad=outputs["grad"])
    assert all(t._version > before[n] for n, t in outputs.items())
    v = outputs["grad"]._version
    nm.netmax_preference_loss(x, labels, offsets, None, f, grad=outputs["grad"])
    assert outputs["grad"]._version > v and x._version == 0 and w._version == 0 and dy._version == 0
    a = torch.ones(4, 8, device="cuda", requires_grad=True)
    saved = torch.ones(4, 8, device="cuda")
    product = (a * saved).sum()
    nm.netmax_orthogonalize(x, out=saved)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
