"""The operators around a language model's layers together, as the training of several workers' models uses them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D64 = torch.float64


def model64(p, tokens, norms):
    """Logits of one worker's model of demo_preferences in double."""
    unit = lambda v: v / torch.sqrt((v * v).mean(-1, keepdim=True) + float(torch.tensor(1e-6)))  # noqa: E731
    e = p["embed"][tokens]
    n = unit(e) * p["first_gain"] if norms else e
    z = n @ p["w1"] + p["b1"]
    f = (0.5 * z * (1 + torch.erf(z / math.sqrt(2)))) @ p["w2"] + p["b2"]
    h = e + p["gate"] * unit(f) * p["post_gain"] if norms else e + f
    return (unit(h) * p["pre_gain"] if norms else h) @ p["out"]


@pytest.mark.parametrize("norms", [False, True], ids=["plain", "norms"])
def test_gradients_of_a_model(norms):
    """Every parameter's gradient against automatic differentiation in double.  A float sum of up to 512 products is within 516 2^-24 = 3.1e-5 of its magnitudes' sum, which is up to sqrt 512 times the
    result where signs are random: 7e-4 for each of the seven products and norms that a gradient goes through, 5e-3 of its norm in all."""
    from paper_2009_05766_amd.demo_preferences import VOCAB, Workers
    w = Workers(3, seed=4, norms=norms)
    g = torch.Generator(device="cuda").manual_seed(1)
    w.params = w.params + 0.05 * torch.randn(w.params.shape, generator=g, device="cuda")        # workers that differ
    tokens = torch.randint(0, VOCAB, (3, 200), generator=g, device="cuda")
    tokens[:, :40] = 7
    logits, kept = w.forward(tokens)
    dlogits = torch.randn(logits.shape, generator=g, device="cuda")
    w.grads.fill_(float("nan"))
    w.backward(dlogits, kept)
    for k in range(3):
        p = {n: w.cut(w.params, n)[k].to(D64).requires_grad_() for n in w.places}
        want = model64(p, tokens[k], norms)
        assert float((logits[k].to(D64) - want.detach()).norm() / want.detach().norm()) < 5e-3
        for n, d in zip(p, torch.autograd.grad(want, list(p.values()), dlogits[k].to(D64))):
            got = w.cut(w.grads, n)[k].to(D64)
            assert float((got - d).norm() / d.norm()) < 5e-3, n
    w.run.close()


def test_clipped_gradients_of_workers():
    """Slices of the workers' rows: each worker's by its own norm, nothing else in the rows touched."""
    from paper_2009_05766_amd.demo_preferences import Workers
    import paper_2009_05766_amd as nm
    w = Workers(4, norms=True)
    g = torch.Generator(device="cuda").manual_seed(2)
    w.grads.copy_(torch.randn(w.grads.shape, generator=g, device="cuda") * torch.tensor([0.1, 1.0, 1e-4, 10.0], device="cuda")[:, None])
    before = w.grads.to(D64)
    size = before.norm(dim=1)
    norm = nm.netmax_clip_grads(w.clipped, 30.0)
    assert bool(((norm.to(D64) - size).abs() <= 2.0 ** -23 * size).all())
    want = before * torch.clamp(30.0 / size, max=1.0)[:, None]
    assert bool(((w.grads.to(D64) - want).abs() <= 2.0 ** -23 * want.abs()).all()) and torch.equal(w.grads[2].to(D64), before[2])
    w.run.close()


def test_run_with_norms_and_clipping():
    from paper_2009_05766_amd.demo_preferences import main
    seen, rewards = main(["--workers", "3", "--steps", "3", "--norms", "--clip", "1.0"])
    assert len(seen) == 3 and len(rewards) == 3 and all(math.isfinite(v) for s in seen for v in s) and all(math.isfinite(r) for r in rewards)
