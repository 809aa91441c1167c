"""Values at which the operators around a language model's layers went wrong once: infinities that nothing norms, products beside the middle of two bfloat16 values, outputs made in inference
mode; sums of very many rows.  Tolerances as in test_gpu_lm_step_ops.py, where they are not bits."""
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


def nearest_bf16(v):
    """Doubles rounded to bfloat16 once, ties to even, by their bits (no value here is subnormal or past the range)."""
    bits = v.view(torch.int64)
    return ((bits + (1 << 44) - 1 + (bits >> 45 & 1)) & -(1 << 45)).view(torch.float64)


def test_clipping_rounds_bfloat16_once():
    """g max / norm in double, rounded once: not to float, which may end in the middle of two bfloat16 values, before.  The values' squares have 14 bits behind the point and their
    sum is exact, so that norm and factor are those of any order; 128 products for each of 40000 norms, one in 2^17 of which float would round to the wrong side."""
    g = ops.gen(3)
    t = (1.0 + torch.randint(0, 128, (40000, 512), generator=g, device="cuda") / 128.0).to(BF16)
    norm = (t.double() ** 2).sum(1).sqrt()
    want = nearest_bf16(t.double() * (float(torch.tensor(0.7, dtype=ops.F32)) / norm)[:, None])
    through_float = (t.double() * (float(torch.tensor(0.7, dtype=ops.F32)) / norm)[:, None]).float().to(BF16)
    assert int((through_float.double() != want).sum()) > 0          # such products are among them
    nm.netmax_clip_grads([t], 0.7, batch=True)
    assert torch.equal(t.double(), want)


def test_clipping_rounds_bfloat16_at_the_ends_of_the_range():
    """Subnormal results are rounded once, too, and what is past the range or no number stays what it is."""
    t = torch.tensor([3.0 * 2.0 ** -133, 2.0 ** -133, 5.0 * 2.0 ** -133, 3.3895e38, -3.3895e38], device="cuda", dtype=BF16)
    big = t.clone()
    assert float(nm.netmax_clip_grads([big], 2.0 ** 127)) > 2.0 ** 127
    factor = 2.0 ** 127 / float((t.double() ** 2).sum().sqrt())
    ops.within(big, t.double() * factor, 2.0 ** -8 * t.double().abs() + 2.0 ** -134, "scaled")
    whole = t.clone()
    nm.netmax_clip_grads([whole], float("inf"), out=[out := torch.zeros_like(t)])
    assert torch.equal(out, t)
    odd = torch.tensor([float("nan"), 1.0, float("inf"), -float("inf")], device="cuda", dtype=BF16)
    nm.netmax_clip_grads([odd[2:]], float("inf"), out=[out := torch.zeros(2, device="cuda", dtype=BF16)])
    assert out.tolist() == [float("inf"), -float("inf")]
    nm.netmax_clip_grads([odd[:2]], 1.0)
    assert bool(odd[:2].isnan().all())


def test_outputs_made_in_inference_mode():
    """They have no count of changes to raise; a call writes them as any other memory."""
    x, v, tokens = torch.ones(4, 8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with torch.inference_mode():
        rows = [torch.full((4, 8), 5.0, device="cuda") for _ in range(8)]
        vectors = [torch.full((8,), 5.0, device="cuda") for _ in range(4)]
        w = torch.ones(8, 8, device="cuda")
    assert nm.netmax_linear(x, w, y=rows[0]) is rows[0] and bool((rows[0] == 8).all())
    assert nm.netmax_embed(tokens, x, scale=2.0, y=rows[0]) is rows[0] and bool((rows[0] == 2).all())
    assert nm.netmax_embed_grad(x, tokens, dtable=rows[1]) is rows[1] and bool((rows[1][0] == 4).all()) and not bool(rows[1][1:].any())
    h, y = nm.netmax_block_norm(x, x, h=rows[2], y=rows[3], post=False)
    assert h is rows[2] and y is rows[3] and bool((h == 2).all()) and bool((y - 1 < 1e-6).all())
    got = nm.netmax_block_norm_grad(x, x, x, x, x, v, v, v, v, dx=rows[4], df=rows[5], dgate=rows[6], dpost_gain=vectors[0], dpost_bias=vectors[1], dpre_gain=vectors[2], dpre_bias=vectors[3])
    assert all(a is b for a, b in zip(got, rows[4:7] + vectors)) and not bool(got.dx.eq(5).any())
    # the root of 32 is no float: rounded once, by at most 2^-24 of itself; the largest norm here is 1/16 of that float, exactly, the factor 1/16 to 2^-24 and its product with 1 rounded once more
    norm = float(nm.netmax_clip_grads([x], float(torch.tensor(32.0).sqrt()) / 16, out=[rows[7]]))
    assert norm == pytest.approx(32 ** 0.5, rel=E) and bool(((rows[7] * 16 - 1).abs() <= 2.5 * E).all())
    with torch.inference_mode():
        nm.netmax_clip_grads([rows[7]], 1.0)


@ops.BOTH
@pytest.mark.parametrize("n", [2049, 33000, 600000])
def test_gradient_of_one_frequent_token(n, dtype):
    """A chunk's 32 rows take at most 31 roundings, a fourth of the chunks n / 128 and one, three more join the fourths and one scales; where a chunk begins or ends with others it is no more."""
    g = ops.gen(n)
    dy = ops.normal(g, n, 24, dtype=dtype, mean=1.0)
    tokens = torch.full((n,), 2, dtype=torch.int32, device="cuda")
    tokens[5::1000] = 1
    got = nm.netmax_embed_grad(dy, tokens, 4, scale=1.7)
    scale = float(torch.tensor(1.7, dtype=ops.F32))
    for v in (1, 2):
        rows = dy.double()[tokens == v] * scale
        want = rows.sum(0)
        ops.within(got[v], want, (n / 128 + 36) * E * rows.abs().sum(0) + ULP[dtype] * want.abs(), f"token {v}")
    assert not bool(got[[0, 3]].any())
