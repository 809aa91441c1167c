"""The operators that a worker's local step on a language model is made of, as cases that can be timed and whose results can be compared.

Kinds of cases
    linear      y = act(x w + b) + r: the forward pass alone, from one token to many, or a training pass with the gradients of x, w and b.
                Several workers' own weights go as one batch.
    orth        a momentum step whose update is orthogonalised by Newton-Schulz products, for a batch of workers' weight matrices.
    policy      the clipped policy loss with a KL term on the logits of sampled tokens, with the gradient of the logits.
    preference  the loss of paired log ratios on the logits of chosen and rejected sequences, with the gradient of the logits.

Ranges: 1 .. 16384 rows and widths 64 .. 8192 for linear layers; matrices of 32 .. 4096 rows and columns, 1 .. 64 workers; vocabularies
of 64 .. 131072, 1 .. 16384 tokens; float32 and bfloat16; sizes that are multiples of nothing, rows that lie further apart than they are long.
"""
import math

import torch

own = False                                  # False: elementary torch operations in 32 bits; True: the library's operators

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
STEPS, COEFFICIENTS = 5, (3.4445, -4.7750, 2.0315)   # Newton-Schulz products and the polynomial a s + b s^3 + c s^5 of each
CLIP = 0.2


def _linear(name, rows, d_in, d_out, dtype, act, train, batch=1, bias=True, residual=False, pad=0):
    return {"name": name, "kind": "linear", "batch": batch, "rows": rows, "in": d_in, "out": d_out, "dtype": dtype, "act": act,
            "train": train, "bias": bias, "residual": residual, "pad": pad}


def _orth(name, batch, rows, cols, dtype, mu=0.95, nesterov=True):
    return {"name": name, "kind": "orth", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "mu": mu, "nesterov": nesterov}


def _policy(name, tokens, vocab, dtype, kl):
    return {"name": name, "kind": "policy", "tokens": tokens, "vocab": vocab, "dtype": dtype, "kl": kl}


def _preference(name, pairs, tokens, vocab, dtype, smoothing=0.0):
    return {"name": name, "kind": "preference", "pairs": pairs, "tokens": tokens, "vocab": vocab, "dtype": dtype, "smoothing": smoothing}


def listed():
    return [
        # one token through a wide layer, as when answers are sampled for a policy loss: the weights are read once, latency counts
        _linear("linear_token_bf16", 1, 2048, 8192, "bf16", "silu", False),
        # 32 sequences that are sampled together, one token each, back onto the residual stream
        _linear("linear_tokens_bf16", 32, 4096, 4096, "bf16", "none", False, residual=True),
        # a layer of the small perceptron's sizes on 16 workers, each with its own weights, as in its training iterations
        _linear("linear_workers_f32", 64, 784, 512, "f32", "silu", True, batch=16),
        # a training pass whose sizes are multiples of nothing
        _linear("linear_odd_bf16", 1111, 777, 2049, "bf16", "gelu", True, residual=True),
        # a training pass over 8192 tokens of a wide layer
        _linear("linear_train_bf16", 8192, 4096, 8192, "bf16", "gelu", True),
        # the update of that perceptron's hidden weights on 16 workers
        _orth("orth_workers_f32", 16, 784, 512, "f32"),
        # a few matrices of odd sizes, plain momentum
        _orth("orth_odd_f32", 3, 1501, 700, "f32", nesterov=False),
        # large weights of eight workers, gradients in bfloat16
        _orth("orth_large_bf16", 8, 2048, 4096, "bf16"),
        # a short batch of sampled tokens of a small vocabulary
        _policy("policy_small_f32", 256, 5000, "f32", 0.05),
        # sampled tokens of a large vocabulary
        _policy("policy_large_bf16", 8192, 131072, "bf16", 0.05),
        # a few pairs of answers
        _preference("preference_few_bf16", 4, 1000, 32000, "bf16"),
        # a training batch of pairs
        _preference("preference_large_bf16", 16, 16384, 50000, "bf16", smoothing=0.1),
    ]


MOST_FLOPS = {"linear": 1.65e12, "orth": 2.4e12}     # no drawn case needs more than the largest listed one of its kind
MOST_LOGITS = {"policy": 8192 * 131072, "preference": 16384 * 50000}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 64, as most layers' are; the others are any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 else max(64, n // 64 * 64)


def draw(rng):
    while True:
        c = _drawn(rng)
        del c["name"]
        if c["kind"] in MOST_FLOPS and work(c)["flops"] <= MOST_FLOPS[c["kind"]]:
            return c
        if c["kind"] in MOST_LOGITS and c["tokens"] * c["vocab"] * SIZE[c["dtype"]] <= 2 * MOST_LOGITS[c["kind"]]:
            return c


def _drawn(rng):
    kind = rng.choice(["linear", "linear", "orth", "orth", "policy", "preference"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind == "linear":
        batch, train = rng.choice([1, 1, 1, rng.randint(2, 16)]), rng.random() < 0.6
        # ReLU's derivative jumps at 0: gradients in float32 are compared with activations that have none such
        act = rng.choice(["none", "gelu", "silu"] + (["relu"] if dtype == "bf16" or not train else []))
        return _linear("", _log(rng, 1, 16384 // batch), _width(rng, 64, 8192), _width(rng, 64, 8192), dtype, act, train, batch,
                       rng.random() < 0.7, rng.random() < 0.5, rng.choice([0, 0, 0, rng.randint(1, 64)]))
    if kind == "orth":
        return _orth("", _log(rng, 1, 64), rng.choice([_log(rng, 32, 4096), _width(rng, 64, 4096)]), _width(rng, 64, 4096), dtype,
                     rng.choice([0.9, 0.95]), rng.random() < 0.7)
    if kind == "policy":
        return _policy("", _log(rng, 1, 16384), _log(rng, 64, 131072), dtype, rng.choice([0.0, 0.02, 0.1]))
    pairs = _log(rng, 1, 64)
    return _preference("", pairs, _log(rng, 4 * pairs, 16384), _log(rng, 64, 131072), dtype, rng.choice([0.0, 0.1]))


# ---- sizes ---------------------------------------------------------------------------------------------------------

def work(case):
    es = SIZE[case["dtype"]]
    if case["kind"] == "linear":
        b, t, i, o = case["batch"], case["rows"], case["in"], case["out"]
        passes = 3 if case["train"] else 1
        values = t * i + i * o + t * o + (o if case["bias"] else 0) + (t * o if case["residual"] else 0)
        if case["train"]:                            # dy in; dx, dw, db out
            values += t * o + t * i + i * o + (o if case["bias"] else 0)
        return {"bytes": float(b * values * es), "flops": 2.0 * passes * b * t * i * o}
    if case["kind"] == "orth":
        # g in, update out, momentum in and out; of the symmetric products x x^T and (x x^T)^2 one triangle
        k, n = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        return {"bytes": float(case["batch"] * k * n * (2 * es + 8)), "flops": float(case["batch"]) * STEPS * (3.0 * k * k * n + float(k) ** 3)}
    # logits in, their gradient out; rows without weight are not read
    share = 0.9 if case["kind"] == "policy" else 0.75
    return {"bytes": (1 + share) * case["tokens"] * case["vocab"] * es, "flops": 6.0 * case["tokens"] * case["vocab"]}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).to(dtype)


def prepare(case, seed):
    g = _generator(seed)
    return {"linear": _prepare_linear, "orth": _prepare_orth, "policy": _prepare_policy, "preference": _prepare_preference}[case["kind"]](case, g)


def _prepare_linear(case, g):
    dt, pad = DTYPES[case["dtype"]], case["pad"]
    lead = (case["batch"],) if case["batch"] > 1 else ()
    t, i, o = case["rows"], case["in"], case["out"]

    def rows(width, scale=1.0):                      # rows that lie `pad` values further apart than they are long
        return _normal(g, *lead, t, width + pad, dtype=dt, scale=scale)[..., :width]

    s = {"case": case, "x": rows(i), "w": _normal(g, *lead, i, o, dtype=dt, scale=i ** -0.5),
         "bias": _normal(g, *lead, o, dtype=dt, scale=0.1) if case["bias"] else None,
         "residual": rows(o) if case["residual"] else None}
    if case["train"]:
        s["dy"] = rows(o, 1e-2)
    return s


def _prepare_orth(case, g):
    """A gradient has a few strong directions, those of its batch, under noise of comparable size."""
    b, m, n = case["batch"], case["rows"], case["cols"]
    r = max(2, min(m, n) // 8)

    def matrix(scale):
        strong = torch.matmul(_normal(g, b, m, r), _normal(g, b, r, n, scale=r ** -0.5))
        return strong.add_(_normal(g, b, m, n, scale=0.5)).mul_(scale)

    return {"case": case, "g": matrix(1e-3).to(DTYPES[case["dtype"]]), "m": matrix(5e-3), "m_out": torch.empty(b, m, n, device="cuda")}


def _logits(case, g):
    """Logits of a model that has learnt something: the sampled token is mostly among the likely ones."""
    t, v, dt = case["tokens"], case["vocab"], DTYPES[case["dtype"]]
    z = torch.randn(t, v, generator=g, device="cuda", dtype=dt).mul_(2.0)
    labels = torch.randint(0, v, (t,), generator=g, device="cuda", dtype=torch.int32)
    at = labels.long()[:, None]
    z.scatter_(1, at, (z.gather(1, at).float() + 4.0 + 3.0 * torch.rand(t, 1, generator=g, device="cuda")).to(dt))
    logp = torch.empty(t, device="cuda")
    for k in range(0, t, 256):
        part = z[k:k + 256].float()
        logp[k:k + 256] = part.gather(1, at[k:k + 256])[:, 0] - torch.logsumexp(part, 1)
    return z, labels, logp


def _prepare_policy(case, g):
    z, labels, logp = _logits(case, g)
    t = case["tokens"]
    # log ratios to the sampling policy on odd hundredths: clearly inside or outside of the clipping range, whose ends are at -0.223 and 0.182
    old = logp - (torch.round(_normal(g, t, scale=10.0)) * 0.02 + 0.01)
    live = (torch.rand(t, generator=g, device="cuda") < 0.9).float()       # padding has no weight
    live[0] = 1.0
    return {"case": case, "logits": z, "labels": labels, "old": old, "ref": logp + _normal(g, t, scale=0.2) if case["kl"] else None,
            "advantage": _normal(g, t), "weight": live / live.sum()}


def _prepare_preference(case, g):
    z, labels, logp = _logits(case, g)
    t, n = case["tokens"], 2 * case["pairs"]
    # ragged sequences that fill all rows; each begins with a prompt, a quarter of it, that has no weight
    share = torch.rand(n, generator=g, device="cuda").add_(0.5).double()
    offsets = torch.cat([torch.zeros(1, device="cuda", dtype=torch.int64), torch.round(torch.cumsum(share, 0) / share.sum() * t).long()])
    place = torch.arange(t, device="cuda")
    seq = torch.bucketize(place, offsets[1:], right=True)
    into = place - offsets[seq]
    weight = (into * 4 >= offsets[seq + 1] - offsets[seq]).float()
    ref = logp + _normal(g, t, scale=0.5)
    return {"case": case, "logits": z, "labels": labels, "offsets": offsets.to(torch.int32), "weight": weight, "seq": seq, "ref": ref, "beta": 0.1}


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return _OWN[kind](state)
    return _PLAIN[kind](state)


def _own_linear(s):
    import paper_2009_05766_amd as nm
    c = s["case"]
    if not c["train"]:
        return nm.netmax_linear(s["x"], s["w"], s["bias"], s["residual"], act=c["act"])
    y, z = nm.netmax_linear(s["x"], s["w"], s["bias"], s["residual"], act=c["act"], keep_preact=True)
    dx, dw, db = nm.netmax_linear_grad(s["dy"], s["x"], s["w"], z, act=c["act"], need_bias=c["bias"])
    return [y, dx, dw] + ([db] if c["bias"] else [])


def _own_orth(s):
    import paper_2009_05766_amd as nm
    c = s["case"]
    update = nm.netmax_orthogonalize(s["g"], s["m"], m_out=s["m_out"], mu=c["mu"], nesterov=c["nesterov"], steps=STEPS, coefficients=COEFFICIENTS)
    return [update, s["m_out"]]


def _own_policy(s):
    import paper_2009_05766_amd as nm
    return list(nm.netmax_policy_loss(s["logits"], s["labels"], s["old"], s["advantage"], s["weight"], ref_logp=s["ref"], clip_low=CLIP,
                                      clip_high=CLIP, kl=s["case"]["kl"]))


def _own_preference(s):
    import paper_2009_05766_amd as nm
    return list(nm.netmax_preference_loss(s["logits"], s["labels"], s["offsets"], s["weight"], s["ref"], beta=s["beta"], smoothing=s["case"]["smoothing"]))


_OWN = {"linear": _own_linear, "orth": _own_orth, "policy": _own_policy, "preference": _own_preference}


def _t(a):
    return a.transpose(-1, -2).contiguous()


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return e * (1.0 + z * (1.0 - e))
    return torch.ones_like(z)


def _plain_linear(s):
    c, dt = s["case"], s["x"].dtype
    x, w = s["x"].float(), s["w"].float()
    z = torch.matmul(x, w)
    if s["bias"] is not None:
        z = z + s["bias"].float().unsqueeze(-2)
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if not c["train"]:
        return y.to(dt)
    dz = s["dy"].float()
    if c["act"] != "none":
        dz = dz * _slope(z, c["act"])
    grads = [torch.matmul(dz, _t(w)).to(dt), torch.matmul(_t(x), dz).to(dt)]
    if c["bias"]:
        grads.append(dz.sum(-2).to(dt))
    return [y.to(dt)] + grads


def _plain_orth(s):
    c = s["case"]
    a, b, k = COEFFICIENTS
    g = s["g"].float()
    m = c["mu"] * s["m"] + g
    u = g + c["mu"] * m if c["nesterov"] else m
    x = u / torch.clamp(torch.sqrt((u * u).sum((-1, -2), keepdim=True)), min=1e-7)
    tall = c["rows"] > c["cols"]
    if tall:
        x = _t(x)
    for _ in range(STEPS):
        p = torch.matmul(x, _t(x))
        x = a * x + torch.matmul(b * p + k * torch.matmul(p, p), x)
    return [(_t(x) if tall else x).to(s["g"].dtype), m]


def _token_logp(z, labels):
    """Log probability of each row's label, and all probabilities."""
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    at = labels.long()[:, None]
    return (z.gather(1, at) - top - torch.log(total))[:, 0], e / total, at


def _logit_grad(p, at, slope):
    """slope * (onehot - p), in p's memory."""
    p.mul_(-slope[:, None])
    return p.scatter_add_(1, at, slope[:, None])


def _plain_policy(s):
    c, dt = s["case"], s["logits"].dtype
    logp, p, at = _token_logp(s["logits"].float(), s["labels"])
    ratio = torch.exp(logp - s["old"])
    a, w = s["advantage"], s["weight"]
    free, clipped = ratio * a, torch.clamp(ratio, 1.0 - CLIP, 1.0 + CLIP) * a
    loss = -torch.minimum(free, clipped)
    slope = torch.where(free <= clipped, -free, torch.zeros_like(free))
    if s["ref"] is not None:
        d = s["ref"] - logp
        loss = loss + c["kl"] * (torch.exp(d) - d - 1.0)
        slope = slope + c["kl"] * (1.0 - torch.exp(d))
    return [w * loss, logp * (w != 0), _logit_grad(p, at, w * slope).to(dt)]


def _plain_preference(s):
    c, dt = s["case"], s["logits"].dtype
    logp, p, at = _token_logp(s["logits"].float(), s["labels"])
    n = 2 * c["pairs"]
    member = (s["seq"][None, :] == torch.arange(n, device="cuda")[:, None]).float()
    total = (member * (s["weight"] * (logp - s["ref"]))[None, :]).sum(1)
    gap = total.view(-1, 2)
    h = s["beta"] * (gap[:, 0] - gap[:, 1])
    e = c["smoothing"]
    soft = lambda v: torch.clamp(v, min=0.0) + torch.log(1.0 + torch.exp(-torch.abs(v)))  # noqa: E731  log(1 + exp(v))
    loss = (1.0 - e) * soft(-h) + e * soft(h)
    dh = 1.0 / (1.0 + torch.exp(-h)) - (1.0 - e)
    by_seq = (s["beta"] / c["pairs"]) * torch.stack([dh, -dh], 1).view(-1)
    return [loss / c["pairs"], total, _logit_grad(p, at, by_seq[s["seq"]] * s["weight"]).to(dt)]


_PLAIN = {"linear": _plain_linear, "orth": _plain_orth, "policy": _plain_policy, "preference": _plain_preference}


# ---- the same in 64 bits -------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "orth": _exact_orth, "policy": _exact_policy, "preference": _exact_preference}[case["kind"]](s)


def _exact_linear(s):
    c = s["case"]
    x, w = s["x"].double().requires_grad_(), s["w"].double().requires_grad_()
    bias = s["bias"].double().requires_grad_() if c["bias"] else None
    z = x @ w if bias is None else x @ w + bias.unsqueeze(-2)
    act = {"none": lambda v: v, "relu": torch.nn.functional.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu}[c["act"]]
    y = act(z)
    if s["residual"] is not None:
        y = y + s["residual"].double()
    if not c["train"]:
        return y.detach()
    grads = torch.autograd.grad(y, [x, w] + ([bias] if c["bias"] else []), s["dy"].double())
    return [y.detach()] + list(grads)


def _exact_orth(s):
    c = s["case"]
    a, b, k = COEFFICIENTS
    out, ms = [], []
    for g, m in zip(s["g"].double(), s["m"].double()):
        m = c["mu"] * m + g
        u = g + c["mu"] * m if c["nesterov"] else m
        x = u / max(float(torch.linalg.matrix_norm(u)), 1e-7)
        if c["rows"] > c["cols"]:                    # odd polynomials: p(x^T) = p(x)^T, here from the other side
            for _ in range(STEPS):
                p = x.T @ x
                x = a * x + x @ (b * p + k * (p @ p))
        else:
            for _ in range(STEPS):
                p = x @ x.T
                x = a * x + (b * p + k * (p @ p)) @ x
        out.append(x)
        ms.append(m)
    return [torch.stack(out), torch.stack(ms)]


def _exact_rows(logits, labels, each):
    """each(log probabilities of some rows, the rows) -> their slope; gives the labels' log probabilities and the gradient."""
    t, v = logits.shape
    logp, grad = torch.empty(t, device="cuda", dtype=torch.float64), torch.empty(t, v, device="cuda", dtype=torch.float64)
    for k in range(0, t, 512):
        rows = slice(k, min(t, k + 512))
        q = torch.log_softmax(logits[rows].double(), 1)
        at = labels[rows].long()[:, None]
        logp[rows] = q.gather(1, at)[:, 0]
        if each is not None:
            slope = each(logp[rows], rows)[:, None]
            grad[rows] = -slope * q.exp_()
            grad[rows] += torch.zeros_like(q).scatter_(1, at, slope)
    return logp, grad


def _exact_policy(s):
    kl, w = s["case"]["kl"], s["weight"].double()

    def loss_of(logp, rows):
        r, a = torch.exp(logp - s["old"][rows].double()), s["advantage"][rows].double()
        loss = torch.maximum(-r * a, -r.clamp(1 - CLIP, 1 + CLIP) * a)
        if s["ref"] is not None:
            d = s["ref"][rows].double() - logp
            loss = loss + kl * (torch.expm1(d) - d)
        return w[rows] * loss

    def slope(logp, rows):
        q = logp.clone().requires_grad_()
        return torch.autograd.grad(loss_of(q, rows).sum(), q)[0]

    logp, grad = _exact_rows(s["logits"], s["labels"], slope)
    return [loss_of(logp, slice(None)), torch.where(w != 0, logp, torch.zeros_like(logp)), grad]


def _exact_preference(s):
    c, w = s["case"], s["weight"].double()
    logp, _ = _exact_rows(s["logits"], s["labels"], None)
    total = torch.zeros(2 * c["pairs"], device="cuda", dtype=torch.float64).index_add_(0, s["seq"], w * (logp - s["ref"].double())).requires_grad_()
    h = s["beta"] * (total[0::2] - total[1::2])
    e, sigma = c["smoothing"], torch.nn.functional.logsigmoid
    loss = -((1 - e) * sigma(h) + e * sigma(-h)) / c["pairs"]
    by_seq = torch.autograd.grad(loss.sum(), total)[0]
    _, grad = _exact_rows(s["logits"], s["labels"], lambda q, rows: by_seq[s["seq"][rows]] * w[rows])
    return [loss.detach(), total.detach(), grad]
