"""Operators of a training step on a language model that lie around its layers, as cases that can be timed and whose results can be compared.

Kinds of cases
    embed   rows of an embedding table, scaled, for given tokens: the lookup alone, from one token to many, or with the gradient of the table.  Several
            workers' own tables go as one batch; tokens outside of the vocabulary are padding and have rows of zeros and no gradient.
    norm    the norms before and after a block, with its gate and the residual stream: u = N(f) gain + bias, h = a x + b gate u, y = N(h) gain + bias, for a
            block's output f and the residual stream x, or y = N(x) gain + bias alone; forward, or with all gradients.  N divides by the root of the mean
            square ("rms") or subtracts the mean first ("layer").
    clip    the norm of all gradients of a model, or of every worker's model, and the gradients scaled down to a largest norm.

Ranges: 1 .. 32768 tokens, vocabularies of 64 .. 131072, widths of 64 .. 8192 for tables; 1 .. 262144 rows of 32 .. 16384 values for norms; 1 .. 400 tensors
of 16 .. 4 x 4096 squared values for clipping; 1 .. 16 workers; float32 and bfloat16; sizes that are multiples of nothing, rows that lie further apart than they are long.
"""
import math

import numpy as np
import torch

own = False                                  # False: elementary torch operations in 32 bits; True: the library's operators

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
EPS = 1e-6
GRAD = 1e-3                                  # size of a gradient's entries


def _embed(name, tokens, vocab, width, dtype, train, batch=1, masked=0.0, pad=0):
    return {"name": name, "kind": "embed", "batch": batch, "tokens": tokens, "vocab": vocab, "width": width, "dtype": dtype, "train": train, "masked": masked, "pad": pad}


def _norm(name, rows, width, dtype, norm, gate, train, batch=1, block=True, bias=False, act="none", pad=0):
    return {"name": name, "kind": "norm", "batch": batch, "rows": rows, "width": width, "dtype": dtype, "norm": norm, "block": block, "gate": gate if block else "none",
            "act": act if block and gate != "none" else "none", "bias": bias, "train": train, "pad": pad}


def _clip(name, tensors, width, dtype, batch=1, share=0.5, pad=0):
    return {"name": name, "kind": "clip", "batch": batch, "tensors": tensors, "width": width, "dtype": dtype, "share": share, "pad": pad}


def listed():
    return [
        # the token that was sampled last, looked up for the next step: latency counts
        _embed("embed_token_bf16", 1, 131072, 4096, "bf16", False),
        # a step of eight workers with small models of their own, as in the training of small language models on preferences
        _embed("embed_workers_f32", 384, 512, 128, "f32", True, batch=8),
        # a padded batch, sizes that are multiples of nothing
        _embed("embed_odd_bf16", 1111, 5003, 777, "bf16", True, masked=0.1, pad=5),
        # a training batch of a large vocabulary
        _embed("embed_train_bf16", 32768, 131072, 4096, "bf16", True),
        # one token on its way between two blocks of a wide model, with a gate of its own
        _norm("norm_token_bf16", 1, 4096, "bf16", "rms", "rows", False, act="sigmoid"),
        # the norm of every head's query: many short rows, no residual stream
        _norm("norm_heads_bf16", 131072, 128, "bf16", "rms", "none", True, block=False),
        # eight workers' small models, every one with gains, biases and gates of its own
        _norm("norm_workers_f32", 384, 128, "f32", "layer", "channel", True, batch=8, bias=True),
        # sizes that are multiples of nothing, rows further apart than they are long
        _norm("norm_odd_f32", 1111, 777, "f32", "layer", "rows", True, bias=True, act="tanh", pad=3),
        # a training batch of a wide model
        _norm("norm_train_bf16", 16384, 8192, "bf16", "rms", "channel", True),
        # the gradients of those eight workers, views of their rows of parameters, a norm for each
        _clip("clip_workers_f32", 6, 128, "f32", batch=8),
        # matrices in bfloat16 and gains in float of odd sizes
        _clip("clip_odd_mixed", 37, 333, "mixed", pad=3),
        # a model of 24 layers
        _clip("clip_model_bf16", 96, 2048, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of the widths are multiples of 64, as most models' are; the others are any number."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.5 or n < 64 else n // 64 * 64


def draw(rng):
    most = {}                                        # no drawn case moves more than the largest listed one of its kind
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), work(c)["bytes"])
    while True:
        c = _drawn(rng)
        del c["name"]
        if work(c)["bytes"] <= most[c["kind"]]:
            return c


def _drawn(rng):
    kind, dtype = rng.choice(["embed", "norm", "norm", "clip"]), rng.choice(["f32", "bf16"])
    batch, pad = rng.choice([1, 1, 1, rng.randint(2, 16)]), rng.choice([0, 0, 0, rng.randint(1, 64)])
    if kind == "embed":
        return _embed("", _log(rng, 1, 32768 // batch), _log(rng, 64, 131072 // batch), _width(rng, 64, 8192), dtype, rng.random() < 0.7, batch,
                      rng.choice([0.0, 0.1, 0.5]), pad)
    if kind == "norm":
        return _norm("", _log(rng, 1, 262144 // batch), _width(rng, 32, 16384), dtype, rng.choice(["rms", "layer"]), rng.choice(["none", "channel", "rows"]),
                     rng.random() < 0.7, batch, rng.random() < 0.75, rng.random() < 0.5, rng.choice(["none", "sigmoid", "tanh"]), pad)
    return _clip("", _log(rng, 1, 400), _width(rng, 16, 4096), rng.choice(["f32", "bf16", "mixed"]), batch, rng.choice([0.01, 0.5, 2.0]), pad if batch == 1 else 0)


# ---- sizes ---------------------------------------------------------------------------------------------------------

def _frequencies(vocab):
    """How often each token is met: text has few frequent tokens and many rare ones."""
    p = 1.0 / (np.arange(vocab) + 3.0)
    return p / p.sum()


def _shapes(case):
    """The tensors of a model, layer by layer."""
    d = case["width"]
    return [((d, d), (d, 4 * d), (4 * d, d), (d,))[k % 4] for k in range(case["tensors"])]


def _type(case, shape):
    return case["dtype"] if case["dtype"] != "mixed" else "f32" if len(shape) == 1 else "bf16"


def work(case):
    b = case["batch"]
    if case["kind"] == "embed":
        t, v, w, es = case["tokens"], case["vocab"], case["width"], SIZE[case["dtype"]]
        met = t * (1.0 - case["masked"])
        rows = float((-np.expm1(met * np.log1p(-_frequencies(v)))).sum()) + t         # of the table, each once; out
        rows += met + v if case["train"] else 0                                       # gradient in; the table's out
        return {"bytes": b * (rows * w * es + 4.0 * t), "flops": b * met * w * (2.0 if case["train"] else 1.0)}
    if case["kind"] == "norm":
        n, es = float(b * case["rows"] * case["width"]), SIZE[case["dtype"]]
        full = case["gate"] == "rows"
        values = 4 + full if case["block"] else 2                                     # x, f, gate; h, y
        if case["train"]:                                                             # dy, dh; dx, df, dgate
            values += 4 + full if case["block"] else 2
        return {"bytes": values * n * es, "flops": n * (15.0 if case["block"] else 5.0) * (3.0 if case["train"] else 1.0)}
    total = [math.prod(s) * SIZE[_type(case, s)] for s in _shapes(case)]
    return {"bytes": 2.0 * b * sum(total), "flops": 3.0 * b * sum(math.prod(s) for s in _shapes(case))}


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _normal(g, *shape, dtype=torch.float32, scale=1.0, mean=0.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(scale).add_(mean).to(dtype)


def prepare(case, seed):
    return {"embed": _prepare_embed, "norm": _prepare_norm, "clip": _prepare_clip}[case["kind"]](case, _generator(seed))


def _lead(case):
    return (case["batch"],) if case["batch"] > 1 else ()


def _prepare_embed(case, g):
    dt, lead, t, v, w = DTYPES[case["dtype"]], _lead(case), case["tokens"], case["vocab"], case["width"]
    table = torch.randn(*lead, v, w + case["pad"], generator=g, device="cuda", dtype=dt)[..., :w]
    sums = torch.from_numpy(np.cumsum(_frequencies(v))).cuda()
    places = torch.randperm(v, generator=g, device="cuda")                            # frequent tokens lie anywhere in the table
    found = torch.searchsorted(sums, torch.rand(*lead, t, generator=g, device="cuda", dtype=torch.float64)).clamp_(max=v - 1)
    tokens = places[found]
    if case["masked"]:
        tokens = torch.where(torch.rand(*lead, t, generator=g, device="cuda") < case["masked"], -1, tokens)
    s = {"case": case, "table": table, "tokens": tokens.to(torch.int32), "scale": w ** 0.5}
    if case["train"]:
        s["dy"] = _normal(g, *lead, t, w + case["pad"], dtype=dt, scale=GRAD)[..., :w]
    return s


def _prepare_norm(case, g):
    dt, lead, n, w = DTYPES[case["dtype"]], _lead(case), case["rows"], case["width"]

    def rows(scale, dtype=dt):                       # rows that lie `pad` values further apart than they are long
        return torch.randn(*lead, n, w + case["pad"], generator=g, device="cuda", dtype=dtype).mul_(scale)[..., :w]

    s = {"case": case, "x": rows(2.0)}
    loud = torch.randint(0, w, (max(1, w // 200),), generator=g, device="cuda")       # a residual stream has a few channels that are much larger
    s["x"][..., loud] *= 20.0
    s["pre_gain"] = _normal(g, *lead, w, dtype=dt, scale=0.1, mean=1.0)
    s["pre_bias"] = _normal(g, *lead, w, dtype=dt, scale=0.1) if case["bias"] else None
    s["f"] = s["gate"] = s["post_gain"] = s["post_bias"] = s["dh"] = None
    if case["block"]:
        s["f"] = rows(0.5)
        s["post_gain"] = _normal(g, *lead, w, dtype=dt, scale=0.1, mean=1.0)
        s["post_bias"] = _normal(g, *lead, w, dtype=dt, scale=0.1) if case["bias"] else None
        if case["gate"] != "none":
            s["gate"] = rows(1.0) if case["gate"] == "rows" else _normal(g, *lead, w, dtype=dt, scale=0.2, mean=0.5)
    if case["train"]:
        s["dy"] = rows(GRAD)
        s["dh"] = rows(GRAD) if case["block"] else None
    s["scales"] = (0.9, 1.1) if case["block"] else (1.0, 1.0)
    return s


def _slices(case):
    """The model's tensors as slices of rows [batch, all values of a type], as they lie in a worker's row of parameters."""
    lead, shapes = _lead(case), _shapes(case)
    sizes = {d: sum(math.prod(s) for s in shapes if _type(case, s) == d) for d in DTYPES}
    rows = [torch.zeros(*lead, n, device="cuda", dtype=DTYPES[d]) for d, n in sizes.items() if n]
    at, cut = {t.dtype: 0 for t in rows}, []
    for s in shapes:
        row = next(t for t in rows if t.dtype == DTYPES[_type(case, s)])
        n = math.prod(s)
        cut.append(row[..., at[row.dtype]:at[row.dtype] + n].view(*lead, *s))
        at[row.dtype] += n
    return rows, cut


def _prepare_clip(case, g):
    shapes = _shapes(case)
    if case["pad"]:                                  # each by itself, rows further apart than they are long
        grads = [torch.zeros(*s[:-1], s[-1] + case["pad"], device="cuda", dtype=DTYPES[_type(case, s)])[..., :s[-1]] for s in shapes]
    else:
        grads = _slices(case)[1]
    rows, out = _slices(case)
    for k, t in enumerate(grads):                    # layers' gradients differ in size
        t.copy_(torch.randn(t.shape, generator=g, device="cuda", dtype=t.dtype).mul_(GRAD * (1.0 + k % 5)))
    size = math.sqrt(sum(math.prod(s) * (GRAD * (1.0 + k % 5)) ** 2 for k, s in enumerate(shapes)))
    s = {"case": case, "grads": grads, "out": out, "rows": rows, "max_norm": case["share"] * size}
    if own:                                          # a training program's gradients lie in the same memory in every step
        import paper_2009_05766_amd as nm
        s["laid_out"] = nm.Gradients(grads, out=out, batch=case["batch"] > 1)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"embed": _own_embed, "norm": _own_norm, "clip": _own_clip}[kind](state)
    return {"embed": _plain_embed, "norm": _plain_norm, "clip": _plain_clip}[kind](state)


def _own_embed(s):
    import paper_2009_05766_amd as nm
    y = nm.netmax_embed(s["tokens"], s["table"], scale=s["scale"])
    if not s["case"]["train"]:
        return y
    return [y, nm.netmax_embed_grad(s["dy"], s["tokens"], s["case"]["vocab"], scale=s["scale"])]


def _own_norm(s):
    import paper_2009_05766_amd as nm
    c, (a, b) = s["case"], s["scales"]
    form = dict(norm=c["norm"], gate_act=c["act"], x_scale=a, f_scale=b, eps=EPS)
    h, y = nm.netmax_block_norm(s["x"], s["f"], s["gate"], s["post_gain"], s["post_bias"], s["pre_gain"], s["pre_bias"], **form)
    out = [h, y] if c["block"] else [y]
    if c["train"]:
        grads = nm.netmax_block_norm_grad(s["dy"], s["dh"], s["x"], s["f"], s["gate"], s["post_gain"], s["post_bias"], s["pre_gain"], s["pre_bias"], **form)
        out += [t for t in grads if t is not None]
    return out


def _own_clip(s):
    import paper_2009_05766_amd as nm
    return [nm.netmax_clip_grads(s["laid_out"], s["max_norm"])] + s["rows"]


def _plain_embed(s):
    c, table, tokens = s["case"], s["table"], s["tokens"].long()
    dt, v, w = table.dtype, c["vocab"], c["width"]
    live = tokens >= 0
    at = tokens.clamp(min=0)
    if c["batch"] > 1:
        at = at + torch.arange(c["batch"], device="cuda")[:, None] * v
    flat = table.reshape(-1, w)
    y = torch.where(live[..., None], flat[at].float() * s["scale"], torch.zeros((), device="cuda")).to(dt)
    if not c["train"]:
        return y
    rows = torch.where(live[..., None], s["dy"].float(), torch.zeros((), device="cuda")).reshape(-1, w)
    grad = torch.zeros(c["batch"] * v, w, device="cuda").index_add_(0, at.reshape(-1), rows)
    return [y, (grad * s["scale"]).to(dt).view(table.shape)]


def _wide(t, like):
    """A vector of channels beside rows."""
    return t.float().unsqueeze(-2) if t.dim() < like.dim() else t.float()


def _unit(v, norm):
    """Rows without their mean (layer) and with a mean square of 1, and what they were multiplied by."""
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    r = 1.0 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _unit_grad(d, unit, r, norm):
    along = (d * unit).mean(-1, keepdim=True)
    if norm == "layer":
        d = d - d.mean(-1, keepdim=True)
    return r * (d - unit * along)


def _gate(t, act):
    """The gate's value and slope."""
    if act == "sigmoid":
        v = 1.0 / (1.0 + torch.exp(-t))
        return v, v * (1.0 - v)
    if act == "tanh":
        v = torch.tanh(t)
        return v, 1.0 - v * v
    return t, torch.ones_like(t)


def _plain_norm(s):
    c, x, dt, (a, b) = s["case"], s["x"].float(), s["x"].dtype, s["scales"]
    gate = slope = None
    h = x
    if c["block"]:
        f_unit, f_r = _unit(s["f"].float(), c["norm"])
        u = f_unit * _wide(s["post_gain"], x)
        if c["bias"]:
            u = u + _wide(s["post_bias"], x)
        v = b * u
        if s["gate"] is not None:
            gate, slope = _gate(_wide(s["gate"], x), c["act"])
            v = v * gate
        h = a * x + v
    h_unit, h_r = _unit(h, c["norm"])
    y = h_unit * _wide(s["pre_gain"], x)
    if c["bias"]:
        y = y + _wide(s["pre_bias"], x)
    out = [h.to(dt), y.to(dt)] if c["block"] else [y.to(dt)]
    if not c["train"]:
        return out
    dy = s["dy"].float()
    dh = _unit_grad(dy * _wide(s["pre_gain"], x), h_unit, h_r, c["norm"])
    pre = [(dy * h_unit).sum(-2).to(dt)] + ([dy.sum(-2).to(dt)] if c["bias"] else [])
    if not c["block"]:
        return out + [dh.to(dt)] + pre
    dh = dh + s["dh"].float()
    du = b * dh
    if gate is not None:
        dgate = du * u * slope
        if c["gate"] == "channel":
            dgate = dgate.sum(-2)
        du = du * gate
    df = _unit_grad(du * _wide(s["post_gain"], x), f_unit, f_r, c["norm"])
    post = [(du * f_unit).sum(-2).to(dt)] + ([du.sum(-2).to(dt)] if c["bias"] else [])
    return out + [(a * dh).to(dt), df.to(dt)] + ([dgate.to(dt)] if gate is not None else []) + post + pre


def _plain_clip(s):
    lead = tuple(range(1 if s["case"]["batch"] > 1 else 0))
    total = 0.0
    for g in s["grads"]:
        v = g.float()
        total = total + (v * v).sum(tuple(range(len(lead), g.dim())), dtype=torch.float64)
    norm = torch.sqrt(total).float()
    factor = torch.clamp(s["max_norm"] / norm, max=1.0)
    for g, to in zip(s["grads"], s["out"]):
        to.copy_(g.float() * factor.view(*factor.shape, *([1] * (g.dim() - factor.dim()))))
    return [norm] + s["rows"]


# ---- the same in 64 bits -------------------------------------------------------------------------------------------

def exact(case, seed):
    return {"embed": _exact_embed, "norm": _exact_norm, "clip": _exact_clip}[case["kind"]](prepare(case, seed))


def _exact_embed(s):
    c, tables, tokens = s["case"], s["table"], s["tokens"]
    if c["batch"] == 1:
        tables, tokens = tables[None], tokens[None]
    ys, grads = [], []
    for k in range(c["batch"]):
        kept = torch.nonzero(tokens[k] >= 0)[:, 0]
        which = tokens[k][kept].long()
        y = torch.zeros(c["tokens"], c["width"], device="cuda", dtype=torch.float64)
        y[kept] = tables[k][which].double() * s["scale"]
        ys.append(y)
        if c["train"]:
            dy = s["dy"] if c["batch"] == 1 else s["dy"][k]
            # token by token: the rows of each lie together once sorted
            order = torch.argsort(which, stable=True)
            seen, counts = torch.unique_consecutive(which[order], return_counts=True)
            grad = torch.zeros(c["vocab"], c["width"], device="cuda", dtype=torch.float64)
            if len(seen):
                grad[seen] = torch.segment_reduce(dy[kept[order]].double() * s["scale"], "sum", lengths=counts, axis=0)
            grads.append(grad)
    y = torch.stack(ys) if c["batch"] > 1 else ys[0]
    return [y, torch.stack(grads) if c["batch"] > 1 else grads[0]] if c["train"] else y


def _exact_norm(s):
    c, (a, b) = s["case"], s["scales"]
    names = [n for n in ("x", "f", "gate", "post_gain", "post_bias", "pre_gain", "pre_bias") if s[n] is not None]
    v = {n: s[n].double().requires_grad_(c["train"]) for n in names}
    wide = {n: t.unsqueeze(-2) if t.dim() < s["x"].dim() else t for n, t in v.items()}

    def normed(t, gain, bias):
        if c["norm"] == "layer":
            t = t - t.mean(-1, keepdim=True)
        t = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * wide[gain]
        return t + wide[bias] if bias in wide else t

    h = wide["x"]
    if c["block"]:
        u = normed(wide["f"], "post_gain", "post_bias")
        if "gate" in wide:
            u = u * {"none": lambda t: t, "sigmoid": torch.sigmoid, "tanh": torch.tanh}[c["act"]](wide["gate"])
        h = a * h + b * u
    y = normed(h, "pre_gain", "pre_bias")
    out = [h.detach(), y.detach()] if c["block"] else [y.detach()]
    if c["train"]:
        ends, into = ([y, h], [s["dy"].double(), s["dh"].double()]) if c["block"] else ([y], [s["dy"].double()])
        out += torch.autograd.grad(ends, [v[n] for n in names], into)
    return out


def _exact_clip(s):
    several = s["case"]["batch"] > 1
    by_worker = [g.double().reshape(s["case"]["batch"], -1) for g in s["grads"]]
    norm = torch.stack([torch.linalg.vector_norm(g, dim=1) for g in by_worker]).square().sum(0).sqrt()
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))
    rows = [torch.zeros(*t.shape, device="cuda", dtype=torch.float64) for t in s["rows"]]
    at = [0 for _ in rows]
    for g, t in zip(by_worker, s["grads"]):
        k = next(i for i, r in enumerate(s["rows"]) if r.dtype == t.dtype)
        rows[k].view(s["case"]["batch"], -1)[:, at[k]:at[k] + g.shape[1]] = g * scale[:, None]
        at[k] += g.shape[1]
    return [norm if several else norm[0]] + rows
