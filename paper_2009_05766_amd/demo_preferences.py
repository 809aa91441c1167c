"""Decentralised training of small language models on preferences: every worker's local step is made of the library's operators, its update is mixed by NetMax.

Each of M workers holds a model of the next token (embedding, a residual block d -> f -> d with GELU, projection onto the vocabulary) and its own data.  First
the workers learn from pairs of sequences, one written by a hidden teacher and one at random (`netmax_preference_loss`); then they write sequences
themselves and are rewarded for the teacher's choices (`netmax_policy_loss`, with a KL term to the model that the second phase began with).  Embeddings and layers run as one batch over the
workers (`netmax_embed`, `netmax_linear` and their gradients), weight matrices are updated by orthogonalised momentum (`netmax_orthogonalize`), and
`netmax_mix` takes those updates as the gradient of a context without momentum.  With --norms the residual block has norms before and after it and a gate for each channel
(`netmax_block_norm`); with --clip every worker's gradients are scaled down to a largest norm (`netmax_clip_grads`).

    python -m paper_2009_05766_amd.demo_preferences [--workers 8] [--steps 60] [--norms] [--clip 1.0]
"""
from __future__ import annotations

import argparse

import numpy as np
import torch

import paper_2009_05766_amd as nm

VOCAB, WIDTH, HIDDEN = 512, 128, 320
PAIRS, LENGTH = 8, 24                                   # per worker: pairs of a batch, tokens of a sequence
LR, MU = 0.02, 0.9


MATRICES = ("embed", "w1", "w2", "out")
NORMS = ("first_gain", "post_gain", "gate", "pre_gain")                     # gains of the norms before, after and behind the block; the block's gate


def _layout(norms: bool):
    """Where each parameter lies in a worker's row: name -> (offset, shape)."""
    places, at = {}, 0
    for name, shape in (("embed", (VOCAB, WIDTH)), ("w1", (WIDTH, HIDDEN)), ("b1", (HIDDEN,)), ("w2", (HIDDEN, WIDTH)), ("b2", (WIDTH,)), ("out", (WIDTH, VOCAB)),
                        *((n, (WIDTH,)) for n in NORMS if norms)):
        places[name] = (at, shape)
        at += int(np.prod(shape))
    return places, at


class Workers:
    def __init__(self, M: int, seed: int = 0, norms: bool = False, clip: float = 0.0):
        self.M, self.norms, self.clip = M, norms, clip
        self.places, D = _layout(norms)
        self.D = D
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        x0 = torch.zeros(M, D, device="cuda")
        for name, scale in (("embed", 1.0), ("w1", WIDTH ** -0.5), ("w2", HIDDEN ** -0.5), ("out", 0.02)):
            shape = self.places[name][1]
            self.cut(x0, name).copy_(torch.randn(shape, generator=self.g, device="cuda") * scale)   # the same start for all
        for name in NORMS if norms else ():
            self.cut(x0, name).fill_(1.0)
        P = (np.ones((M, M)) - np.eye(M)) / (M - 1)
        self.run = nm.NetMax(M=M, D=D, ld=-(-D // nm.NETMAX_TILE) * nm.NETMAX_TILE, model=nm.NETMAX_FLAT, lr=LR, momentum=0.0, rho=float(P.max()) / (4 * LR),
                             seed=seed, P=P)
        self.run.set("x", x0)
        self.params, self.grads, self.moments = x0, torch.zeros(M, D, device="cuda"), torch.zeros(M, D, device="cuda")
        self.clipped = nm.Gradients([self.cut(self.grads, n) for n in self.places], batch=True)
        self.iteration = 0

    def cut(self, rows, name):
        """A parameter of all workers as a view of their rows [M, D]."""
        at, shape = self.places[name]
        return rows[:, at:at + int(np.prod(shape))].view(rows.shape[0], *shape)

    def forward(self, tokens):
        """Logits [M, T, VOCAB] of what follows each of tokens [M, T], and what the backward pass needs."""
        p = lambda name: self.cut(self.params, name)  # noqa: E731
        ids = tokens.to(torch.int32)
        e = nm.netmax_embed(ids, p("embed"))
        n = nm.netmax_block_norm(e, pre_gain=p("first_gain"))[1] if self.norms else e
        a, z = nm.netmax_linear(n, p("w1"), p("b1"), act="gelu", keep_preact=True)
        f = None
        if self.norms:
            f = nm.netmax_linear(a, p("w2"), p("b2"))
            h = nm.netmax_block_norm(e, f, p("gate"), p("post_gain"), None, p("pre_gain"), need_h=False)[1]
        else:
            h = nm.netmax_linear(a, p("w2"), p("b2"), e)                                            # onto the residual stream
        return nm.netmax_linear(h, p("out")), (ids, e, n, a, z, f, h)

    def backward(self, dlogits, kept):
        """Gradients of all parameters into the workers' rows."""
        ids, e, n, a, z, f, h = kept
        p, g = (lambda name: self.cut(self.params, name)), (lambda name: self.cut(self.grads, name))  # noqa: E731
        dh, _, _ = nm.netmax_linear_grad(dlogits, h, p("out"), dw=g("out"), need_bias=False)
        df = dh
        if self.norms:
            dh, df = nm.netmax_block_norm_grad(dh, None, e, f, p("gate"), p("post_gain"), None, p("pre_gain"), dgate=g("gate"), dpost_gain=g("post_gain"), dpre_gain=g("pre_gain"))[:2]
        da, _, _ = nm.netmax_linear_grad(df, a, p("w2"), dw=g("w2"), db=g("b2"))
        dn, _, _ = nm.netmax_linear_grad(da, n, p("w1"), z, act="gelu", dw=g("w1"), db=g("b1"))
        de = nm.netmax_block_norm_grad(dn, dh, e, pre_gain=p("first_gain"), dpre_gain=g("first_gain")).dx if self.norms else dh + dn
        nm.netmax_embed_grad(de, ids, dtable=g("embed"))

    def update(self):
        """One NetMax iteration: orthogonalised momentum of the matrices, momentum of the vectors, second step of the update with a drawn peer's copy."""
        g, m = self.grads, self.moments
        if self.clip:
            nm.netmax_clip_grads(self.clipped, self.clip)
        for name in self.places:
            g_, m_ = self.cut(g, name), self.cut(m, name)
            if name in MATRICES:
                rows, cols = self.places[name][1]
                nm.netmax_orthogonalize(g_, m_, mu=MU, out=g_, scale=0.2 * max(rows, cols) ** 0.5)
            else:
                g_.copy_(m_.mul_(MU).add_(g_))
        self.run.sample_peers(self.iteration)
        self.run.set("g", g)
        self.run.mix(self.iteration)
        self.params = self.run.get("x", self.D)
        self.iteration += 1


def teacher(seed: int = 1):
    """The hidden teacher: for each token the few tokens that may follow it."""
    return torch.randint(0, VOCAB, (VOCAB, 4), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


def write(rules, first, length, generator):
    """Sequences by the teacher's rules, or at random without rules: [..., length + 1] from the first tokens on."""
    seq = [first]
    for _ in range(length):
        if rules is None:
            seq.append(torch.randint(0, VOCAB, first.shape, generator=generator, device="cuda"))
        else:
            pick = torch.randint(0, rules.shape[1], first.shape, generator=generator, device="cuda")
            seq.append(rules[seq[-1], pick])
    return torch.stack(seq, -1)


def preference_step(w: Workers, rules):
    """Pairs that share their first token; returns the mean loss and the share of pairs that the workers' models order as the teacher does."""
    M = w.M
    first = torch.randint(0, VOCAB, (M, PAIRS), generator=w.g, device="cuda")
    both = torch.stack([write(rules, first, LENGTH, w.g), write(None, first, LENGTH, w.g)], 2).view(M, 2 * PAIRS, LENGTH + 1)
    logits, kept = w.forward(both[..., :-1].reshape(M, -1))
    labels = both[..., 1:].reshape(-1).to(torch.int32)
    offsets = torch.arange(0, 2 * M * PAIRS + 1, device="cuda", dtype=torch.int32) * LENGTH
    ref = torch.full((labels.numel(),), -float(np.log(VOCAB)), device="cuda")                       # the uniform model
    loss, ratio, grad = nm.netmax_preference_loss(logits.view(-1, VOCAB), labels, offsets, None, ref, beta=0.1, scale=1.0 / PAIRS)
    w.backward(grad.view(M, -1, VOCAB), kept)
    w.update()
    return float(loss.sum()) / M, float((ratio[0::2] > ratio[1::2]).float().mean())


def policy_step(w: Workers, rules, reference):
    """Sequences by the workers' own models, rewarded for each of the teacher's choices; returns the mean reward of a token."""
    M = w.M
    tokens = torch.randint(0, VOCAB, (M, 2 * PAIRS * LENGTH), generator=w.g, device="cuda")
    logits, kept = w.forward(tokens)
    chosen = torch.multinomial(torch.softmax(logits.view(-1, VOCAB), 1), 1, generator=w.g)[:, 0]
    reward = (rules[tokens.reshape(-1)] == chosen[:, None]).any(1).float()
    per_worker = reward.view(M, -1)
    advantage = ((per_worker - per_worker.mean(1, keepdim=True)) / (per_worker.std(1, keepdim=True) + 1e-4)).view(-1)
    old = torch.log_softmax(logits.view(-1, VOCAB), 1).gather(1, chosen[:, None])[:, 0]
    own, w.params = w.params, reference
    ref = torch.log_softmax(w.forward(tokens)[0].view(-1, VOCAB), 1).gather(1, chosen[:, None])[:, 0]
    w.params = own
    weight = torch.full_like(old, 1.0 / tokens.shape[1])
    _, _, grad = nm.netmax_policy_loss(logits.view(-1, VOCAB), chosen.to(torch.int32), old, advantage, weight, ref_logp=ref, kl=0.01)
    w.backward(grad.view(M, -1, VOCAB), kept)
    w.update()
    return float(reward.mean())


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--steps", type=int, default=60, help="iterations of each phase")
    ap.add_argument("--norms", action="store_true", help="norms before and after the residual block, and a gate for each channel")
    ap.add_argument("--clip", type=float, default=0.0, help="largest norm of a worker's gradients (0: any)")
    a = ap.parse_args(argv)
    w, rules, seen = Workers(a.workers, norms=a.norms, clip=a.clip), teacher(), []
    for k in range(a.steps):
        seen.append(preference_step(w, rules))
        if k % 10 == 0 or k + 1 == a.steps:
            print(f"pairs  {k:4d}: loss {seen[-1][0]:.4f}, pairs in order {seen[-1][1]:.3f}, consensus distance {w.run.consensus_dist():.4g}", flush=True)
    reference, rewards = w.params.clone(), []
    for k in range(a.steps):
        rewards.append(policy_step(w, rules, reference))
        if k % 10 == 0 or k + 1 == a.steps:
            print(f"policy {k:4d}: reward {rewards[-1]:.4f}, consensus distance {w.run.consensus_dist():.4g}", flush=True)
    w.run.close()
    return seen, rewards


if __name__ == "__main__":
    main()
