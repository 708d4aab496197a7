"""A word-level language model trained by decentralised workers, every part of a worker's step on its rows of X and G.

n workers on a ring each hold the model's parameters in their row of X: a tied embedding, the projection of a gated linear
recurrence, and an output bias.  An iteration looks the words up in the workers' own tables, runs the recurrence, takes the
softmax loss of the next words over the tied table, goes back through all of it into the workers' rows of G (the output
layer's gradient first, the lookups' added to it), takes an AdamW step with moments in 8 bits and each worker's gradient clipped
to its norm, and ends with a CHOCO-Gossip step that sends the largest 5 % of each tensor's differences.  Then the first worker
continues a text word by word from the state its prompt left.

The text is a seeded Markov chain in which each word has four likely successors, so there is something to learn:
guessing costs log(vocab), knowing the chain about log(4).

    python examples/decentral_lm.py [--steps 200] [--workers 4]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1907_09356_amd import binding as B, synth, train  # noqa: E402


class Model:
    """Views of the workers' parameters in rows of n x ld floats."""

    def __init__(self, vocab, dim):
        self.vocab, self.dim = vocab, dim
        self.shapes = {"table": (vocab, dim), "project": (dim, 3 * dim), "project_bias": (3 * dim,), "bias": (vocab,)}
        self.layers = synth.layer_table([math.prod(s) for s in self.shapes.values()], fraction=0.05)
        self.d = synth.layers_dim(self.layers)
        self.ld = (self.d + 63) // 64 * 64

    def views(self, rows):
        return {name: rows[:, int(a):int(a) + int(count)].view(rows.shape[0], *shape)
                for (name, shape), a, count in zip(self.shapes.items(), self.layers[0], self.layers[1])}

    def forward(self, X, words, keep=False):
        """Output of the recurrence for words (n, sequences, steps) and what the way back needs."""
        p, (n, sequences, steps) = self.views(X), words.shape
        x = train.embed(words.reshape(n, -1), p["table"], scale=self.dim ** 0.5)
        z = torch.baddbmm(p["project_bias"][:, None], x, p["project"]).view(n * sequences, steps, 3 * self.dim)
        f, u, o = z.split(self.dim, 2)
        y, last, saved = train.recurrence(f, u, o, save=keep)
        return y.view(n, -1, self.dim), last, (x, f, u, o, saved)

    def gradient(self, X, G, words, target):
        """Fills G with the gradients of the workers' mean losses; returns the losses."""
        p, g = self.views(X), self.views(G)
        n, sequences, steps = words.shape
        count, dim = sequences * steps, self.dim
        y, _, (x, f, u, o, saved) = self.forward(X, words, keep=True)
        table_t = p["table"].transpose(1, 2).contiguous()
        logits = torch.baddbmm(p["bias"][:, None], y, table_t)
        logp = logits.log_softmax(2)
        at = target.reshape(n, count, 1)
        losses = -logp.gather(2, at).mean((1, 2))
        dlogits = logp.exp_()
        dlogits.scatter_add_(2, at, torch.full_like(at, -1, dtype=torch.float32))
        dlogits /= count
        g["bias"].copy_(dlogits.sum(1))
        g["table"].copy_(torch.bmm(dlogits.transpose(1, 2).contiguous(), y))
        dy = torch.bmm(dlogits, p["table"].contiguous())
        df, du, do, _ = train.recurrence_grad(f, u, saved, dy.view(n * sequences, steps, dim), o)
        dz = torch.cat((df, du, do), 2).view(n, count, 3 * dim)
        g["project_bias"].copy_(dz.sum(1))
        g["project"].copy_(torch.bmm(x.transpose(1, 2).contiguous(), dz))
        dx = torch.bmm(dz, p["project"].transpose(1, 2).contiguous())
        train.embed_grad(words.reshape(n, -1), dx, g["table"], scale=dim ** 0.5, accumulate=True)
        return losses

    def generate(self, X, prompt, count):
        """The likeliest continuation of prompt (sequences, steps) by the first worker, a word at a time."""
        X = X[:1]
        p = self.views(X)
        y, state, _ = self.forward(X, prompt[None])
        y = y.view(prompt.shape[0], prompt.shape[1], self.dim)[:, -1]
        words = []
        for _ in range(count):
            words.append((y @ p["table"][0].t() + p["bias"][0]).argmax(1))
            x = train.embed(words[-1][None], p["table"], scale=self.dim ** 0.5)[0]
            f, u, o = (x @ p["project"][0] + p["project_bias"][0])[:, None].split(self.dim, 2)
            y = train.recurrence(f, u, o, h0=state, h_last=state)[0][:, 0]
        return torch.stack(words, 1)


def chain_text(vocab, shape, generator, successors):
    """Words of the Markov chain, (..., steps)."""
    words = torch.empty(shape, dtype=torch.int64, device=successors.device)
    words[..., 0] = torch.randint(0, vocab, shape[:-1], generator=generator, device=successors.device)
    pick = torch.randint(0, successors.shape[1], shape, generator=generator, device=successors.device)
    for t in range(1, shape[-1]):
        words[..., t] = successors[words[..., t - 1], pick[..., t]]
    return words


def run(steps=200, workers=4, vocab=500, dim=64, sequences=20, length=35, seed=1, log=print):
    """Trains; returns (first losses, last losses, consensus distance, share of generated words that the chain allows)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda")
    model = Model(vocab, dim)
    X = torch.zeros((workers, model.ld), device="cuda")
    first = {"table": dim ** -0.5 * 0.5, "project": dim ** -0.5, "project_bias": 0.0, "bias": 0.0}
    for name, view in model.views(X).items():      # Algorithm 1 starts all workers from one point
        view.copy_(torch.empty(view.shape[1:], device="cuda").normal_(0.0, first[name], generator=gen).expand_as(view))
    G = torch.zeros_like(X)
    start, count, _ = model.layers
    decay = [0.01 if len(s) > 1 else 0.0 for s in model.shapes.values()]
    opt = train.AdamW(X, model.d, (start, count), weight_decay=decay, state_bits=8, seed=seed)
    gossip = B.Choco(X, model.d, *synth.ring_csr(workers), 0.15, B.Q_TOPK, layers=model.layers)
    begin = losses = None
    for t in range(steps):
        text = chain_text(vocab, (workers, sequences, length + 1), gen, successors)
        losses = model.gradient(X, G, text[..., :-1], text[..., 1:])
        begin = losses if begin is None else begin
        clip = (1.0 / G.norm(dim=1)).clamp_(max=1.0)
        opt.step(G, 0.01 * min(1.0, (steps - t) / (0.3 * steps)), grad_scale=clip)
        gossip.gossip_step()
        if t % 20 == 0 or t + 1 == steps:
            log("step %4d  loss %s  consensus distance %.4g" % (t, " ".join("%.3f" % v for v in losses.tolist()),
                                                             gossip.metrics()["consensus"]))
    prompt = chain_text(vocab, (8, 12), gen, successors)
    words = torch.cat((prompt[:, -1:], model.generate(X, prompt, 20)), 1)
    allowed = (successors[words[:, :-1]] == words[:, 1:, None]).any(2).float().mean().item()
    log("continuations: %.0f %% of the words follow as the chain allows" % (100 * allowed))
    consensus = gossip.metrics()["consensus"]
    gossip.close()
    opt.close()
    return begin.tolist(), losses.tolist(), consensus, allowed


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=4)
    a = ap.parse_args()
    run(a.steps, a.workers)
