"""A word-level language model trained by decentralised workers, every part of a worker's step on its rows of X and G.

n workers on a ring each hold the model's parameters in their row of X: a tied embedding, the projection of a gated linear
recurrence (or of linear attention, whose heads' decays are gates of every step), and an output bias.  An iteration looks the words up
in the workers' own tables, runs the recurrence (or the attention), takes the softmax loss of the next words over the tied table, goes
back through all of it into the workers' rows of G (the output layer's gradient first, the lookups' added to it), takes an AdamW step
with moments in 8 bits (or a step along the projections' orthogonalised momentum, and AdamW for the rest), each worker's gradient
clipped to its norm, and ends with a CHOCO-Gossip step that sends the largest 5 % of each tensor's differences.  Then the first worker
continues a text word by word from the state its prompt left.

The text is a seeded Markov chain in which each word has four likely successors, so there is something to learn:
guessing costs log(vocab), knowing the chain about log(4).

    python examples/decentral_lm.py [--steps 200] [--workers 4] [--mixer attention] [--optimiser muon]
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

    def __init__(self, vocab, dim, mixer="recurrence", heads=4):
        self.vocab, self.dim, self.mixer, self.heads = vocab, dim, mixer, heads
        wide = 3 * dim if mixer == "recurrence" else 3 * dim + heads      # f, u, o, or q, k, v and the heads' gates
        self.shapes = {"table": (vocab, dim), "project": (dim, wide), "project_bias": (wide,), "bias": (vocab,)}
        self.layers = synth.layer_table([math.prod(s) for s in self.shapes.values()], fraction=0.05)
        self.d = synth.layers_dim(self.layers)
        self.ld = (self.d + 63) // 64 * 64

    def views(self, rows):
        return {name: rows[:, int(a):int(a) + int(count)].view(rows.shape[0], *shape)
                for (name, shape), a, count in zip(self.shapes.items(), self.layers[0], self.layers[1])}

    def mix(self, z, state=None, keep=False):
        """The mixer on projections z (sequences, steps, wide) from a state on: output, last state, what the way back needs."""
        if self.mixer == "recurrence":
            f, u, o = z.split(self.dim, 2)
            y, last, saved = train.recurrence(f, u, o, h0=state, save=keep, h_last=state)
            return y, last, (f, u, o, saved)
        each = self.dim // self.heads
        q, k, v = (part.unflatten(2, (self.heads, each)) for part in z[..., :3 * self.dim].split(self.dim, 2))
        k, gate = k / each, z[..., 3 * self.dim:] + 3.0       # heads remember some twenty steps at first
        g = torch.nn.functional.logsigmoid(gate)
        y, last, saved = train.linear_attention(q, k, v, g, h0=state, save=keep, h_last=state)
        return y.flatten(2), last, (q, k, v, g, gate, saved)

    def mix_grad(self, dy, kept):
        """The gradient of z."""
        if self.mixer == "recurrence":
            f, u, o, saved = kept
            return torch.cat(train.recurrence_grad(f, u, saved, dy, o)[:3], 2)
        q, k, v, g, gate, saved = kept
        dq, dk, dv, dg, _ = train.linear_attention_grad(q, k, v, g, saved, dy.unflatten(2, (self.heads, -1)))
        return torch.cat((dq.flatten(2), dk.flatten(2) / k.shape[3], dv.flatten(2), dg * torch.sigmoid(-gate)), 2)

    def forward(self, X, words, keep=False):
        """Output of the mixer for words (n, sequences, steps) and what the way back needs."""
        p, (n, sequences, steps) = self.views(X), words.shape
        x = train.embed(words.reshape(n, -1), p["table"], scale=self.dim ** 0.5)
        z = torch.baddbmm(p["project_bias"][:, None], x, p["project"]).view(n * sequences, steps, -1)
        y, last, kept = self.mix(z, keep=keep)
        return y.reshape(n, -1, self.dim), last, (x, kept)

    def gradient(self, X, G, words, target):
        """Fills G with the gradients of the workers' mean losses; returns the losses."""
        p, g = self.views(X), self.views(G)
        n, sequences, steps = words.shape
        count, dim = sequences * steps, self.dim
        y, _, (x, kept) = self.forward(X, words, keep=True)
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
        dz = self.mix_grad(dy.view(n * sequences, steps, dim), kept).view(n, count, -1)
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
            y = self.mix((x @ p["project"][0] + p["project_bias"][0])[:, None], state)[0][:, 0]
        return torch.stack(words, 1)

    def optimisers(self, X, kind, seed):
        """What updates the tensors, with a factor of the learning rate for each."""
        start, count, _ = self.layers
        decay = [0.01 if len(s) > 1 else 0.0 for s in self.shapes.values()]
        if kind == "adamw":
            return [(train.AdamW(X, self.d, (start, count), weight_decay=decay, state_bits=8, seed=seed), 1.0)]
        matrix = [name == "project" for name in self.shapes]
        rows, cols = zip(*(s for s, m in zip(self.shapes.values(), matrix) if m))
        rest = [i for i, m in enumerate(matrix) if not m]
        return [(train.Muon(X, self.d, ([a for a, m in zip(start, matrix) if m], rows, cols), weight_decay=0.01), 2.0),
                (train.AdamW(X, self.d, (start[rest], count[rest]), weight_decay=[decay[i] for i in rest], state_bits=8, seed=seed), 1.0)]


def chain_text(vocab, shape, generator, successors):
    """Words of the Markov chain, (..., steps)."""
    words = torch.empty(shape, dtype=torch.int64, device=successors.device)
    words[..., 0] = torch.randint(0, vocab, shape[:-1], generator=generator, device=successors.device)
    pick = torch.randint(0, successors.shape[1], shape, generator=generator, device=successors.device)
    for t in range(1, shape[-1]):
        words[..., t] = successors[words[..., t - 1], pick[..., t]]
    return words


def run(steps=200, workers=4, vocab=500, dim=64, sequences=20, length=35, seed=1, log=print, mixer="recurrence", optimiser="adamw"):
    """Trains; returns (first losses, last losses, consensus distance, share of generated words that the chain allows)."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    successors = torch.randint(0, vocab, (vocab, 4), generator=gen, device="cuda")
    model = Model(vocab, dim, mixer)
    X = torch.zeros((workers, model.ld), device="cuda")
    first = {"table": dim ** -0.5 * 0.5, "project": dim ** -0.5, "project_bias": 0.0, "bias": 0.0}
    for name, view in model.views(X).items():      # Algorithm 1 starts all workers from one point
        view.copy_(torch.empty(view.shape[1:], device="cuda").normal_(0.0, first[name], generator=gen).expand_as(view))
    G = torch.zeros_like(X)
    optimisers = model.optimisers(X, optimiser, seed)
    gossip = B.Choco(X, model.d, *synth.ring_csr(workers), 0.15, B.Q_TOPK, layers=model.layers)
    begin = losses = None
    for t in range(steps):
        text = chain_text(vocab, (workers, sequences, length + 1), gen, successors)
        losses = model.gradient(X, G, text[..., :-1], text[..., 1:])
        begin = losses if begin is None else begin
        clip = (1.0 / G.norm(dim=1)).clamp_(max=1.0)
        for opt, factor in optimisers:
            opt.step(G, factor * 0.01 * min(1.0, (steps - t) / (0.3 * steps)), grad_scale=clip)
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
    for opt, _ in optimisers:
        opt.close()
    return begin.tolist(), losses.tolist(), consensus, allowed


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--mixer", choices=["recurrence", "attention"], default="recurrence")
    ap.add_argument("--optimiser", choices=["adamw", "muon"], default="adamw")
    a = ap.parse_args()
    run(a.steps, a.workers, mixer=a.mixer, optimiser=a.optimiser)
