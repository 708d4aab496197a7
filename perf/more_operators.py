"""A sequence mixer with matrix states and an optimiser for its matrices, as cases that can be timed and checked.

A case is one call of an operator as a training or generating program makes it, on inputs made from a seed:

  linear       attention whose state decays by head, S_t = e^g_t S_{t-1} + k_t v_t^T, y_t = S_t^T q_t, over a ragged batch or
               one token of it (`train.linear_attention`)
  linear_grad  its backward pass (`train.linear_attention_grad`)
  orthogonal   Newton-Schulz iterations that bring a matrix' singular values near one (`train.orthogonalize`)
  muon         an optimiser step over the matrices of all workers along orthogonalised momentum (`train.Muon`)

With `own` false the same is computed by elementary torch operations in 32 bits, the sums of logarithms in 64.  `exact`
follows the definitions in 64 bits.
"""
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 64      # steps that the plain form takes at once
LR, DECAY, MOMENTUM = 0.02, 0.01, 0.95
ITERATIONS = 5
A, B, C = 3.4445, -4.7750, 2.0315       # of one iteration: X <- A X + (B (X X^T) + C (X X^T)^2) X
ELAPSED = 2     # optimiser steps that lie behind a run when `run` is first called


def listed():
    return [
        # generation: one token of each of 20 sequences on eight workers, the word-level model's 650 channels as 13 heads
        dict(name="linear_one_token", kind="linear", batch=160, steps=1, heads=13, dk=50, dv=50, type="f32", gate="step"),
        # ... and of a larger model's 64 sequences
        dict(name="linear_one_token_bf16", kind="linear", batch=64, steps=1, heads=16, dk=128, dv=128, type="bf16",
             gate="head"),
        # eight workers' minibatches of 20 sequences, 35 words each
        dict(name="linear_bptt", kind="linear", batch=160, steps=35, heads=13, dk=50, dv=50, type="f32", gate="step",
             ragged=True),
        # two long documents of different lengths
        dict(name="linear_long_bf16", kind="linear", batch=2, steps=32_768, heads=16, dk=128, dv=128, type="bf16",
             gate="step", ragged=True),
        # prompts in fp16, four heads to a query and key
        dict(name="linear_shared_f16", kind="linear", batch=8, steps=2000, heads=20, q_heads=5, k_heads=5, dk=64, dv=64,
             type="f16", gate="head"),
        # the backward passes of a minibatch, of a few long sequences and of one with keys and queries shared by heads
        dict(name="linear_grad_bptt", kind="linear_grad", batch=160, steps=35, heads=13, dk=50, dv=50, type="f32",
             gate="step", ragged=True),
        dict(name="linear_grad_long_bf16", kind="linear_grad", batch=4, steps=16_384, heads=10, dk=128, dv=128,
             type="bf16", gate="head"),
        dict(name="linear_grad_shared", kind="linear_grad", batch=3, steps=1001, heads=12, q_heads=4, k_heads=4, dk=64,
             dv=96, type="f32", gate="step", ragged=True),
        # one matrix of odd sides, and a stack of gradients in bf16
        dict(name="orthogonal_odd", kind="orthogonal", batch=1, rows=333, cols=1000, type="f32"),
        dict(name="orthogonal_stack_bf16", kind="orthogonal", batch=16, rows=1024, cols=640, type="bf16"),
        # four workers' projections in the small language model; eight workers' three recurrent layers of the word-level one
        dict(name="muon_small", kind="muon", n=4, layers="small", grad="f32"),
        dict(name="muon_recurrent", kind="muon", n=8, layers="recurrent", grad="f32"),
    ]


def draw(rng):
    """One more case of the listed kinds: sizes over the whole range by their logarithm, odd ones among them."""
    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    kind = rng.choice(["linear", "linear", "linear", "linear_grad", "linear_grad", "orthogonal", "muon"])
    some = rng.choice(["f32", "f32", "bf16", "bf16", "f16"])
    if kind in ("linear", "linear_grad"):
        dk = rng.choice([spread(8, 256), 64, 128])
        dv = rng.choice([dk, dk, spread(8, 256)])
        shared = rng.choice([1, 1, 2, 4])
        heads = shared * max(1, spread(1, 24) // shared)
        wide = max(dk, dv)
        batch = max(1, min(spread(1, 200), 30_000_000 // (heads * wide * wide)))
        most = (100_000_000 if kind == "linear" else 50_000_000) // (batch * heads * wide)
        steps = 1 if kind == "linear" and rng.random() < 0.3 else spread(2, max(3, min(32_768, most)))
        c = dict(kind=kind, batch=batch, steps=steps, heads=heads, dk=dk, dv=dv, type=some, gate=rng.choice(["step", "head"]),
                 ragged=steps > 1 and rng.random() < 0.5)
        for name in rng.choice([(), ("q_heads", "k_heads"), ("k_heads", "v_heads")]):
            c[name] = heads // shared
        return c
    if kind == "orthogonal":
        rows, cols = spread(17, 2048), spread(17, 2048)
        return dict(kind=kind, batch=max(1, min(spread(1, 24), 10_000_000_000 // (rows * cols * min(rows, cols)))), rows=rows,
                    cols=cols, type=rng.choice(["f32", "bf16"]))
    layers = rng.choice(["small", "recurrent", "mixed", "mixed"])
    c = dict(kind=kind, n=rng.choice([1, 2, 4, 8]), layers=layers, grad=rng.choice(["f32", "f32", "bf16"]))
    if layers == "recurrent":
        c["hidden"] = rng.randrange(60, 651, 2)
    elif layers == "small":
        c["hidden"] = rng.randrange(16, 129)
    else:
        c.update(lengths=rng.randrange(2, 12), table=rng.randrange(1 << 30))
    return c


# ---- inputs -----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _linear_inputs(c, seed):
    """(q, k, v, g, h0, lengths or None, dy, dh of the last state): q, k and v are columns of one projection."""
    gen = _generator(seed)
    n, T, H, dk, dv = c["batch"], c["steps"], c["heads"], c["dk"], c["dv"]
    hq, hk, hv = (c.get(name, H) for name in ("q_heads", "k_heads", "v_heads"))
    kind = TYPES[c["type"]]
    proj = torch.empty((n, T, (hq + hk) * dk + hv * dv), device="cuda", dtype=kind).normal_(0.0, 1.0, generator=gen)
    q, k = proj[..., :hq * dk].view(n, T, hq, dk), proj[..., hq * dk:(hq + hk) * dk].view(n, T, hk, dk)
    v = proj[..., (hq + hk) * dk:].view(n, T, hv, dv)
    k *= dk ** -0.5
    if c["gate"] == "head":     # heads that remember from 8 steps to 512
        g = torch.log1p(-torch.exp2(-3.0 - 6.0 * torch.rand(H, device="cuda", generator=gen)))
    else:                       # gates of every step, sigmoid(3 + noise): some twenty steps
        g = -torch.log1p(torch.exp(-3.0 - torch.randn((n, T, H), device="cuda", generator=gen)))
    h0 = torch.empty((n, H, dk, dv), device="cuda").normal_(0.0, 0.5, generator=gen)
    lengths = None
    if c.get("ragged"):
        lengths = torch.randint(T // 2, T + 1, (n,), device="cuda", generator=gen, dtype=torch.int32)
    dy = dh = None
    if c["kind"] == "linear_grad":
        dy = torch.empty((n, T, H, dv), device="cuda", dtype=kind).normal_(0.0, 1.0, generator=gen)
        dh = torch.empty((n, H, dk, dv), device="cuda").normal_(0.0, 1.0, generator=gen)
    return q, k, v, g, h0, lengths, dy, dh


def _spectrum(gen, shape):
    """Matrices as gradients and momenta are: a few strong directions over noise."""
    x = torch.empty(shape, device="cuda").normal_(0.0, 0.01, generator=gen)
    n, rows, cols = shape
    rank = max(1, min(rows, cols) // 16)
    left = torch.empty((n, rows, rank), device="cuda").normal_(0.0, 0.03, generator=gen)
    right = torch.empty((n, rank, cols), device="cuda").normal_(0.0, 1.0, generator=gen)
    return x + torch.bmm(left, right) * rank ** -0.5


def _shapes(c):
    """(rows, cols) of the matrices that lie one behind the other in a worker's row."""
    layers = c["layers"]
    if layers == "small":           # queries, keys and values of one layer from its input
        hidden = c.get("hidden", 64)
        return [(hidden, 3 * hidden)]
    if layers == "recurrent":       # three layers, from the input and from the state
        hidden = c.get("hidden", 650)
        return [(4 * hidden, hidden)] * 6
    gen = torch.Generator().manual_seed(c["table"])
    side = torch.rand((c["lengths"], 2), generator=gen)
    side = (24 * (1200 / 24) ** side).round().long()
    return [tuple(s) for s in side.tolist()]


def _muon_inputs(c, seed):
    """(X, G, how far each worker's gradient was clipped, starts): the workers' parameter rows and gradients."""
    gen = _generator(seed)
    start, at = [], 0
    for rows, cols in _shapes(c):
        start.append(at)
        at = (at + rows * cols + 3) // 4 * 4
    shape = (c["n"], (at + 63) // 64 * 64)
    X = torch.empty(shape, device="cuda").normal_(0.0, 0.05, generator=gen)
    G = torch.zeros(shape, device="cuda", dtype=TYPES[c["grad"]])
    for a, (rows, cols) in zip(start, _shapes(c)):
        G[:, a:a + rows * cols] = _spectrum(gen, (c["n"], rows, cols)).flatten(1).to(G.dtype)
    clip = torch.rand(c["n"], device="cuda", generator=gen) * 0.5 + 0.5
    return X, G, clip, start


def prepare(case, seed):
    c = case
    if c["kind"] in ("linear", "linear_grad"):
        q, k, v, g, h0, lengths, dy, dh = _linear_inputs(c, seed)
        state = dict(kind=c["kind"], case=c, q=q, k=k, v=v, g=g, h0=h0, lengths=lengths, dy=dy, dh=dh)
        if own and c["kind"] == "linear_grad":      # what the forward pass kept
            from paper_1907_09356_amd import train
            state["saved"] = train.linear_attention(q, k, v, g, h0=h0, lengths=lengths, save=True)[2]
        return state
    if c["kind"] == "orthogonal":
        gen = _generator(seed)
        return dict(kind="orthogonal", case=c, x=_spectrum(gen, (c["batch"], c["rows"], c["cols"])).to(TYPES[c["type"]]))
    X, G, clip, start = _muon_inputs(c, seed)
    state = dict(kind="muon", case=c, X=X, G=G, clip=clip, start=start)
    if own:
        from paper_1907_09356_amd import train
        rows, cols = zip(*_shapes(c))
        state["opt"] = train.Muon(X, X.shape[1], (start, rows, cols), momentum=MOMENTUM, weight_decay=DECAY,
                                  iterations=ITERATIONS)
    else:
        state["m"] = [torch.zeros((c["n"],) + s, device="cuda") for s in _shapes(c)]
    for _ in range(ELAPSED):
        _step(state)
    return state


# ---- one pass ---------------------------------------------------------------------------------
def run(state):
    kind = state["kind"]
    if kind == "linear":
        return _linear(state)
    if kind == "linear_grad":
        return _linear_grad(state)
    if kind == "orthogonal":
        if own:
            from paper_1907_09356_amd import train
            return train.orthogonalize(state["x"], iterations=ITERATIONS)
        return _orthogonal(state["x"].float())
    _step(state)
    X, m = state["X"], state["opt"].momentum() if "opt" in state else state["m"]
    return {"x": X, "m": m}


def _in_chunks(s, x):
    """(batch, steps, heads, ...) as (batch, all heads, chunks, steps of a chunk, ...) of fp32, zero outside a sequence."""
    T, H = x.shape[1], s["case"]["heads"]
    if s["lengths"] is not None:
        inside = torch.arange(T, device="cuda") < s["lengths"][:, None]
        x = torch.where(inside.view(inside.shape + (1,) * (x.dim() - 2)), x, 0.0)
    x = x.float().repeat_interleave(H // x.shape[2], 2)
    size = min(T, CHUNK)
    whole = -(-T // size) * size
    x = torch.nn.functional.pad(x, (0, 0) * (x.dim() - 2) + (0, whole - T))
    return x.movedim(2, 1).unflatten(2, (-1, size))


def _whole(s, x):
    """Back from chunks: (batch, steps, heads, ...)."""
    return x.flatten(2, 3)[:, :, :s["case"]["steps"]].movedim(1, 2)


def _differences(x):
    """e^(x_t - x_s) where s <= t, else 0, of fp32; x in 64 bits."""
    n = x.shape[-1]
    below = torch.ones((n, n), device="cuda", dtype=torch.bool).tril()
    return torch.where(below, x[..., :, None] - x[..., None, :], -torch.inf).exp().float()


def _gates(s):
    """Logarithms of the decay since a chunk began and its powers between two steps; those since the first chunk between two
    chunks' ends (the first entry: the beginning)."""
    c = s["case"]
    g = s["g"].expand(c["batch"], c["steps"], c["heads"])
    since = _in_chunks(s, g[..., None])[..., 0].double().cumsum(3)
    ends = torch.nn.functional.pad(since[..., -1].cumsum(2), (1, 0))
    return since, _differences(since), _differences(ends)


def _states(s, k, v, since, between):
    """States before each chunk, and after the last one: (batch, heads, chunks + 1, dk, dv)."""
    left = (since[..., -1:] - since).exp().float()
    enter = torch.matmul((k * left[..., None]).transpose(3, 4), v)
    enter = torch.cat((s["h0"][:, :, None], enter), 2)
    return torch.matmul(between, enter.flatten(3)).view(enter.shape)


def _linear(s):
    if own:
        from paper_1907_09356_amd import train
        y, last, _ = train.linear_attention(s["q"], s["k"], s["v"], s["g"], h0=s["h0"], lengths=s["lengths"])
        return {"y": y, "h": last}
    q, k, v = (_in_chunks(s, s[name]) for name in ("q", "k", "v"))
    since, within, between = _gates(s)
    states = _states(s, k, v, since, between)
    y = torch.matmul(torch.matmul(q, k.transpose(3, 4)) * within, v)
    y = y + torch.matmul(q * since.exp().float()[..., None], states[:, :, :-1])
    return {"y": _whole(s, y).to(s["v"].dtype), "h": states[:, :, -1].contiguous()}


def _shared(s, x, like):
    """A gradient of all heads summed over those that share one."""
    x = _whole(s, x)
    return x.unflatten(2, like.shape[2:3] + (-1,)).sum(3).to(like.dtype)


def _linear_grad(s):
    if own:
        from paper_1907_09356_amd import train
        dq, dk, dv, dg, dh0 = train.linear_attention_grad(s["q"], s["k"], s["v"], s["g"], s["saved"], s["dy"],
                                                          lengths=s["lengths"], dlast=s["dh"])
        return {"dq": dq, "dk": dk, "dv": dv, "dg": dg, "dh0": dh0}
    q, k, v, dy = (_in_chunks(s, s[name]) for name in ("q", "k", "v", "dy"))
    since, within, between = _gates(s)
    before = _states(s, k, v, since, between)[:, :, :-1]
    here, left = since.exp().float()[..., None], (since[..., -1:] - since).exp().float()[..., None]
    enter = torch.cat((torch.matmul((q * here).transpose(3, 4), dy), s["dh"][:, :, None]), 2)
    after = torch.matmul(between.transpose(2, 3), enter.flatten(3)).view(enter.shape)      # gradients of states
    dh0, after = after[:, :, 0].contiguous(), after[:, :, 1:]
    score, dscore = torch.matmul(q, k.transpose(3, 4)), torch.matmul(dy, v.transpose(3, 4)) * within
    from_state, from_later = torch.matmul(dy, before.transpose(3, 4)) * here, torch.matmul(v, after.transpose(3, 4)) * left
    dq = torch.matmul(dscore, k) + from_state
    dk = torch.matmul(dscore.transpose(3, 4), q) + from_later
    dv = torch.matmul((score * within).transpose(3, 4), dy) + torch.matmul(k, after) * left
    # the gate of a step carries what goes from steps before it to that one or later: both in the chunk, one, or none
    pairs = torch.nn.functional.pad((score * dscore).flip(3).cumsum(3).flip(3).cumsum(4), (1, 0))[..., :-1]
    dg = pairs.diagonal(dim1=3, dim2=4) + (q * from_state).sum(4).flip(3).cumsum(3).flip(3)
    dg = dg + torch.nn.functional.pad((k * from_later).sum(4).cumsum(3), (1, 0))[..., :-1]
    dg = dg + (since[..., -1:].exp().float() * (before * after).sum((3, 4))[..., None])
    dg = _whole(s, dg[..., None])[..., 0]
    if s["lengths"] is not None:
        dg = torch.where((torch.arange(dg.shape[1], device="cuda") < s["lengths"][:, None])[..., None], dg, 0.0)
    dg = dg.contiguous() if s["g"].dim() == 3 else dg.sum((0, 1))
    return {"dq": _shared(s, dq, s["q"]), "dk": _shared(s, dk, s["k"]), "dv": _shared(s, dv, s["v"]), "dg": dg, "dh0": dh0}


def _iterate(x):
    gram = torch.bmm(x, x.transpose(1, 2).contiguous())
    return A * x + torch.bmm(B * gram + C * torch.bmm(gram, gram), x)


def _orthogonal(x):
    """x (batch, rows, cols) after ITERATIONS iterations, from x over its Frobenius norm."""
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / x.flatten(1).norm(dim=1)[:, None, None]
    for _ in range(ITERATIONS):
        x = _iterate(x)
    return x.transpose(1, 2).contiguous() if tall else x


def _step(s):
    if "opt" in s:
        s["opt"].step(s["G"], LR, grad_scale=s["clip"])
        return
    for a, m in zip(s["start"], s["m"]):
        n, rows, cols = m.shape
        x, g = (s[name][:, a:a + rows * cols].view(n, rows, cols) for name in ("X", "G"))
        g = g.float() * s["clip"][:, None, None]
        m.copy_(MOMENTUM * m + g)
        x.copy_(x * (1 - LR * DECAY) - LR * max(1.0, rows / cols) ** 0.5 * _orthogonal(g + MOMENTUM * m))


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("linear", "linear_grad"):
        H, dk, dv = c["heads"], c["dk"], c["dv"]
        hq, hk, hv = (c.get(name, H) for name in ("q_heads", "k_heads", "v_heads"))
        steps = c["batch"] * c["steps"] * (0.75 if c.get("ragged") else 1.0)
        whole, size = c["batch"] * c["steps"], BYTES[c["type"]]      # outputs are zero outside a sequence
        gates, states = 4 * steps * H if c["gate"] == "step" else 0, 8 * c["batch"] * H * dk * dv
        inputs, ops = (hq + hk) * dk + hv * dv, steps * H * dk * dv
        if c["kind"] == "linear":       # step by step: decay and add a product, multiply by q
            return {"bytes": size * (steps * inputs + whole * H * dv) + gates + states, "flops": 5 * ops}
        # the states again and their gradients, three products, one for the gates
        return {"bytes": size * (steps * (inputs + H * dv) + whole * inputs) + 2 * gates + states, "flops": 14 * ops}
    if c["kind"] == "orthogonal":
        n, shapes = c["batch"], [(c["rows"], c["cols"])]
        size = BYTES[c["type"]] + 4
    else:       # x and the momentum in and out, g in
        n, shapes, size = c["n"], _shapes(c), 16 + BYTES[c["grad"]]
    flops = 0
    for rows, cols in shapes:       # a product of two symmetric matrices and one with its own transpose by half
        a, b = min(rows, cols), max(rows, cols)
        flops += ITERATIONS * (a * a * b + a ** 3 + 2 * a * a * b)
    return {"bytes": n * size * sum(rows * cols for rows, cols in shapes), "flops": n * flops}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    return {"linear": _exact_linear, "linear_grad": _exact_linear_grad, "orthogonal": _exact_orthogonal,
            "muon": _exact_muon}[case["kind"]](case, seed)


class _Recurrence:
    """The inputs of a step in 64 bits for all heads, and the state from step to step."""

    def __init__(self, c, seed):
        self.q, self.k, self.v, self.g, self.h0, self.lengths, self.dy, self.dh = _linear_inputs(c, seed)
        self.c = c

    def of(self, x, t):
        x = x[:, t].double()
        return x.repeat_interleave(self.c["heads"] // x.shape[1], 1)

    def gate(self, t):
        g = self.g if self.g.dim() == 1 else self.g[:, t]
        return g.double().exp().expand(self.c["batch"], -1)[..., None, None]

    def inside(self, t):
        if self.lengths is None:
            return torch.ones((self.c["batch"], 1, 1, 1), device="cuda", dtype=torch.bool)
        return (t < self.lengths)[:, None, None, None]

    def after(self, S, t):
        new = self.gate(t) * S + self.of(self.k, t)[..., :, None] * self.of(self.v, t)[..., None, :]
        return torch.where(self.inside(t), new, S)


def _exact_linear(c, seed):
    r = _Recurrence(c, seed)
    y = torch.zeros((c["batch"], c["steps"], c["heads"], c["dv"]), device="cuda", dtype=torch.float64)
    S = r.h0.double()
    for t in range(c["steps"]):
        S = r.after(S, t)
        y[:, t] = torch.where(r.inside(t)[..., 0], (r.of(r.q, t)[..., None] * S).sum(2), 0.0)
    return {"y": y, "h": S}


def _exact_linear_grad(c, seed):
    r = _Recurrence(c, seed)
    T, H, batch = c["steps"], c["heads"], c["batch"]
    wide = {"device": "cuda", "dtype": torch.float64}
    dq, dk, dv, dg = (torch.zeros((batch, T, H) + d, **wide) for d in ((c["dk"],), (c["dk"],), (c["dv"],), ()))
    span = max(1, int(T ** 0.5))
    kept, S = [], r.h0.double()
    for t in range(T):
        if t % span == 0:
            kept.append(S)
        S = r.after(S, t)
    E = r.dh.double()       # gradient of the state after step t
    for first in reversed(range(0, T, span)):
        S = [kept.pop()]
        for t in range(first, min(first + span, T)):
            S.append(r.after(S[-1], t))
        for t in reversed(range(first, min(first + span, T))):
            inside, dy = r.inside(t), r.of(r.dy, t)
            here, now = S[t - first], S[t - first + 1]
            full = E + r.of(r.q, t)[..., :, None] * dy[..., None, :]
            dq[:, t] = torch.where(inside[..., 0], (now * dy[..., None, :]).sum(3), 0.0)
            dk[:, t] = torch.where(inside[..., 0], (full * r.of(r.v, t)[..., None, :]).sum(3), 0.0)
            dv[:, t] = torch.where(inside[..., 0], (full * r.of(r.k, t)[..., :, None]).sum(2), 0.0)
            dg[:, t] = torch.where(inside[..., 0, 0], (full * here * r.gate(t)).sum((2, 3)), 0.0)
            E = torch.where(inside, full * r.gate(t), E)
    share = [x.unflatten(2, like.shape[2:3] + (-1,)).sum(3) for x, like in ((dq, r.q), (dk, r.k), (dv, r.v))]
    return {"dq": share[0], "dk": share[1], "dv": share[2], "dg": dg if r.g.dim() == 3 else dg.sum((0, 1)), "dh0": E}


def _exact_polynomial(x):
    """The iterations in 64 bits on a stack of matrices, from the left or the right, whichever Gram matrix is smaller."""
    x = x / x.square().sum((1, 2), keepdim=True).sqrt()
    for _ in range(ITERATIONS):
        t = x.transpose(1, 2).contiguous()
        if x.shape[1] <= x.shape[2]:
            p = torch.matmul(x, t)
            x = A * x + B * torch.matmul(p, x) + C * torch.matmul(p, torch.matmul(p, x))
        else:
            p = torch.matmul(t, x)
            x = A * x + B * torch.matmul(x, p) + C * torch.matmul(torch.matmul(x, p), p)
    return x


def _exact_orthogonal(c, seed):
    gen = _generator(seed)
    return _exact_polynomial(_spectrum(gen, (c["batch"], c["rows"], c["cols"])).to(TYPES[c["type"]]).double())


def _exact_muon(c, seed):
    X, G, clip, start = _muon_inputs(c, seed)
    X, moments = X.double(), []
    for a, (rows, cols) in zip(start, _shapes(c)):
        g = G[:, a:a + rows * cols].reshape(-1, rows, cols).double() * clip.double()[:, None, None]
        x, m = X[:, a:a + rows * cols].reshape(-1, rows, cols), torch.zeros_like(g)
        for _ in range(ELAPSED + 1):
            m = MOMENTUM * m + g
            x = x - LR * (DECAY * x + max(1.0, rows / cols) ** 0.5 * _exact_polynomial(g + MOMENTUM * m))
        X[:, a:a + rows * cols] = x.flatten(1)
        moments.append(m)
    return {"x": X, "m": moments}
