"""The local step of a language model's workers, operator by operator, as cases that can be timed and checked.

A case is one call of an operator as a training or generating program makes it, on inputs made from a seed:

  embed        rows of every worker's embedding looked up and scaled (`train.embed`)
  embed_grad   its gradient summed by token into the workers' gradient rows (`train.embed_grad`)
  recur        a gated linear recurrence over a ragged batch, or one token of it (`train.recurrence`)
  recur_grad   its backward pass (`train.recurrence_grad`)
  adamw        an AdamW step over all tensors of all workers, moments in 32 or 8 bits (`train.AdamW`)

With `own` false the same is computed by elementary torch operations in 32 bits.  `exact` follows the
definitions in 64 bits.
"""
import functools

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-3, 0.1
BLOCK = 256     # entries of a tensor that share a scale where the moments are held in 8 bits
ELAPSED = 2     # optimiser steps that lie behind a run when `run` is first called


def listed():
    return [
        # one token for each of 20 sequences on eight workers, out of the word-level model's 33,278 x 650 table
        dict(name="embed_one_token", kind="embed", n=8, tokens=20, vocab=33278, dim=650, table="f32", out="f32"),
        # prompts of a larger model in bf16, a tenth of the positions padding
        dict(name="embed_prompts_bf16", kind="embed", n=1, tokens=49_153, vocab=100_003, dim=2048, table="bf16",
             out="bf16", padding=0.1),
        # the word-level model on eight workers, 32 sequences of 35 words each: the gradient fills its slice of G
        dict(name="embed_grad_workers", kind="embed_grad", n=8, tokens=1120, vocab=33278, dim=650, out="f32"),
        # a tied table: the output layer's gradient is there already and the lookups' is added, frequent words often
        dict(name="embed_grad_tied_bf16", kind="embed_grad", n=1, tokens=65_536, vocab=100_003, dim=1024, out="bf16",
             padding=0.1, add=True),
        # generation: one token of every sequence, the state carried from call to call
        dict(name="recur_one_token", kind="recur", batch=160, steps=1, dim=650, type="f32", gate=True),
        # eight workers' minibatches of 20 sequences, 35 words each
        dict(name="recur_bptt", kind="recur", batch=160, steps=35, dim=650, type="f32", gate=True, ragged=True),
        # two long documents of different lengths
        dict(name="recur_long_bf16", kind="recur", batch=2, steps=32_768, dim=2048, type="bf16", gate=True, ragged=True),
        # the backward passes of a minibatch and of a few long sequences without an output gate
        dict(name="recur_grad_bptt", kind="recur_grad", batch=160, steps=35, dim=650, type="f32", gate=True, ragged=True),
        dict(name="recur_grad_long_bf16", kind="recur_grad", batch=4, steps=16_384, dim=1280, type="bf16", gate=False),
        # eight workers on the 0.27 M image model's 65 tensors, no decay on the short ones
        dict(name="adamw_image", kind="adamw", n=8, layers="image", grad="f32", bits=32),
        # eight workers on the language model's 31.8 M entries, moments in 32 bits
        dict(name="adamw_language", kind="adamw", n=8, layers="language", grad="f32", bits=32),
        # ... and in 8 bits, gradients out of a backward pass in bf16
        dict(name="adamw_language_8bit", kind="adamw", n=4, layers="language", grad="bf16", bits=8),
    ]


def draw(rng):
    """One more case of the listed kinds: sizes over the whole range by their logarithm, odd ones among them."""
    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    kind = rng.choice(["embed", "embed_grad", "recur", "recur_grad", "adamw", "adamw"])
    some = rng.choice(["f32", "f32", "bf16", "bf16", "f16"])
    if kind in ("embed", "embed_grad"):
        n = rng.choice([1, 1, 2, 4, 8, 16])
        dim = spread(33, 2048)
        vocab = max(2, min(spread(500, 130_000), 260_000_000 // (n * dim)))
        c = dict(kind=kind, n=n, tokens=max(1, min(spread(16, 65_536), 100_000_000 // (n * dim))), vocab=vocab, dim=dim,
                 out=some, padding=rng.choice([0.0, 0.0, 0.1, 0.4]))
        if kind == "embed":
            c["table"] = rng.choice([some, "f32"])
        else:
            c["add"] = rng.random() < 0.5
        return c
    if kind in ("recur", "recur_grad"):
        dim = spread(33, 2048)
        batch = spread(1, 200)
        steps = 1 if kind == "recur" and rng.random() < 0.15 else spread(2, max(3, min(32_768, 80_000_000 // (dim * batch))))
        return dict(kind=kind, batch=batch, steps=steps, dim=dim, type=some, gate=rng.random() < 0.7,
                    ragged=steps > 1 and rng.random() < 0.5)
    layers = rng.choice(["image", "language", "mixed", "mixed"])
    c = dict(kind=kind, n=rng.choice([1, 2, 4, 8]), layers=layers, grad=rng.choice(["f32", "f32", "bf16"]),
             bits=rng.choice([32, 8]))
    if layers == "language":
        c.update(vocab=spread(500, 20_000), hidden=rng.randrange(60, 401, 2))
    elif layers == "mixed":
        c.update(lengths=rng.randrange(3, 60), longest=spread(2000, 1_000_000), pad=rng.choice([1, 4, 4]),
                 table=rng.randrange(1 << 30))
    return c


# ---- inputs -----------------------------------------------------------------------------------
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _tokens(c, gen):
    """Words by a law of 1 / rank, frequent ones all over the table; -1 where a sequence is padded."""
    shape = (c["n"], c["tokens"])
    rank = torch.rand(shape, device="cuda", generator=gen, dtype=torch.float64)
    word = ((c["vocab"] ** rank).long() - 1).clamp_(0, c["vocab"] - 1)
    word = (word * 7919) % c["vocab"]
    pad = torch.rand(shape, device="cuda", generator=gen) < c.get("padding", 0.0)
    return torch.where(pad, -1, word)


def _rows(n, d, align=64):
    return n, (d + align - 1) // align * align


def _embed_inputs(c, seed):
    """(tokens, buffer of the workers' rows, table or gradient slice of it, gradients of the looked-up rows)."""
    gen = _generator(seed)
    tokens = _tokens(c, gen)
    n, vocab, dim = c["n"], c["vocab"], c["dim"]
    kind = TYPES[c["table"]] if c["kind"] == "embed" else torch.float32
    rows = torch.empty(_rows(n, vocab * dim), device="cuda", dtype=kind).normal_(0.0, 0.05, generator=gen)
    table = rows[:, :vocab * dim].view(n, vocab, dim)
    dout = None
    if c["kind"] == "embed_grad":
        dout = torch.empty((n, c["tokens"], dim), device="cuda", dtype=TYPES[c["out"]]).normal_(0.0, 0.01, generator=gen)
    return tokens, rows, table, dout


def _recur_inputs(c, seed):
    """(f, u, o or None, h0, lengths or None, dy, dh of the last state): f, u and o are columns of one projection."""
    gen = _generator(seed)
    B, T, C = c["batch"], c["steps"], c["dim"]
    parts = 3 if c["gate"] else 2
    proj = torch.empty((B, T, parts * C), device="cuda", dtype=TYPES[c["type"]]).normal_(0.0, 1.0, generator=gen)
    f, u = proj[..., :C], proj[..., C:2 * C]
    f += 2.0        # gates that remember: about seven steps on average
    o = proj[..., 2 * C:] if c["gate"] else None
    h0 = torch.empty((B, C), device="cuda").normal_(0.0, 0.5, generator=gen)
    lengths = None
    if c.get("ragged"):
        lengths = torch.randint(T // 2, T + 1, (B,), device="cuda", generator=gen, dtype=torch.int32)
    dy = dh = None
    if c["kind"] == "recur_grad":
        dy = torch.empty((B, T, C), device="cuda", dtype=TYPES[c["type"]]).normal_(0.0, 1.0, generator=gen)
        dh = torch.empty((B, C), device="cuda").normal_(0.0, 1.0, generator=gen)
    return f, u, o, h0, lengths, dy, dh


@functools.lru_cache(maxsize=4)
def _layout(layers, lengths, longest, pad, table, vocab, hidden):
    """(start, length) of every tensor in a worker's row."""
    if layers == "image":       # a 20-layer residual network: weights, and a scale and a shift behind each
        out = []
        for cin, cout in [(3, 16)] + [(16, 16)] * 6 + [(16, 32)] + [(32, 32)] * 5 + [(32, 64)] + [(64, 64)] * 5:
            out += [9 * cin * cout, cout, cout]
        out += [16 * 32, 32, 32, 32 * 64, 64, 64, 640, 10]
    elif layers == "language":  # a tied embedding, three recurrent layers, an output bias
        out = [vocab * hidden]
        for _ in range(3):
            out += [4 * hidden * hidden, 4 * hidden * hidden, 4 * hidden, 4 * hidden]
        out += [vocab]
    else:                       # few long tensors among many short ones
        g = np.random.default_rng(table)
        out = np.maximum(1, longest * 10.0 ** (-4 * g.random(lengths))).astype(np.int64).tolist()
    start, at = [], 0
    for length in out:
        start.append(at)
        at = (at + length + pad - 1) // pad * pad
    return np.array(start, dtype=np.int64), np.array(out, dtype=np.int64)


def _tensors(c):
    return _layout(c["layers"], c.get("lengths", 0), c.get("longest", 0), c.get("pad", 4), c.get("table", 0),
                   c.get("vocab", 33278), c.get("hidden", 650))


def _decay(length):
    """Weight decay of each tensor: none on scales, shifts and biases."""
    return np.where(length >= 1000, DECAY, 0.0)


def _adamw_inputs(c, seed):
    """(X, G, how far each worker's gradient was clipped): the workers' parameter rows and gradients."""
    gen = _generator(seed)
    start, length = _tensors(c)
    shape = _rows(c["n"], int(start[-1] + length[-1]))
    X = torch.empty(shape, device="cuda").normal_(0.0, 0.05, generator=gen)
    G = torch.empty(shape, device="cuda", dtype=TYPES[c["grad"]]).normal_(0.0, 0.01, generator=gen)
    clip = torch.rand(c["n"], device="cuda", generator=gen) * 0.5 + 0.5
    return X, G, clip


def prepare(case, seed):
    c = case
    if c["kind"] in ("embed", "embed_grad"):
        tokens, rows, table, dout = _embed_inputs(c, seed)
        return dict(kind=c["kind"], case=c, tokens=tokens, rows=rows, table=table, dout=dout, scale=c["dim"] ** 0.5)
    if c["kind"] in ("recur", "recur_grad"):
        f, u, o, h0, lengths, dy, dh = _recur_inputs(c, seed)
        state = dict(kind=c["kind"], case=c, f=f, u=u, o=o, h0=h0, lengths=lengths, dy=dy, dh=dh)
        if own and c["kind"] == "recur_grad":    # what the forward pass kept
            from paper_1907_09356_amd import train
            state["saved"] = train.recurrence(f, u, o, h0=h0, lengths=lengths, save=True)[2]
        return state
    X, G, clip = _adamw_inputs(c, seed)
    start, length = _tensors(c)
    d = int(start[-1] + length[-1])
    state = dict(kind="adamw", case=c, X=X, G=G, clip=clip, d=d, seed=int(seed), t=0)
    if own:
        from paper_1907_09356_amd import train
        state["opt"] = train.AdamW(X, d, (start, length), weight_decay=_decay(length), betas=(BETA1, BETA2), eps=EPS,
                                   state_bits=c["bits"], seed=int(seed))
    else:
        state.update(_plain_optimiser(c, X, start, length, d))
    for _ in range(ELAPSED):
        _step(state)
    return state


# ---- one pass ---------------------------------------------------------------------------------
def run(state):
    kind = state["kind"]
    if kind == "embed":
        return _embed(state)
    if kind == "embed_grad":
        return _embed_grad(state)
    if kind == "recur":
        return _recur(state)
    if kind == "recur_grad":
        return _recur_grad(state)
    _step(state)
    return _parameters_and_moments(state)


def _embed(s):
    out = TYPES[s["case"]["out"]]
    if own:
        from paper_1907_09356_amd import train
        return train.embed(s["tokens"], s["table"], scale=s["scale"], out_dtype=out)
    tokens = s["tokens"]
    there = (tokens >= 0) & (tokens < s["table"].shape[1])
    worker = torch.arange(tokens.shape[0], device="cuda")[:, None]
    rows = s["table"][worker, torch.where(there, tokens, 0)].float() * s["scale"]
    return torch.where(there[..., None], rows, 0.0).to(out)


def _embed_grad(s):
    c = s["case"]
    add = c.get("add", False)
    if own:
        from paper_1907_09356_amd import train
        train.embed_grad(s["tokens"], s["dout"], s["table"], scale=s["scale"], accumulate=add)
        return s["table"]
    tokens, table = s["tokens"], s["table"]
    n, vocab, dim = table.shape
    there = (tokens >= 0) & (tokens < vocab)
    rows = torch.where(there[..., None], s["dout"].float() * s["scale"], 0.0)
    at = torch.arange(n, device="cuda")[:, None] * vocab + torch.where(there, tokens, 0)
    total = torch.zeros((n * vocab, dim), device="cuda")
    total.index_add_(0, at.reshape(-1), rows.reshape(-1, dim))
    table.copy_(table + total.view(table.shape) if add else total.view(table.shape))
    return table


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from zero, in doubling strides."""
    reach = 1
    while reach < a.shape[1]:
        b = torch.cat((b[:, :reach], b[:, reach:] + a[:, reach:] * b[:, :-reach]), 1)
        a = torch.cat((a[:, :reach], a[:, reach:] * a[:, :-reach]), 1)
        reach *= 2
    return b


def _sigmoid(x):
    return 1.0 / (1.0 + torch.exp(-x))


def _inside(s):
    """Which steps belong to their sequence, (batch, steps, 1)."""
    f, lengths = s["f"], s["lengths"]
    steps = torch.arange(f.shape[1], device="cuda")[None, :, None]
    return steps < (f.shape[1] if lengths is None else lengths[:, None, None])


def _states(s):
    """Gate, what enters, and the states of all steps; a step outside its sequence passes the state on."""
    f, u = s["f"].float(), s["u"].float()
    inside = _inside(s)
    a = torch.where(inside, _sigmoid(f), 1.0)
    b = torch.where(inside, _sigmoid(-f), 0.0) * u
    first = torch.cat((a[:, :1] * s["h0"][:, None] + b[:, :1], b[:, 1:]), 1)
    return a, b, _scan(a, first)


def _recur(s):
    if own:
        from paper_1907_09356_amd import train
        y, last, _ = train.recurrence(s["f"], s["u"], s["o"], h0=s["h0"], lengths=s["lengths"])
        return {"y": y, "h": last}
    h = _states(s)[2]
    y = h if s["o"] is None else h * _sigmoid(s["o"].float())
    y = torch.where(_inside(s), y, 0.0)
    return {"y": y.to(s["f"].dtype), "h": h[:, -1].clone()}


def _recur_grad(s):
    if own:
        from paper_1907_09356_amd import train
        df, du, do, dh0 = train.recurrence_grad(s["f"], s["u"], s["saved"], s["dy"], s["o"], lengths=s["lengths"],
                                                dlast=s["dh"])
        return {"df": df, "du": du, "dh0": dh0} if do is None else {"df": df, "du": du, "do": do, "dh0": dh0}
    a, _, h = _states(s)
    inside = _inside(s)
    f, u = s["f"].float(), s["u"].float()
    dy = torch.where(inside, s["dy"].float(), 0.0)
    gate = 1.0 if s["o"] is None else _sigmoid(s["o"].float())
    into = dy * gate                              # what reaches a state through its own output
    into = torch.cat((into[:, :-1], into[:, -1:] + s["dh"][:, None]), 1)
    after = torch.cat((a[:, 1:], torch.ones_like(a[:, :1])), 1)
    e = _scan(after.flip(1), into.flip(1)).flip(1)
    before = torch.cat((s["h0"][:, None], h[:, :-1]), 1)
    enter = torch.where(inside, _sigmoid(-f), 0.0)
    kind = s["f"].dtype
    out = {"df": (e * (before - u) * a * enter).to(kind), "du": (e * enter).to(kind), "dh0": a[:, 0] * e[:, 0]}
    if s["o"] is not None:
        out["do"] = (dy * h * gate * _sigmoid(-s["o"].float())).to(kind)
    return out


# ---- AdamW ------------------------------------------------------------------------------------
def _plain_optimiser(c, X, start, length, d):
    """The plain form's state: moments, which tensor's decay an entry takes, and in which block it lies."""
    n = X.shape[0]
    index = np.repeat(np.arange(len(length)), length)
    at = np.arange(len(index)) - np.repeat(np.cumsum(length) - length, length)      # place in its tensor
    where = np.repeat(start, length) + at                                            # place in the row
    out = dict(where=torch.from_numpy(where).cuda(), decay=torch.from_numpy(_decay(length)[index].astype(np.float32)).cuda())
    if c["bits"] == 32:
        out.update(m=torch.zeros((n, len(where)), device="cuda"), v=torch.zeros((n, len(where)), device="cuda"))
        return out
    blocks = (length + BLOCK - 1) // BLOCK
    block = (np.cumsum(blocks) - blocks)[index] + at // BLOCK
    out.update(block=torch.from_numpy(block).cuda(), blocks=int(blocks.sum()))
    for name in ("m", "v"):
        out[name] = torch.zeros((n, len(where)), device="cuda", dtype=torch.int16)
        out[name + "_scale"] = torch.zeros((n, int(blocks.sum())), device="cuda")
    return out


def _step(s):
    s["t"] += 1
    if "opt" in s:
        s["opt"].step(s["G"], LR, grad_scale=s["clip"])
        return
    c, t, where = s["case"], s["t"], s["where"]
    g = s["G"][:, where].float() * s["clip"][:, None]
    m, v = _moments(s)
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + (g * g) * (1 - BETA2)
    X = s["X"]
    p = X[:, where]
    step = m * (LR / (1 - BETA1 ** t)) / (v.sqrt() * (1 / (1 - BETA2 ** t) ** 0.5) + EPS)
    X[:, where] = p * (1 - LR * s["decay"]) - step
    if c["bits"] == 32:
        s["m"], s["v"] = m, v
        return
    words = _words(s["d"], X.shape[0], t - 1, 3, s["seed"])[:, where]
    s["m"], s["m_scale"] = _held(s, m, words & 0xFFFF, 15)
    s["v"], s["v_scale"] = _held(s, v, words >> 16, 31)
    s["v"] = torch.where((v > 0) & (s["v"] == 0), 1, s["v"])      # what is positive is not held as zero


def _held(s, x, r, top):
    """`x` in 8 bits: relative to the power of two that brings a block's largest into (0.9375, 1.875], 3 bits follow the
    leading one of a float with exponents from 0 to `top`, and the rest is rounded up with the probability r / 65536
    says.  (codes with the sign of x, scales)"""
    block = s["block"]
    most = torch.zeros((x.shape[0], s["blocks"]), device="cuda").scatter_reduce_(1, block.expand(x.shape), x.abs(), "amax")
    bits = most.view(torch.int32)
    power = (bits & 0x7F800000) + torch.where((bits & 0x7FFFFF) > 0x700000, 1 << 23, 0).int()
    up = ((254 << 23) - power).view(torch.float32)
    y = x.abs() * up[:, block]
    low = y * 2.0 ** (top - 127)                  # exponents below the format's come out as denormal numbers
    bits = low.view(torch.int32) + (r << 4).int()
    code = torch.clamp(bits >> 20, max=8 * top + 7).short()
    return torch.where(x < 0, -code, code), power.view(torch.float32)


def _value(code, top):
    """What a code of _held stands for, relative to its block's scale: at most 1.875."""
    size = (code.abs().int() << 20).view(torch.float32) * 2.0 ** (127 - top)
    return torch.where(code < 0, -size, size)


def _moments(s):
    if s["case"]["bits"] == 32:
        return s["m"], s["v"]
    return _value(s["m"], 15) * s["m_scale"][:, s["block"]], _value(s["v"], 31) * s["v_scale"][:, s["block"]]


def _parameters_and_moments(s):
    d = s["d"]
    if "opt" in s:
        m, v = s["opt"].moments()
        return {"x": s["X"][:, :d], "m": m, "v": v}
    out = {"x": s["X"][:, :d]}
    for name, x in zip(("m", "v"), _moments(s)):
        out[name] = torch.zeros((x.shape[0], d), device="cuda")
        out[name][:, s["where"]] = x
    return out


def _words(d, n, t, stream, seed):
    """Philox4x32-10 (Salmon et al., SC'11), one 32-bit word per entry: (n, d) of int64."""
    keep = 0xFFFFFFFF
    c0 = torch.arange((d + 3) // 4, device="cuda")[None].expand(n, -1)
    c1 = torch.arange(n, device="cuda")[:, None].expand(c0.shape)
    c2, c3 = torch.full_like(c0, t & keep), torch.full_like(c0, stream | (t >> 32 << 8))
    k0, k1 = seed & keep, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57     # 64-bit products, their sign bit a bit like any other
        c0, c1, c2, c3 = ((p1 >> 32) & keep) ^ c1 ^ k0, p1 & keep, ((p0 >> 32) & keep) ^ c3 ^ k1, p0 & keep
        k0, k1 = (k0 + 0x9E3779B9) & keep, (k1 + 0xBB67AE85) & keep
    return torch.stack((c0, c1, c2, c3), 2).reshape(n, -1)[:, :d]


# ---- what a pass cannot do without ------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] in ("embed", "embed_grad"):
        looked_up = c["n"] * c["tokens"] * c["dim"] * (1 - c.get("padding", 0.0))
        words, size = 8 * c["n"] * c["tokens"], BYTES[c["out"]]
        # of the looked-up rows, those that differ: words drawn by rank, counted as the expected number
        rank = np.log1p(1.0 / np.arange(1, c["vocab"] + 1)) / np.log(c["vocab"] + 1)
        there = c["tokens"] * (1 - c.get("padding", 0.0))
        distinct = float(c["n"] * np.sum(1 - (1 - rank) ** there)) * c["dim"]
        if c["kind"] == "embed":
            return {"bytes": words + distinct * BYTES[c["table"]] + c["n"] * c["tokens"] * c["dim"] * size, "flops": looked_up}
        table = 8 * distinct if c.get("add") else 4 * c["n"] * c["vocab"] * c["dim"]
        return {"bytes": words + looked_up * size + table, "flops": 2 * looked_up}
    if c["kind"] in ("recur", "recur_grad"):
        entries = c["batch"] * c["steps"] * c["dim"] * (0.75 if c.get("ragged") else 1.0)
        whole = c["batch"] * c["steps"] * c["dim"]          # outputs are zero outside a sequence
        ends, gates = 8 * c["batch"] * c["dim"], 3 if c["gate"] else 2
        size = BYTES[c["type"]]
        if c["kind"] == "recur":
            return {"bytes": size * (gates * entries + whole) + ends, "flops": 10 * entries}
        return {"bytes": size * ((gates + 1) * entries + gates * whole) + ends, "flops": 25 * entries}
    start, length = _tensors(c)
    entries, size = c["n"] * int(length.sum()), BYTES[c["grad"]]
    if c["bits"] == 32:     # x, m and v in and out, g in
        return {"bytes": (24 + size) * entries, "flops": 15 * entries}
    # the moments one byte each with a scale per block; then written once more as the values they stand for
    scales = 16 * c["n"] * int(((length + BLOCK - 1) // BLOCK).sum())
    return {"bytes": (8 + size + 4 + 8) * entries + scales, "flops": 60 * entries}


# ---- the definitions in 64 bits ---------------------------------------------------------------
def exact(case, seed):
    return {"embed": _exact_embed, "embed_grad": _exact_embed_grad, "recur": _exact_recur, "recur_grad": _exact_recur_grad,
            "adamw": _exact_adamw}[case["kind"]](case, seed)


def _exact_embed(c, seed):
    tokens, _, table, _ = _embed_inputs(c, seed)
    y = torch.zeros((c["n"], c["tokens"], c["dim"]), device="cuda", dtype=torch.float64)
    for w in range(c["n"]):
        there = torch.nonzero(tokens[w] >= 0)[:, 0]
        y[w, there] = table[w].index_select(0, tokens[w, there]).double() * c["dim"] ** 0.5
    return y


def _exact_embed_grad(c, seed):
    tokens, _, table, dout = _embed_inputs(c, seed)
    total = table.double() if c.get("add") else torch.zeros(table.shape, device="cuda", dtype=torch.float64)
    for w in range(c["n"]):
        order = torch.argsort(tokens[w])            # one word after the other, padding first
        word, count = torch.unique_consecutive(tokens[w, order], return_counts=True)
        sums = torch.cat((torch.zeros((1, c["dim"]), device="cuda", dtype=torch.float64),
                          (dout[w, order].double() * c["dim"] ** 0.5).cumsum(0)))
        ends = count.cumsum(0)
        real = word >= 0
        total[w, word[real]] += (sums[ends] - sums[ends - count])[real]
    return total


def _exact_states(c, seed):
    """Step by step: yields (step, inputs in 64 bits, state before, state after, which sequences the step is in)."""
    f, u, o, h, lengths, _, _ = _recur_inputs(c, seed)
    h = h.double()
    for t in range(c["steps"]):
        inside = torch.ones((c["batch"], 1), device="cuda", dtype=torch.bool) if lengths is None else (t < lengths)[:, None]
        a = torch.sigmoid(f[:, t].double())
        new = torch.where(inside, a * h + (1 - a) * u[:, t].double(), h)
        yield t, a, u[:, t].double(), None if o is None else torch.sigmoid(o[:, t].double()), h, new, inside
        h = new


def _exact_recur(c, seed):
    y = torch.zeros((c["batch"], c["steps"], c["dim"]), device="cuda", dtype=torch.float64)
    for t, _, _, s, _, h, inside in _exact_states(c, seed):
        y[:, t] = torch.where(inside, h if s is None else s * h, 0.0)
    return {"y": y, "h": h}


def _exact_recur_grad(c, seed):
    f, u, o, h0, lengths, dy, dh = _recur_inputs(c, seed)
    shape = (c["batch"], c["steps"], c["dim"])
    before = torch.empty(shape, device="cuda", dtype=torch.float64)
    for t, _, _, _, h, _, _ in _exact_states(c, seed):
        before[:, t] = h
    out = {name: torch.zeros(shape, device="cuda", dtype=torch.float64) for name in (("df", "du") if o is None else ("df", "du", "do"))}
    e = dh.double()
    for t in reversed(range(c["steps"])):
        inside = torch.ones((c["batch"], 1), device="cuda", dtype=torch.bool) if lengths is None else (t < lengths)[:, None]
        a, x, d = torch.sigmoid(f[:, t].double()), u[:, t].double(), dy[:, t].double()
        here = e + d
        if o is not None:
            s = torch.sigmoid(o[:, t].double())
            here = e + d * s
            out["do"][:, t] = torch.where(inside, d * (a * before[:, t] + (1 - a) * x) * s * (1 - s), 0.0)
        out["df"][:, t] = torch.where(inside, here * (before[:, t] - x) * a * (1 - a), 0.0)
        out["du"][:, t] = torch.where(inside, here * (1 - a), 0.0)
        e = torch.where(inside, here * a, e)
    return {**out, "dh0": e}


def _exact_adamw(c, seed):
    X, G, clip = _adamw_inputs(c, seed)
    start, length = _tensors(c)
    d = int(start[-1] + length[-1])
    out = {"x": X[:, :d].double(), "m": torch.zeros((c["n"], d), device="cuda", dtype=torch.float64)}
    out["v"] = torch.zeros_like(out["m"])
    for t in range(1, ELAPSED + 2):
        words = _words(d, c["n"], t - 1, 3, int(seed)) if c["bits"] == 8 else None
        for at, long, decay in zip(start.tolist(), length.tolist(), _decay(length).tolist()):
            for first in range(at, at + long, 1 << 22):      # in pieces of whole blocks
                p = slice(first, min(first + (1 << 22), at + long))
                x, m, v = (out[k][:, p] for k in ("x", "m", "v"))
                g = G[:, p].double() * clip.double()[:, None]
                m.mul_(BETA1).add_((1 - BETA1) * g)
                v.mul_(BETA2).add_((1 - BETA2) * g * g)
                x.sub_(LR * (m / (1 - BETA1 ** t) / ((v / (1 - BETA2 ** t)).sqrt() + EPS) + decay * x))
                if c["bits"] == 8:
                    m.copy_(_exact_held(m, (words[:, p] & 0xFFFF).double() / 65536, 4))
                    v.copy_(_exact_held(v, (words[:, p] >> 16).double() / 65536, 5))
    return out


def _exact_held(x, r, exponent_bits):
    """`x` as 8 bits hold it: a float of 3 mantissa and so many exponent bits with gradual underflow, relative to a power of
    two (the block's largest: above a half of 1.875, at most that), rounded up where its distance to the next lower
    one and r add up to a whole step."""
    n, long = x.shape
    whole = -(-long // BLOCK) * BLOCK
    y = torch.nn.functional.pad(x.abs(), (0, whole - long)).view(n, -1, BLOCK)
    most = y.amax(2, keepdim=True)
    share, exponent = torch.frexp(most / 1.875)      # share in [0.5, 1), exactly 0.5 for a power of two
    scale = torch.where(share > 0.5, torch.exp2(exponent.double()), torch.exp2(exponent.double() - 1))
    y = (y / scale).view(n, -1)[:, :long]
    exponent = torch.frexp(y)[1].sub(1).clamp(min=2 - 2 ** exponent_bits).double()
    step = torch.exp2(exponent - 3)
    size = torch.floor(y / step + r) * step
    if exponent_bits == 5:
        size = torch.where((y > 0) & (size == 0), step, size)
    back = size.clamp(max=1.875) * scale.expand(n, -1, BLOCK).reshape(n, -1)[:, :long]
    return torch.where(x < 0, -back, back)
