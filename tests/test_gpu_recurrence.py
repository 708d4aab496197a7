"""The gated linear recurrence and its backward pass against a step-by-step computation in 64 bits.

Tolerances follow the computation.  A gate is good to g(x) = (8 + 2 |x|) 2^-24 relative to itself (its exponential's argument is
rounded, then three operations).  Along the steps the error of a state obeys
  bh_t = a bh_{t-1} + (g + 2^-22) (a |h_{t-1}| + (1 - a) |u_t|)
(2^-22: the step's own roundings); a state that is put together from the states of pieces has every product a ... a
rounded on the way, which counts as errors of the same size once more: a factor of 3 on the whole.  The same holds for e_t
going back.  A result adds its own factors' errors and the rounding to its type."""
import numpy as np
import pytest
import torch

from paper_1907_09356_amd import binding as B
from paper_1907_09356_amd import train as T

pytestmark = pytest.mark.gpu
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}


def sigmoid(x):
    return 1 / (1 + np.exp(-x))


def gate_error(x):
    return (8 + 2 * np.abs(x)) * 2.0 ** -24


def forward(f, u, o, h0, lengths):
    """y, last states, all states (index 0: before the first step) and their error bounds, in 64 bits."""
    B_, S, C = f.shape
    h, bh = h0.copy(), np.zeros_like(h0)
    H, BH = [h], [bh]
    y, by = np.zeros_like(f), np.zeros_like(f)
    for t in range(S):
        on = (t < lengths)[:, None]
        a, i = sigmoid(f[:, t]), sigmoid(-f[:, t])
        new = a * h + i * u[:, t]
        bnew = a * bh + (gate_error(f[:, t]) + 2.0 ** -22) * (a * np.abs(h) + i * np.abs(u[:, t]))
        h, bh = np.where(on, new, h), np.where(on, bnew, bh)
        s = 1.0 if o is None else sigmoid(o[:, t])
        r = 2.0 ** -23 if o is None else gate_error(o[:, t]) + 2.0 ** -23
        y[:, t] = np.where(on, s * h, 0.0)
        by[:, t] = np.where(on, s * (3 * bh + r * np.abs(h)), 0.0)
        H.append(h)
        BH.append(bh)
    return y, by, h, 3 * bh, H, [3 * b for b in BH]


def backward(f, u, o, lengths, H, BH, dy, dlast):
    out = {k: np.zeros_like(f) for k in ("df", "du", "do", "bdf", "bdu", "bdo")}
    e, be = dlast.copy(), np.zeros_like(dlast)
    for t in reversed(range(f.shape[1])):
        on = (t < lengths)[:, None]
        a, i = sigmoid(f[:, t]), sigmoid(-f[:, t])
        ga, d = gate_error(f[:, t]) + 2.0 ** -22, dy[:, t]
        s = 1.0 if o is None else sigmoid(o[:, t])
        gs = 0.0 if o is None else gate_error(o[:, t])
        here = e + d * s
        bhere = be + (gs + 2.0 ** -22) * np.abs(d * s) + 2.0 ** -23 * np.abs(e)
        diff = H[t] - u[:, t]
        for name, value, bound in (
                ("df", here * diff * a * i, (3 * bhere * np.abs(diff) + np.abs(here) * (BH[t] + 2.0 ** -23 * (np.abs(H[t]) + np.abs(u[:, t])))) * a * i
                 + 3 * ga * np.abs(here * diff) * a * i),
                ("du", here * i, 3 * bhere * i + ga * np.abs(here) * i),
                ("do", d * H[t + 1] * s * (1 - s) if o is not None else 0.0 * d,
                 np.abs(d) * (BH[t + 1] + (2 * gs + 2.0 ** -22) * np.abs(H[t + 1])) * s * (1 - s))):
            out[name][:, t] = np.where(on, value, 0.0)
            out["b" + name][:, t] = np.where(on, bound, 0.0)
        e = np.where(on, a * here, e)
        be = np.where(on, a * bhere + ga * np.abs(a * here), be)
    out["dh0"], out["bdh0"] = e, 3 * be
    return out


def check(name, got, want, bound, dtype):
    err = np.abs(got.double().cpu().numpy() - want)
    bound = bound + HALF_ULP[dtype] * (np.abs(want) + bound) + TINY[dtype]
    worst = np.max(err - bound) if err.size else 0.0
    assert worst <= 0, (name, float(worst), float(np.max(err)))


def inputs(batch, steps, dim, dtype, gated, seed, spread=1.5, shift=1.0):
    g = np.random.default_rng(seed)
    parts = 3 if gated else 2
    proj = torch.from_numpy((g.standard_normal((batch, steps, parts * dim)) * spread).astype(np.float32)).to(dtype)
    proj[..., :dim] += shift
    f, u = proj[..., :dim], proj[..., dim:2 * dim]
    o = proj[..., 2 * dim:] if gated else None
    h0 = torch.from_numpy(g.standard_normal((batch, dim)).astype(np.float32))
    dy = torch.from_numpy(g.standard_normal((batch, steps, dim)).astype(np.float32)).to(dtype)
    dlast = torch.from_numpy(g.standard_normal((batch, dim)).astype(np.float32))
    return proj, f, u, o, h0, dy, dlast


def d64(t):
    return None if t is None else t.double().numpy()


def both(batch, steps, dim, dtype, gated, lengths, seed, state=True, **kw):
    proj, f, u, o, h0, dy, dlast = inputs(batch, steps, dim, dtype, gated, seed, **kw)
    if not state:
        h0, dlast = torch.zeros_like(h0), torch.zeros_like(dlast)
    on = np.full(batch, steps) if lengths is None else np.clip(np.asarray(lengths), 0, steps)
    p = proj.cuda()
    cf, cu, co = p[..., :dim], p[..., dim:2 * dim], p[..., 2 * dim:] if gated else None
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    y, last, saved = T.recurrence(cf, cu, co, h0=h0.cuda() if state else None, lengths=ln, save=True)
    wy, by, wl, bl, H, BH = forward(d64(f), d64(u), d64(o), d64(h0), on)
    check("y", y, wy, by, dtype)
    check("h", last, wl, bl, torch.float32)
    for k in range(saved.shape[0]):
        check("saved", saved[k], H[T.SAVE_STEPS * k], BH[T.SAVE_STEPS * k], torch.float32)
    # without `saved` the same bits
    y2, last2, none = T.recurrence(cf, cu, co, h0=h0.cuda() if state else None, lengths=ln)
    assert none is None and torch.equal(y2, y) and torch.equal(last2, last)
    df, du, do, dh0 = T.recurrence_grad(cf, cu, saved, dy.cuda(), co, lengths=ln, dlast=dlast.cuda() if state else None)
    want = backward(d64(f), d64(u), d64(o), on, H, BH, d64(dy), d64(dlast))
    check("df", df, want["df"], want["bdf"], dtype)
    check("du", du, want["du"], want["bdu"], dtype)
    check("dh0", dh0, want["dh0"], want["bdh0"], torch.float32)
    assert (do is None) == (not gated)
    if gated:
        check("do", do, want["do"], want["bdo"], dtype)


SHAPES = [(1, 1, 1), (3, 1, 650), (2, 2, 64), (1, 15, 33), (2, 16, 128), (3, 17, 65), (1, 31, 2), (2, 35, 650), (1, 128, 100),
          (2, 129, 257), (1, 300, 512), (5, 257, 40), (1, 2051, 66), (2, 1024, 300), (1, 5003, 34), (70, 40, 9)]


@pytest.mark.parametrize("batch,steps,dim", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("gated", [True, False])
def test_against_64_bits(batch, steps, dim, dtype, gated):
    both(batch, steps, dim, dtype, gated, None, seed=steps + dim)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("lengths", [[0, 0, 0, 0], [0, 1, 16, 17], [300, 5, 299, 0], [-3, 1000, 32, 31], [255, 256, 257, 1]])
def test_ragged_batches(dtype, gated, lengths):
    both(4, 300, 70, dtype, gated, lengths, seed=21)
    both(4, 300, 128, dtype, gated, lengths, seed=22, state=False)


def test_ragged_long_sequences():
    both(3, 4200, 64, torch.float32, True, [4200, 0, 2113], seed=23)
    both(2, 4200, 130, torch.bfloat16, False, [17, 4100], seed=24)


@pytest.mark.parametrize("shift", [-60.0, -8.0, 8.0, 60.0])
def test_gates_at_their_ends(shift):
    # gates that forget everything, or keep a state over thousands of steps
    both(2, 1100, 72, torch.float32, True, None, seed=25, shift=shift, spread=1.0)
    both(2, 200, 72, torch.float16, False, [200, 77], seed=26, shift=shift, spread=1.0)


def test_gates_to_the_last_places():
    # one step with dy = 1: du is 1 - sigmoid(f), dh0 sigmoid(f), and y = sigmoid(o) h0 where the state is kept.  An exponential good
    # to 4 2^-24 (its instruction 2, two roundings), a sum, a reciprocal (2), a product or difference: 10, one more for the second order
    size = np.concatenate((np.linspace(-86, 86, 20_000), np.random.default_rng(1).standard_normal(20_000) * 4)).astype(np.float32)
    x = torch.from_numpy(size).cuda().view(4, 1, -1)
    zero, one = torch.zeros_like(x), torch.ones_like(x)
    h0 = one[:, 0].contiguous()
    y = T.recurrence(torch.full_like(x, 120.0), zero, x, h0=h0)[0]
    saved = T.recurrence(x, zero, h0=h0, save=True)[2]
    _, du, _, dh0 = T.recurrence_grad(x, zero, saved, one)
    at = size.astype(np.float64)
    for got, want in ((y, sigmoid(at)), (dh0, sigmoid(at)), (du, sigmoid(-at))):
        assert np.max(np.abs(got.double().cpu().numpy().ravel() / want - 1)) <= 11 * 2.0 ** -24


@pytest.mark.parametrize("steps", [37, 700])
def test_infinite_gates_and_masked_steps(steps):
    # f = +-inf: keep, or take the input; NaN and infinities beyond a sequence's end are not looked at
    f = torch.zeros((2, steps, 80))
    f[:, ::2], f[:, 1::2] = float("inf"), float("-inf")
    u = torch.from_numpy(np.random.default_rng(1).standard_normal((2, steps, 80)).astype(np.float32))
    o = torch.full((2, steps, 80), float("inf"))
    short = steps - 5
    for x in (f, u, o):
        x[1, short:] = float("nan")
    f[1, -1] = float("inf")
    lengths = torch.tensor([steps, short], dtype=torch.int32).cuda()
    y, last, saved = T.recurrence(f.cuda(), u.cuda(), o.cuda(), lengths=lengths, save=True)
    want = torch.zeros((2, steps, 80))
    for t in range(steps):
        want[:, t] = u[:, t] if t % 2 else (want[:, t - 1] if t else 0.0)
    last_want = torch.stack((want[0, -1], want[1, short - 1]))
    want[1, short:] = 0.0
    assert torch.equal(y.cpu(), want) and torch.equal(last.cpu(), last_want)
    dy = torch.ones((2, steps, 80))
    dy[1, short:] = float("nan")
    df, du, do, dh0 = T.recurrence_grad(f.cuda(), u.cuda(), saved, dy.cuda(), o.cuda(), lengths=lengths)
    assert bool((df == 0).all()) and bool((do == 0).all())
    assert du[0, 1::2].min() >= 1 and bool((du[:, ::2] == 0).all()) and bool((du[1, short:] == 0).all())
    assert bool((dh0 == 1).all())       # kept over the first step, overwritten in the second


def test_a_nan_gate_reaches_its_channel_only():
    f = torch.zeros((1, 60, 64)).cuda()
    f[0, 20, 5] = float("nan")
    u = torch.ones((1, 60, 64)).cuda()
    y, last, _ = T.recurrence(f, u)
    assert bool(torch.isnan(y[0, 20:, 5]).all()) and int(torch.isnan(y).sum()) == 40 and int(torch.isnan(last).sum()) == 1


def test_gradient_by_differences():
    # central differences of the 64-bit forward pass, h = 1e-5: their own error is of the order of h^2 and 1e-16 / h, below 1e-9
    # relative to the loss's size; the kernel's bound is the one above
    batch, steps, dim = 2, 21, 3
    lengths = np.array([21, 18])
    proj, f, u, o, h0, dy, dlast = inputs(batch, steps, dim, torch.float32, True, 31)
    p = proj.cuda()
    cf, cu, co = p[..., :dim], p[..., dim:2 * dim], p[..., 2 * dim:]
    ln = torch.from_numpy(lengths.astype(np.int32)).cuda()
    saved = T.recurrence(cf, cu, co, h0=h0.cuda(), lengths=ln, save=True)[2]
    df, du, do, dh0 = T.recurrence_grad(cf, cu, saved, dy.cuda(), co, lengths=ln, dlast=dlast.cuda())
    x = {"f": d64(f), "u": d64(u), "o": d64(o), "h0": d64(h0)}

    def loss(**moved):
        v = {**x, **moved}
        y, _, last, _, _, _ = forward(v["f"], v["u"], v["o"], v["h0"], lengths)
        return float((y * d64(dy)).sum() + (last * d64(dlast)).sum())

    _, _, _, _, H, BH = forward(x["f"], x["u"], x["o"], x["h0"], lengths)
    bounds = backward(x["f"], x["u"], x["o"], lengths, H, BH, d64(dy), d64(dlast))
    g = np.random.default_rng(5)
    for name, got in (("f", df), ("u", du), ("o", do), ("h0", dh0)):
        got = got.double().cpu().numpy()
        for _ in range(40):
            at = tuple(int(g.integers(0, m)) for m in got.shape)
            sides = []
            for step in (1e-5, -1e-5):
                moved = x[name].copy()
                moved[at] += step
                sides.append(loss(**{name: moved}))
            quotient = (sides[0] - sides[1]) / 2e-5
            assert abs(quotient - got[at]) <= bounds["bd" + name][at] + 2.0 ** -24 * abs(quotient) + 1e-8, (name, at)


def test_token_by_token_is_the_whole_sequence():
    batch, steps, dim = 5, 40, 650
    proj, f, u, o, h0, _, _ = inputs(batch, steps, dim, torch.bfloat16, True, 41)
    f, u, o = f.cuda(), u.cuda(), o.cuda()
    state = h0.cuda()
    rows = []
    for t in range(steps):      # in place: the state's buffer is read and written
        y, last, _ = T.recurrence(f[:, t:t + 1], u[:, t:t + 1], o[:, t:t + 1], h0=state, h_last=state)
        assert last is state
        rows.append(y)
    wy, by, wl, bl, _, _ = forward(d64(f.cpu()), d64(u.cpu()), d64(o.cpu()), d64(h0), np.full(batch, steps))
    check("y", torch.cat(rows, 1), wy, by, torch.bfloat16)
    check("h", state, wl, bl, torch.float32)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 2, 3])
def test_layouts(dtype, offset):
    # steps before sequences, columns that start anywhere, steps of odd width
    batch, steps, dim = 3, 50, 66
    g = np.random.default_rng(51)
    width = 3 * dim + 5
    base = torch.from_numpy(g.standard_normal((steps, batch, width)).astype(np.float32)).to(dtype).cuda()
    f, u, o = (base[..., offset + k * dim:offset + (k + 1) * dim].transpose(0, 1) for k in range(3))
    out = torch.full((steps, batch, dim + 3), 9.0, dtype=dtype, device="cuda")
    y, last, saved = T.recurrence(f, u, o, save=True, out=out[..., offset:offset + dim].transpose(0, 1))
    plain = [t.contiguous() for t in (f, u, o)]
    y2, last2, saved2 = T.recurrence(*plain, save=True)
    assert torch.equal(y, y2) and torch.equal(last, last2) and torch.equal(saved, saved2)
    assert bool((out[..., :offset] == 9).all()) and bool((out[..., offset + dim:] == 9).all())
    dy = torch.from_numpy(g.standard_normal((steps, batch, dim + 3)).astype(np.float32)).to(dtype).cuda()
    view = dy[..., offset:offset + dim].transpose(0, 1)
    for a, b in zip(T.recurrence_grad(f, u, saved, view, o), T.recurrence_grad(*plain[:2], saved2, view.contiguous(), plain[2])):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1, 2])
def test_layouts_of_long_sequences(dtype, offset):
    # the same for sequences of several tiles: steps before sequences, columns that start anywhere, ragged
    batch, steps, dim = 3, 2100, 66
    gen = torch.Generator(device="cuda").manual_seed(54)
    base = torch.empty((steps, batch, 3 * dim + 5), device="cuda", dtype=dtype).normal_(generator=gen)
    f, u, o = (base[..., offset + k * dim:offset + (k + 1) * dim].transpose(0, 1) for k in range(3))
    lengths = torch.tensor([2100, 129, 1937], dtype=torch.int32).cuda()
    h0 = torch.empty((batch, dim), device="cuda").normal_(generator=gen)
    out = torch.full((steps, batch, dim + 3), 9.0, dtype=dtype, device="cuda")
    y, last, saved = T.recurrence(f, u, o, h0=h0, lengths=lengths, save=True, out=out[..., offset:offset + dim].transpose(0, 1))
    plain = [t.float().contiguous().double().cpu().numpy() for t in (f, u, o, h0)]
    wy, by, wl, bl, H, BH = forward(*plain, lengths.cpu().numpy())
    check("y", y, wy, by, dtype)
    check("h", last, wl, bl, torch.float32)
    assert bool((out[..., :offset] == 9).all()) and bool((out[..., offset + dim:] == 9).all())
    dy = torch.empty((steps, batch, dim + 3), device="cuda", dtype=dtype).normal_(generator=gen)
    view = dy[..., offset:offset + dim].transpose(0, 1)
    df, du, do, dh0 = T.recurrence_grad(f, u, saved, view, o, lengths=lengths)
    want = backward(plain[0], plain[1], plain[2], lengths.cpu().numpy(), H, BH, view.double().cpu().numpy(), np.zeros((batch, dim)))
    for name, got in (("df", df), ("du", du), ("do", do)):
        check(name, got, want[name], want["b" + name], dtype)
    check("dh0", dh0, want["dh0"], want["bdh0"], torch.float32)


@pytest.mark.parametrize("steps,dim", [(100, 130), (129, 130), (2500, 66)])
def test_the_last_state_in_place_of_the_first(steps, dim):
    proj, f, u, o, h0, _, _ = inputs(3, steps, dim, torch.float32, True, 42)
    f, u, o, state = f.cuda(), u.cuda(), o.cuda(), h0.cuda()
    y, last, _ = T.recurrence(f, u, o, h0=state)
    y2, last2, _ = T.recurrence(f, u, o, h0=state, h_last=state)
    assert last2 is state and torch.equal(y, y2) and torch.equal(last, state)


@pytest.mark.parametrize("steps", [90, 1500])
def test_infinite_states_stay_in_their_channel_from_their_step_on(steps):
    # from h0, or from an input on: not finite to the end (infinite, or NaN where what is left of the state is below fp32's range)
    for start in (0, 3, steps // 2):
        f = torch.randn((2, steps, 70), device="cuda")
        u = torch.randn((2, steps, 70), device="cuda")
        h0 = torch.zeros((2, 70), device="cuda")
        if start == 0:
            h0[1, 4] = float("inf")
        else:
            u[1, start, 4] = float("-inf")
        y, last, saved = T.recurrence(f, u, h0=h0, save=True)
        hit = torch.zeros((2, steps, 70), dtype=torch.bool, device="cuda")
        hit[1, start:, 4] = True
        assert torch.equal(~torch.isfinite(y), hit)
        assert torch.equal(~torch.isfinite(last), hit[:, -1])
        df, du, _, dh0 = T.recurrence_grad(f, u, saved, torch.ones_like(f))
        hit[1, :, 4] = True
        assert bool(torch.isfinite(df[~hit]).all()) and bool(torch.isfinite(du).all()) and bool(torch.isfinite(dh0).all())


def test_one_gate_for_all_steps():
    # inputs may repeat: a stride of zero
    batch, steps, dim = 2, 45, 96
    g = np.random.default_rng(52)
    f = torch.from_numpy(g.standard_normal((batch, 1, dim)).astype(np.float32)).cuda().expand(batch, steps, dim)
    u = torch.from_numpy(g.standard_normal((batch, steps, dim)).astype(np.float32)).cuda()
    y, last, _ = T.recurrence(f, u)
    y2, last2, _ = T.recurrence(f.contiguous(), u)
    assert torch.equal(y, y2) and torch.equal(last, last2)


def test_strides_of_more_than_32_bits():
    batch, steps, dim = 2, 6, 64
    step = 1 << 29
    base = torch.zeros((batch - 1) * 1000 + (steps - 1) * step + dim, dtype=torch.bfloat16, device="cuda")
    f = base.as_strided((batch, steps, dim), (1000, step, 1))
    f.copy_(torch.from_numpy(np.random.default_rng(53).standard_normal((batch, steps, dim)).astype(np.float32)))
    u = torch.ones((batch, steps, dim), dtype=torch.bfloat16, device="cuda")
    y, last, saved = T.recurrence(f, u, save=True)
    y2, last2, saved2 = T.recurrence(f.contiguous(), u, save=True)
    assert torch.equal(y, y2) and torch.equal(last, last2)
    for a, b in zip(T.recurrence_grad(f, u, saved, f), T.recurrence_grad(f.contiguous(), u, saved2, f.contiguous())):
        assert a is None and b is None or torch.equal(a, b)


def test_many_sequences():
    batch = 70_000      # more than a grid's second dimension holds
    f = torch.randn((batch, 2, 3), device="cuda")
    u = torch.randn((batch, 2, 3), device="cuda")
    y, last, saved = T.recurrence(f, u, save=True)
    wy, by, wl, bl, H, BH = forward(d64(f.cpu()), d64(u.cpu()), None, np.zeros((batch, 3)), np.full(batch, 2))
    check("y", y, wy, by, torch.float32)
    df, du, _, dh0 = T.recurrence_grad(f, u, saved, u)
    want = backward(d64(f.cpu()), d64(u.cpu()), None, np.full(batch, 2), H, BH, d64(u.cpu()), np.zeros((batch, 3)))
    check("df", df, want["df"], want["bdf"], torch.float32)
    check("dh0", dh0, want["dh0"], want["bdh0"], torch.float32)


@pytest.mark.parametrize("dtype,batch", [(torch.float32, 40), (torch.bfloat16, 44), (torch.bfloat16, 120)])
@pytest.mark.parametrize("gated", [True, False])
def test_results_that_do_not_fit_the_caches(dtype, batch, gated):
    # more than 128 and more than 384 MB are written, and read, past the caches: the same bits as a few sequences at a time
    steps, dim, few = 700, 770, 4
    gen = torch.Generator(device="cuda").manual_seed(batch)
    proj = torch.empty((batch, steps, 3 * dim), device="cuda", dtype=dtype).normal_(generator=gen)
    f, u, o = proj.split(dim, 2)
    o = o if gated else None
    dy = torch.empty((batch, steps, dim), device="cuda", dtype=dtype).normal_(generator=gen)
    y, last, saved = T.recurrence(f, u, o, save=True)
    grads = T.recurrence_grad(f, u, saved, dy, o)
    for b in range(0, batch, few):
        p = slice(b, b + few)
        part = T.recurrence(f[p], u[p], None if o is None else o[p], save=True)
        assert torch.equal(part[0], y[p]) and torch.equal(part[1], last[p]) and torch.equal(part[2], saved[:, p])
        for a, c in zip(T.recurrence_grad(f[p], u[p], part[2], dy[p], None if o is None else o[p]), grads):
            assert a is None and c is None or torch.equal(a, c[p])


def test_empty_shapes():
    h0 = torch.ones((3, 8), device="cuda")
    f = torch.zeros((3, 0, 8), device="cuda")
    y, last, saved = T.recurrence(f, f, h0=h0, save=True)
    assert y.shape == (3, 0, 8) and torch.equal(last, h0) and saved.shape == (0, 3, 8)
    df, du, do, dh0 = T.recurrence_grad(f, f, saved, f, dlast=2 * h0)
    assert df.shape == (3, 0, 8) and do is None and torch.equal(dh0, 2 * h0)
    f = torch.zeros((0, 4, 8), device="cuda")
    assert T.recurrence(f, f)[0].shape == (0, 4, 8)


@pytest.mark.parametrize("steps,dim", [(35, 100), (3000, 64)])
def test_other_streams_and_graphs(steps, dim):
    proj, f, u, o, h0, dy, dlast = inputs(2, steps, dim, torch.float32, True, 61)
    f, u, o, dy = (t.contiguous().cuda() for t in (f, u, o, dy))
    y, last, saved = T.recurrence(f, u, o, save=True)
    grads = T.recurrence_grad(f, u, saved, dy, o)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2, last2, saved2 = T.recurrence(f, u, o, save=True)
        grads2 = T.recurrence_grad(f, u, saved2, dy, o)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(saved, saved2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y3, last3, saved3 = T.recurrence(f, u, o, save=True)
        grads3 = T.recurrence_grad(f, u, saved3, dy, o)
    for replay in range(3):
        for t in (y3, last3, saved3) + grads3:
            t.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y3) and torch.equal(last, last3)
        for a, b, c in zip(grads, grads2, grads3):
            assert torch.equal(a, b) and torch.equal(a, c), replay
        T.recurrence(f * 0.5, u)                # eager work between the replays
        torch.cuda.synchronize()


def test_arguments_are_checked():
    f = torch.zeros((2, 20, 8), device="cuda")
    saved = torch.zeros((3, 2, 8), device="cuda")
    for bad in (lambda: T.recurrence(f, f.bfloat16()), lambda: T.recurrence(f, f[:, :3]), lambda: T.recurrence(f.double(), f.double()),
                lambda: T.recurrence(f, f, h0=saved[0, :1]), lambda: T.recurrence(f, f, lengths=torch.zeros(2, device="cuda")),
                lambda: T.recurrence(f.transpose(1, 2), f.transpose(1, 2)), lambda: T.recurrence_grad(f, f, saved[:1], f),
                lambda: T.recurrence_grad(f, f, saved, f.cpu())):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(B.ChocoError):
        T.recurrence(f, f, out=torch.zeros((2, 1, 8), device="cuda").expand(2, 20, 8))
