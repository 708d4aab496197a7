"""AdamW against a plain computation in 64 bits, step by step from the state that the device holds.

Tolerances, in fp32's 2^-24: a moment is two products and a sum (4 of the terms' magnitudes: three roundings, the constants'
own); x' is a product, a product of four factors each good to a few units, a difference (3 of |x|, 40 of the step).  In 8 bits
the codes are compared: exactly, except where the value to be rounded lies within 2^-17 of a code's width of going
the other way (fp32 values of up to 16 such widths are good to 5 roundings), and where a block's largest lies as near to the
next power of two."""
import numpy as np
import pytest
import torch

from paper_1907_09356_amd import binding as B
from paper_1907_09356_amd import synth
from paper_1907_09356_amd import train as T

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BLOCK = 256


def philox(d, n, t, stream, seed):
    """One 32-bit word per entry (n, d): Philox4x32-10 (Salmon et al., SC'11)."""
    mask = np.uint64(0xFFFFFFFF)
    shift = np.uint64(32)
    c = [np.broadcast_to(np.arange((d + 3) // 4, dtype=np.uint64), (n, (d + 3) // 4)),
         np.broadcast_to(np.arange(n, dtype=np.uint64)[:, None], (n, (d + 3) // 4)),
         np.full((n, (d + 3) // 4), t & 0xFFFFFFFF, dtype=np.uint64),
         np.full((n, (d + 3) // 4), stream | (t >> 32 << 8), dtype=np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> shift) ^ c[1] ^ np.uint64(k0), p1 & mask, (p0 >> shift) ^ c[3] ^ np.uint64(k1), p0 & mask]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 2).reshape(n, -1)[:, :d]


def blocks(tensors):
    for start, length in zip(*tensors):
        for at in range(int(start), int(start + length), BLOCK):
            yield slice(at, min(at + BLOCK, int(start + length)))


def held(x, r, tensors, exponent_bits):
    """What 8 bits hold of x (64 bits): (value, the values on either side of a rounding that is too close to call)."""
    out, low, high = np.zeros_like(x), np.zeros_like(x), np.zeros_like(x)
    for p in blocks(tensors):
        y = np.abs(x[:, p])
        most = y.max(1, keepdims=True)
        scale = np.exp2(np.ceil(np.log2(np.where(most > 0, most, 1.0) / 1.875)))      # the largest: in (0.9375, 1.875]
        y = y / scale
        exponent = np.maximum(np.frexp(y)[1] - 1, 2 - 2 ** exponent_bits)
        width = np.exp2(exponent - 3.0)
        place = y / width + r[:, p] / 65536.0
        for dest, q in ((out, place), (low, place - 2.0 ** -17), (high, place + 2.0 ** -17)):
            v = np.floor(q) * width
            if exponent_bits == 5:
                v = np.where((y > 0) & (v == 0), width, v)
            dest[:, p] = np.copysign(np.clip(v, 0, 1.875) * scale, x[:, p])
    return out, low, high


def inside(tensors, d):
    at = np.zeros(d, dtype=bool)
    for start, length in zip(*tensors):
        at[int(start):int(start + length)] = True
    return at


def per_entry(values, tensors, d, default):
    out = np.full(d, default, dtype=np.float64)
    for value, start, length in zip(values, *tensors):
        out[int(start):int(start + length)] = np.float32(value)
    return out


def rows(n, d, ld, seed, spread):
    x = np.zeros((n, ld), dtype=np.float32)
    x[:] = np.random.default_rng(seed).standard_normal((n, ld)) * spread
    return x


TABLES = {
    "whole": (1000, None),
    "one entry": (1, None),
    "padded": (synth.layers_dim(synth.layer_table([3, 700, 1, 256, 2048, 257, 1029])), synth.layer_table([3, 700, 1, 256, 2048, 257, 1029])[:2]),
    "anywhere": (6003, ([1, 2, 300, 300, 301, 2600, 2605, 5999], [1, 290, 0, 1, 2299, 5, 3000, 3])),
    "long": (40_001, ([0, 20_000], [19_999, 20_001])),
    "image": (synth.layers_dim(synth.layer_table(synth.resnet20_like_lengths())), synth.layer_table(synth.resnet20_like_lengths())[:2]),
}


@pytest.mark.parametrize("name", list(TABLES))
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("clip", [False, True])
def test_steps_against_64_bits(name, bits, grad, clip):
    d, tensors = TABLES[name]
    n, ld = (2 if name == "image" else 3), (d + 7) // 4 * 4
    table = ([0], [d]) if tensors is None else tensors
    g = np.random.default_rng(len(name))
    decay, scale = g.random(len(table[0])) * 0.2, 0.5 + g.random(len(table[0]))
    X = torch.from_numpy(rows(n, d, ld, 1, 0.05)).cuda()
    betas, eps, lr, seed = (0.9, 0.999), 1e-8, float(np.float32(0.01)), 0x123456789ABCDEF
    kw = dict(weight_decay=decay if tensors is not None else decay[0], lr_scale=scale if tensors is not None else scale[0])
    opt = T.AdamW(X, d, tensors, betas=betas, eps=eps, state_bits=bits, seed=seed, **kw)
    wd, ls, on = per_entry(decay, table, d, 0.0), per_entry(scale, table, d, 1.0), inside(table, d)
    factor = torch.tensor([0.25, 1.0, 3.0][:n], dtype=torch.float32).cuda() if clip else None
    start = X.cpu().numpy().copy()
    for t in range(1, 4):
        G = torch.from_numpy(rows(n, d, ld, 10 + t, 0.01 * t)).to(grad).cuda()
        x0, (m0, v0) = X[:, :d].double().cpu().numpy(), (s.double().cpu().numpy() for s in opt.moments())
        opt.step(G, lr, grad_scale=factor)
        assert opt.get_step() == t
        gr = G[:, :d].double().cpu().numpy() * (factor.double().cpu().numpy()[:, None] if clip else 1.0)
        if clip:
            gr = gr.astype(np.float32).astype(np.float64)        # the scaled gradient is an fp32 number
        m, v = betas[0] * m0 + (1 - betas[0]) * gr, betas[1] * v0 + (1 - betas[1]) * gr * gr
        step = lr * ls * (m / (1 - betas[0] ** t) / (np.sqrt(v / (1 - betas[1] ** t)) + eps))
        x = np.where(on, x0 - step - lr * ls * wd * x0, x0)
        err = np.abs(X[:, :d].double().cpu().numpy() - x)
        # the moments' own errors move the step: relative to it they are those of m and (halved) v
        size_m = betas[0] * np.abs(m0) + (1 - betas[0]) * np.abs(gr)
        move = np.abs(step) / np.maximum(np.abs(m), 1e-30) * size_m
        assert np.all(err <= U * (3 * np.abs(x0) + 40 * np.abs(step) + 8 * move) + 1e-30), float(err.max())
        gm, gv = (s.double().cpu().numpy() for s in opt.moments())
        assert not gm[:, ~on].any() and not gv[:, ~on].any()
        if bits == 32:
            assert np.all(np.abs(gm - np.where(on, m, 0)) <= 4 * U * size_m + 1e-30)
            assert np.all(np.abs(gv - np.where(on, v, 0)) <= 5 * U * v + 1e-30)
            continue
        words = philox(d, n, t - 1, 3, seed)
        for got, want, r, e in ((gm, m, words & np.uint64(0xFFFF), 4), (gv, v, words >> np.uint64(16), 5)):
            mid, low, high = held(np.where(on, want, 0.0), r.astype(np.float64), table, e)
            near = lambda a: np.abs(got - a) <= 8 * U * np.abs(a) + 1e-38        # noqa: E731
            assert np.all(near(mid) | near(low) | near(high))
            assert np.mean(~near(mid)) < 1e-3
    at = X.cpu().numpy()
    assert np.array_equal(at[:, :d][:, ~on], start[:, :d][:, ~on]) and np.array_equal(at[:, d:], start[:, d:])
    opt.close()


def test_philox_known_answers():
    import os
    for line in open(os.path.join(os.path.dirname(os.path.abspath(__file__)), "golden", "philox4x32_10_kat.txt")):
        if line.startswith("#") or not line.strip():
            continue
        w = [int(v, 16) for v in line.split()]
        if w[0] == 0:       # (the counter's first word is an entry / 4 here: only small ones can be reached)
            t = w[2] | (w[3] >> 8) << 32
            assert philox(4, w[1] + 1, t, w[3] & 0xFF, w[4] | w[5] << 32)[w[1]].tolist() == w[6:]


def test_rounding_is_unbiased():
    # no gradient but for one entry of each block, which keeps the scale: v shrinks by 0.1 % a step although its codes lie
    # 6 to 12 % apart, m by 10 %.  The mean over N independent entries of spread s is good to 5 s / sqrt(N)
    n, d, steps = 16, 256 * 50, 40
    X = torch.zeros((n, d), device="cuda")
    opt = T.AdamW(X, d, state_bits=8, seed=5)
    G = torch.from_numpy((0.5 + np.random.default_rng(1).random((n, d))).astype(np.float32)).cuda()
    G[:, ::256] = 2.0
    opt.step(G, 0.0)
    m0, v0 = (t.double().cpu().numpy() for t in opt.moments())
    G.zero_()
    G[:, ::256] = 2.0
    for _ in range(steps):
        opt.step(G, 0.0)
    m, v = (t.double().cpu().numpy() for t in opt.moments())
    inner = np.broadcast_to(np.arange(d) % 256 != 0, (n, d))
    for now, before, beta in ((m, m0, 0.9), (v, v0, 0.999)):
        ratio = (now / (before * beta ** steps))[inner]
        assert abs(ratio.mean() - 1) <= 5 * ratio.std() / np.sqrt(ratio.size), (beta, ratio.mean(), ratio.std())
        assert 0.0 < ratio.std() < 0.5


def test_a_positive_second_moment_is_never_held_as_zero():
    d = 512
    G = torch.full((1, d), 1e-6, device="cuda")
    G[0, ::256] = 1e3
    X = torch.zeros((1, d), device="cuda")
    opt = T.AdamW(X, d, state_bits=8)
    for _ in range(20):
        opt.step(G, 1e-3)
    assert bool((opt.moments()[1] > 0).all())
    assert float(X.abs().max()) <= 20 * 1e-3 * 1.0001          # no step longer than the stepsize


@pytest.mark.parametrize("bits", [32, 8])
def test_no_gradient_at_all(bits):
    X = torch.ones((2, 700), device="cuda")
    opt = T.AdamW(X, 700, state_bits=bits, weight_decay=0.5)
    opt.step(torch.zeros_like(X), 0.1)
    assert bool((X == np.float32(1 - np.float32(0.1) * np.float32(0.5))).all())
    m, v = opt.moments()
    assert not bool(m.any()) and not bool(v.any())
    # gradients whose squares are below the normal numbers
    opt.step(torch.full_like(X, 1e-21), 0.1)
    assert bool(torch.isfinite(X).all()) and bool(torch.isfinite(opt.moments()[0]).all())


@pytest.mark.parametrize("bits", [32, 8])
def test_the_least_eps_and_gradients_whose_squares_underflow(bits):
    # x starts at 0, so x' is the step alone.  v is off by what fp32 loses below its normal numbers, 2^-149, which is 2^-14 of
    # the least eps once it is under the root; the step's other roundings as above, m's own below the normal numbers 2^-149 too
    sizes = [0.0, 1e-38, 1e-35, 1e-30, 1e-24, 1e-22, 1e-21, 3e-21, 1e-20, 1e-19, 3e-19, 1e-18, 1e-17, 1e-15, 1e-10, 1.0]
    g = np.repeat(np.array(sizes), BLOCK) * (0.5 + np.random.default_rng(1).random(BLOCK * len(sizes)))
    G = torch.from_numpy(g.astype(np.float32)[None]).cuda()
    gr = G.double().cpu().numpy()
    X = torch.zeros_like(G)
    betas = (0.9, 0.999)
    eps = 2.0 ** -60 / (1 - betas[1]) ** 0.5
    opt = T.AdamW(X, g.size, betas=betas, eps=eps, state_bits=bits, seed=3)
    for t in range(1, 4):
        m0, v0 = (s.double().cpu().numpy() for s in opt.moments())
        X.zero_()
        opt.step(G, 1.0)
        m, v = betas[0] * m0 + (1 - betas[0]) * gr, betas[1] * v0 + (1 - betas[1]) * gr * gr
        step = m / (1 - betas[0] ** t) / (np.sqrt(v / (1 - betas[1] ** t)) + eps)
        bound = np.abs(step) * (2.0 ** -14 + 64 * U + 4 * 2.0 ** -149 / np.maximum(m, 1e-300))
        assert np.all(np.abs(X.double().cpu().numpy() + step) <= bound), t
        gm, gv = (s.double().cpu().numpy() for s in opt.moments())
        assert np.all(gv[v >= 2.0 ** -148] > 0) and np.all(gm[m > 0] > 0)
        assert not gm[gr == 0].any() and not gv[gr == 0].any()
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_worker_whose_factor_is_not_finite_is_left_alone(bits):
    n, d = 5, 1500
    X = torch.from_numpy(rows(n, d, d, 1, 0.1)).cuda()
    opt = T.AdamW(X, d, state_bits=bits)
    G = torch.from_numpy(rows(n, d, d, 2, 0.1)).cuda()
    opt.step(G, 0.01)
    x0, (m0, v0), s0 = X.clone(), (t.clone() for t in opt.moments()), opt.state().clone()
    G[1], G[3] = float("inf"), float("nan")
    factor = torch.tensor([1.0, float("nan"), 0.0, float("inf"), -float("inf")], device="cuda")
    opt.step(G, 0.01, grad_scale=factor)
    m, v = (t.clone() for t in opt.moments())
    for w in (1, 3, 4):
        assert torch.equal(X[w], x0[w]) and torch.equal(m[w], m0[w]) and torch.equal(v[w], v0[w])
    for w in (0, 2):
        assert not torch.equal(X[w], x0[w]) and bool(torch.isfinite(X[w]).all())
    opt.state().copy_(s0)       # put back: the same step gives the same bits
    x1, X[:] = X.clone(), x0
    opt.set_step(1)
    opt.step(G, 0.01, grad_scale=factor)
    assert torch.equal(X, x1) and torch.equal(opt.moments()[0], m) and torch.equal(opt.moments()[1], v)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_not_finite_do_not_reach_other_blocks(bad):
    d = 2048
    G = torch.full((2, d), 0.5, device="cuda")
    G[0, 700] = bad
    for bits in (32, 8):
        X = torch.zeros((2, d), device="cuda")
        opt = T.AdamW(X, d, state_bits=bits)
        opt.step(G, 0.1)
        m, v = opt.moments()
        spoilt = torch.zeros((2, d), dtype=torch.bool, device="cuda")
        spoilt[0, (700 if bits == 32 else 512):(701 if bits == 32 else 768)] = True
        ok = ~spoilt
        assert bool(torch.isfinite(m[ok]).all()) and bool(torch.isfinite(v[ok]).all())
        assert not bool(torch.isfinite(v[spoilt]).any())
        x_ok = torch.ones((2, d), dtype=torch.bool, device="cuda")
        x_ok[0, 700] = False
        assert bool((X[x_ok] == X[1, 0]).all()) and bool(torch.isnan(X[0, 700]))


def test_with_gossip_steps():
    # AdamW takes the place of the local update: the same X, then a gossip step that conserves the workers' mean
    n, (start, length, k) = 8, synth.layer_table(synth.resnet20_like_lengths())
    d = int(start[-1] + length[-1])
    ld = (d + 63) // 64 * 64
    X = torch.from_numpy(rows(n, d, ld, 3, 0.05)).cuda()
    X[:, d:] = 0
    ctx = B.Choco(X, d, *synth.ring_csr(n), 0.3, B.Q_TOPK, layers=(start, length, k))
    opt = T.AdamW(X, d, (start, length), state_bits=8, weight_decay=0.01)
    for t in range(4):
        opt.step(torch.from_numpy(rows(n, d, ld, 20 + t, 0.01)).cuda(), 1e-3)
        before = X[:, :d].double().mean(0)
        ctx.gossip_step()
        assert float((X[:, :d].double().mean(0) - before).abs().max()) < 1e-7
    assert np.isfinite(ctx.metrics()["consensus"])
    ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_rows_of_more_than_32_bits_of_entries(bits):
    # the second of two rows of 1.2 * 2^30 entries lies beyond 2^30 entries, its end beyond 2^31; tensors at both ends
    n, d = 2, 1_288_490_188
    X = torch.zeros((n, d), device="cuda")
    G = torch.zeros((n, d), dtype=torch.bfloat16, device="cuda")
    G[:, :3], G[:, -1025:] = 1.0, -1.0
    opt = T.AdamW(X, d, ([0, d - 2000], [5, 2000]), state_bits=bits)
    opt.step(G, 0.25)
    assert X[:, :6].cpu().tolist() == [[pytest.approx(-0.25, rel=1e-5)] * 3 + [0.0] * 3] * 2
    assert X[:, -1027:-1023].cpu().tolist() == [[0.0] * 2 + [pytest.approx(0.25, rel=1e-5)] * 2] * 2
    assert int((X != 0).sum()) == 2 * (3 + 1025)


def test_state_that_does_not_fit_the_caches():
    # more than 320 MB go past the caches: the same bits as a worker at a time; in 8 bits, whose words depend on the worker, the
    # first worker's
    n, d = 9, 4_000_003
    ld = d + 1
    gen = torch.Generator(device="cuda").manual_seed(4)
    X0 = torch.empty((n, ld), device="cuda").normal_(generator=gen)
    G = torch.empty((n, ld), device="cuda").normal_(generator=gen)
    for bits in (32, 8):
        X = X0.clone()
        opt = T.AdamW(X, d, ([0, 1_000_004], [1_000_001, 2_999_999]), state_bits=bits, weight_decay=0.1)
        for w in range(n if bits == 32 else 1):
            x = X0[w:w + 1].clone()
            alone = T.AdamW(x, d, ([0, 1_000_004], [1_000_001, 2_999_999]), state_bits=bits, weight_decay=0.1)
            for _ in range(2):
                alone.step(G[w:w + 1], 0.01)
            if w == 0:
                for _ in range(2):
                    opt.step(G, 0.01)
            assert torch.equal(x[0], X[w])
            for a, b in zip(alone.moments(), opt.moments()):
                assert torch.equal(a[0], b[w])
            alone.close()
        opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_other_streams_and_graphs(bits):
    n, d = 3, 5000
    X0 = torch.from_numpy(rows(n, d, d, 1, 0.1)).cuda()
    G = torch.from_numpy(rows(n, d, d, 2, 0.1)).cuda()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        X = X0.clone()
        opt = T.AdamW(X, d, state_bits=bits, seed=9)
        graph = torch.cuda.CUDAGraph()
        s0 = opt.state().clone()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            opt.step(G, 0.01)
        for replay in range(3):         # each replay is the step it was captured as
            graph.replay()
            side.synchronize()
            y, z = X.clone(), opt.state().clone()
            X.copy_(X0)
            opt.state().copy_(s0)
            opt.set_step(0)
            opt.step(G, 0.01)
            side.synchronize()
            assert torch.equal(X, y) and torch.equal(opt.state(), z), replay
            X.copy_(X0)
            opt.state().copy_(s0)
    side.synchronize()


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_keep_what_they_were(bits):
    # neither a later step changes them nor does writing to them change the optimiser
    n, d = 2, 1300
    X = torch.from_numpy(rows(n, d, d, 1, 0.1)).cuda()
    G = torch.from_numpy(rows(n, d, d, 2, 0.1)).cuda()
    opt = T.AdamW(X, d, state_bits=bits)
    opt.step(G, 0.01)
    before = opt.moments()
    kept = [t.clone() for t in before]
    opt.step(2 * G, 0.01)
    for a, b in zip(before, kept):
        assert torch.equal(a, b)
    now = opt.moments()
    kept = [t.clone() for t in now]
    for t in now:
        t.fill_(7.0)
    for a, b in zip(opt.moments(), kept):
        assert torch.equal(a, b)
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_the_current_stream_is_followed(bits):
    # made on one stream, used on another one whose earlier work is still under way, then captured on a third
    n, d = 3, 5000
    X0 = torch.from_numpy(rows(n, d, d, 1, 0.1)).cuda()
    grads = [torch.from_numpy(rows(n, d, d, 2 + t, 0.1)).cuda() for t in range(3)]
    plain = X0.clone()
    opt = T.AdamW(plain, d, state_bits=bits, seed=9)
    want = []
    for G in grads:
        opt.step(G, 0.01)
        want.append((plain.clone(),) + tuple(t.clone() for t in opt.moments()))
    opt.close()
    X, G = X0.clone(), torch.zeros_like(X0)
    opt = T.AdamW(X, d, state_bits=bits, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for t in range(2):
            torch.cuda._sleep(5_000_000)
            G.copy_(grads[t])
            opt.step(G, 0.01)
            got = (X.clone(),) + tuple(s.clone() for s in opt.moments())
            G.zero_()
            for a, b in zip(got, want[t]):
                assert torch.equal(a, b), t
    torch.cuda.synchronize()
    x1, s1 = X.clone(), opt.state().clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.copy_(grads[2])
        opt.step(G, 0.01)
    assert torch.equal(X, x1)           # captured, not run
    for replay in range(3):
        graph.replay()
        for a, b in zip((X,) + opt.moments(), want[2]):
            assert torch.equal(a, b), replay
        X.copy_(x1)
        opt.state().copy_(s1)
        G.zero_()
        torch.cuda.synchronize()
    opt.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_as_copies(bits):
    # the C call writes both moments whatever they are held in, zero outside the tensors
    n, d, tensors = 2, 700, ([5, 300], [200, 333])
    X = torch.from_numpy(rows(n, d, d, 1, 0.1)).cuda()
    opt = T.AdamW(X, d, tensors, state_bits=bits)
    opt.step(torch.from_numpy(rows(n, d, d, 2, 0.1)).cuda(), 0.01)
    m, v = torch.full_like(X, 7.0), torch.full_like(X, 7.0)
    assert T.lib().choco_adamw_moments(opt.handle, m.data_ptr(), v.data_ptr()) == B.OK
    for got, want in zip((m, v), opt.moments()):
        assert torch.equal(got, want) and not bool(got[:, ~torch.from_numpy(inside(tensors, d))].any()) and bool(got[:, 5:205].any())
    opt.close()


def test_arguments_are_checked():
    X = torch.zeros((2, 64), device="cuda")
    opt = T.AdamW(X, 60)
    for bad in (lambda: opt.step(X[:1], 0.1), lambda: opt.step(X.half(), 0.1), lambda: opt.step(X, 0.1, grad_scale=X[0]),
                lambda: T.AdamW(X[:, :60], 60), lambda: T.AdamW(X.bfloat16(), 60)):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(B.ChocoError):
        T.AdamW(X, 65)
    with pytest.raises(B.ChocoError):
        opt.step(X, float("nan"))
    assert opt.get_step() == 0
    opt.close()
