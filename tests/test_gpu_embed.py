"""Embedding lookup and its gradient against plain computations in 64 bits.

Tolerances: a looked-up row is one fp32 product, rounded once: bit for bit.  A sum of k rows in fp32, in whatever order, is
off by at most k + 1 roundings (one of them the scale's) of 2^-24 of the sum of magnitudes, the first order of the
standard bound; 2 more are allowed for the second order and, accumulating, for what was there."""
import numpy as np
import pytest
import torch

from paper_1907_09356_amd import binding as B
from paper_1907_09356_amd import train as T

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def rng(seed):
    return np.random.default_rng(seed)


def draw_tokens(n, count, vocab, seed, how):
    g = rng(seed)
    if how == "frequent":      # few words make up most of the text, some of it padding
        t = np.minimum(np.floor(vocab ** g.random((n, count))).astype(np.int64) - 1, vocab - 1)
        t[g.random((n, count)) < 0.2] = -1
    elif how == "one":
        t = np.full((n, count), vocab - 1)
    elif how == "outside":     # none of them in the table
        t = np.where(g.random((n, count)) < 0.5, -1 - g.integers(0, 10, (n, count)), vocab + g.integers(0, 10, (n, count)))
    else:
        t = g.integers(0, vocab, (n, count))
    return t.astype(np.int64)


def values(shape, seed, dtype):
    x = torch.from_numpy(rng(seed).standard_normal(shape).astype(np.float32))
    return x.to(dtype)


SIZES = [   # n, tokens, vocab, dim, how
    (1, 1, 1, 1, "uniform"), (1, 1, 5, 650, "uniform"), (3, 7, 11, 33, "uniform"), (2, 64, 50, 4, "frequent"),
    (2, 65, 200, 130, "one"), (8, 20, 333, 650, "uniform"), (1, 300, 40, 257, "frequent"), (2, 50, 9, 12, "outside"),
    (1, 2049, 700, 96, "frequent"), (1, 9001, 1500, 20, "frequent"), (2, 4100, 33, 66, "uniform"), (1, 5000, 7, 5, "one"),
    (2, 128, 60, 70, "frequent"), (2, 129, 60, 70, "frequent"), (1, 128, 3, 10, "one"), (1, 8192, 5000, 4, "frequent"),
    (1, 8193, 5000, 4, "frequent"), (1, 131_072, 9000, 2, "frequent"),
    (1, 40_000, 70_000, 3, "frequent"), (1, 20_011, 300, 40, "one"), (3, 17_000, 1000, 8, "uniform"), (1, 6000, 1_100_000, 2, "frequent"),
]


@pytest.mark.parametrize("n,count,vocab,dim,how", SIZES)
@pytest.mark.parametrize("kinds", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16),
                                   (torch.float16, torch.float32)])
def test_lookup(n, count, vocab, dim, how, kinds):
    tokens = draw_tokens(n, count, vocab, 1, how)
    table = values((n, vocab, dim), 2, kinds[0])
    scale = float(np.float32(dim ** 0.5))
    for dtype in (torch.int64, torch.int32):
        y = T.embed(torch.from_numpy(tokens).to(dtype).cuda(), table.cuda(), scale=scale, out_dtype=kinds[1]).cpu()
        there = (tokens >= 0) & (tokens < vocab)
        want = torch.zeros((n, count, dim))
        for w in range(n):
            want[w, there[w]] = table[w, tokens[w, there[w]]].float() * np.float32(scale)
        assert torch.equal(y, want.to(kinds[1]))


def grad_reference(tokens, dy, vocab, scale):
    """(sum, sum of magnitudes, number of rows) per table row, in 64 bits."""
    n, count, dim = dy.shape
    total, size, rows = np.zeros((n, vocab, dim)), np.zeros((n, vocab, dim)), np.zeros((n, vocab, 1))
    d = dy.double().numpy() * scale
    for w in range(n):
        there = np.nonzero((tokens[w] >= 0) & (tokens[w] < vocab))[0]
        np.add.at(total[w], tokens[w, there], d[w, there])
        np.add.at(size[w], tokens[w, there], np.abs(d[w, there]))
        np.add.at(rows[w], tokens[w, there], 1.0)
    return total, size, rows


def check_grad(got, old, tokens, dy, vocab, scale):
    total, size, rows = grad_reference(tokens, dy, vocab, scale)
    base = 0.0 if old is None else old.double().numpy()
    err = np.abs(got.double().numpy() - (base + total))
    bound = U * (rows + 3) * size + (0.0 if old is None else U * (np.abs(base) + size))
    assert np.all(err <= bound), float(np.max(err - bound))
    if old is not None:
        untouched = np.broadcast_to(rows == 0, err.shape)
        assert np.array_equal(got.numpy()[untouched], old.numpy()[untouched])


@pytest.mark.parametrize("n,count,vocab,dim,how", SIZES)
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(n, count, vocab, dim, how, kind, accumulate):
    tokens = draw_tokens(n, count, vocab, 3, how)
    dy = values((n, count, dim), 4, kind)
    old = values((n, vocab, dim), 5, torch.float32)
    dtable = old.cuda()
    scale = float(np.float32(0.3))
    dev = torch.from_numpy(tokens).cuda()
    T.embed_grad(dev, dy.cuda(), dtable, scale=scale, accumulate=accumulate)
    check_grad(dtable.cpu(), old if accumulate else None, tokens, dy, vocab, scale)
    again = old.cuda()      # the order of a sum goes by the tokens alone
    T.embed_grad(dev.int(), dy.cuda(), again, scale=scale, accumulate=accumulate)
    assert torch.equal(again, dtable)


@pytest.mark.parametrize("n,count,vocab,dim,how", [(1, 262_143, 9000, 2, "frequent"), (1, 262_144, 9000, 2, "frequent"),
                                                   (2, 300_001, 70_000, 3, "frequent"), (1, 270_000, 900, 4, "one")])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_long_lists(n, count, vocab, dim, how, accumulate):
    test_gradient(n, count, vocab, dim, how, torch.bfloat16, accumulate)


def test_gradient_by_differences():
    # the loss sum(w * y) is linear in the table: a difference quotient is exact but for its own roundings
    n, count, vocab, dim = 1, 9, 6, 5
    tokens = draw_tokens(n, count, vocab, 6, "frequent")
    dy = values((n, count, dim), 7, torch.float32)
    table = values((n, vocab, dim), 8, torch.float32)
    dtable = torch.zeros_like(table).cuda()
    T.embed_grad(torch.from_numpy(tokens).cuda(), dy.cuda(), dtable, scale=2.0)
    for v in range(vocab):
        for c in range(dim):
            sides = []
            for step in (0.5, -0.5):
                moved = table.clone()
                moved[0, v, c] += step
                y = T.embed(torch.from_numpy(tokens).cuda(), moved.cuda(), scale=2.0).cpu()
                sides.append((y.double() * dy.double()).sum().item())
            size = float((dy.double().abs() * 2 * 4).sum())          # |y| stays below 4 (the seed's values)
            assert abs((sides[0] - sides[1]) - dtable[0, v, c].item()) <= 16 * U * size


@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4, 6])
def test_rows_that_start_anywhere(offset):
    # tables inside the workers' rows, looked-up rows with padding between them: aligned to their entries only
    n, count, vocab, dim = 3, 37, 23, 12
    tokens = draw_tokens(n, count, vocab, 9, "frequent")
    dev = torch.from_numpy(tokens).cuda()
    for kind in (torch.float32, torch.bfloat16):
        X = values((n, offset + vocab * dim + 5), 10, kind).cuda()
        table = X[:, offset:offset + vocab * dim].view(n, vocab, dim)
        buffer = torch.full((n, count + 1, dim + offset), 7.0, dtype=kind, device="cuda")
        out = buffer[:, :count, :dim]
        T.embed(dev, table, out=out)
        want = torch.zeros((n, count, dim), dtype=kind)
        for w in range(n):
            ok = tokens[w] >= 0
            want[w, ok] = table[w].cpu()[tokens[w, ok]]
        assert torch.equal(out.cpu(), want)
        assert bool((buffer[:, count:] == 7).all()) and bool((buffer[:, :, dim:] == 7).all())
        for accumulate in (False, True):
            G = torch.full((n, offset + vocab * dim + 5), 3.0, device="cuda")
            slot = G[:, offset:offset + vocab * dim].view(n, vocab, dim)
            old = slot.cpu()
            T.embed_grad(dev, out, slot, accumulate=accumulate)
            check_grad(slot.cpu(), old if accumulate else None, tokens, want, vocab, 1.0)
            assert bool((G[:, :offset] == 3).all()) and bool((G[:, offset + vocab * dim:] == 3).all())


def test_no_tokens_clear_the_gradient_or_leave_it():
    dtable = torch.ones((2, 9, 5), device="cuda")
    tokens, dy = torch.zeros((2, 0), dtype=torch.int64, device="cuda"), torch.zeros((2, 0, 5), device="cuda")
    T.embed_grad(tokens, dy, dtable, accumulate=True)
    assert bool((dtable == 1).all())
    T.embed_grad(tokens, dy, dtable)
    assert bool((dtable == 0).all())
    assert T.embed(tokens, dtable).shape == (2, 0, 5)


def test_infinities_and_nans_stay_in_their_rows():
    tokens = torch.tensor([[0, 1, 1, -1, 3, 9]]).cuda()
    dy = torch.ones((1, 6, 70)).cuda()
    dy[0, 0], dy[0, 2], dy[0, 3], dy[0, 5] = float("inf"), float("nan"), float("nan"), float("inf")   # the last two: outside
    dtable = torch.zeros((1, 5, 70), device="cuda")
    T.embed_grad(tokens, dy, dtable)
    got = dtable.cpu()[0]
    assert bool(torch.isinf(got[0]).all()) and bool(torch.isnan(got[1]).all())
    assert bool((got[2] == 0).all()) and bool((got[3] == 1).all()) and bool((got[4] == 0).all())


def test_tables_of_more_than_32_bits_of_entries():
    # bf16 table of 2^31 + 2^20 entries; gradient of the same number in fp32: the first rows and the last ones
    dim = 1 << 11
    vocab = (1 << 20) + 512
    table = torch.zeros((1, vocab, dim), dtype=torch.bfloat16, device="cuda")
    table[0, -1], table[0, -2], table[0, 0] = 1.0, 2.0, 3.0
    tokens = torch.tensor([[vocab - 1, 0, vocab - 2, vocab]]).cuda()
    y = T.embed(tokens, table)
    assert y[0, :, 0].tolist() == [1.0, 3.0, 2.0, 0.0] and y[0, :, -1].tolist() == [1.0, 3.0, 2.0, 0.0]
    del table
    dtable = torch.ones((1, vocab, dim), device="cuda")
    dy = torch.full((1, 4, dim), 5.0, device="cuda")
    T.embed_grad(tokens, dy, dtable)
    assert dtable[0, :, 0].nonzero()[:, 0].tolist() == [0, vocab - 2, vocab - 1]
    assert float(dtable[0].sum(dtype=torch.float64)) == 3 * 5.0 * dim


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_results_that_do_not_fit_the_caches(kind):
    # rows of more than 96 MB are written and read past the caches: the same bits as in shares of them (lookups), and as sums
    # in 64 bits within the bound (gradients)
    count, vocab, dim = 60_000, 9000, 1024 if kind == torch.bfloat16 else 512
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.from_numpy(draw_tokens(1, count, vocab, 13, "frequent")).cuda()
    table = torch.empty((1, vocab, dim), dtype=kind, device="cuda").normal_(generator=gen)
    y = T.embed(tokens, table, scale=3.0)
    for at in range(0, count, 15_000):
        assert torch.equal(y[:, at:at + 15_000], T.embed(tokens[:, at:at + 15_000].contiguous(), table, scale=3.0))
    there = tokens[0] >= 0
    rows = y[0, there].double()
    for accumulate in (False, True):
        old = torch.empty((1, vocab, dim), device="cuda").normal_(generator=gen)
        got = old.clone()
        T.embed_grad(tokens, y, got, scale=0.5, accumulate=accumulate)
        base = old[0].double() if accumulate else torch.zeros((vocab, dim), dtype=torch.float64, device="cuda")
        want = base.index_add(0, tokens[0, there], rows * 0.5)
        size = torch.zeros_like(base).index_add_(0, tokens[0, there], rows.abs() * 0.5)
        number = torch.bincount(tokens[0, there], minlength=vocab)[:, None]
        bound = U * (number + 3) * size + U * (base.abs() + size)
        assert bool(((got[0].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("count", [100, 500, 9000, 40_000])
def test_gradients_that_do_not_fit_the_caches(count):
    # more than 64 MB to be cleared, by either way of putting tokens in order and without; rows of 0.3 to 104 MB to add up
    n, vocab, dim = 2, 20_001, 650
    gen = torch.Generator(device="cuda").manual_seed(count)
    tokens = torch.from_numpy(draw_tokens(n, count, vocab, 14, "frequent")).cuda()
    dy = torch.empty((n, count, dim), device="cuda").normal_(generator=gen)
    buffer = torch.full((n, vocab * dim + 6), 5.0, device="cuda")
    got = buffer[:, 1:vocab * dim + 1].view(n, vocab, dim)
    T.embed_grad(tokens, dy, got, scale=2.0)
    for w in range(n):
        there = tokens[w] >= 0
        at, rows = tokens[w, there], 2.0 * dy[w, there].double()
        zero = torch.zeros((vocab, dim), dtype=torch.float64, device="cuda")
        want, size = zero.index_add(0, at, rows), zero.index_add(0, at, rows.abs())
        number = torch.bincount(at, minlength=vocab)[:, None]
        assert bool(((got[w].double() - want).abs() <= U * (number + 3) * size).all())
    assert bool((buffer[:, :1] == 5).all()) and bool((buffer[:, vocab * dim + 1:] == 5).all())


def test_other_streams_and_graphs():
    n, count, vocab, dim = 2, 1500, 5000, 50
    tokens = torch.from_numpy(draw_tokens(n, count, vocab, 11, "frequent")).cuda()
    dy = values((n, count, dim), 12, torch.float32).cuda()
    want = torch.zeros((n, vocab, dim), device="cuda")
    T.embed_grad(tokens, dy, want)
    y = T.embed(tokens, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = torch.ones_like(want)
        T.embed_grad(tokens, dy, got)
        out = T.embed(tokens, got)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(out, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        T.embed_grad(tokens, dy, got)
        T.embed(tokens, got, out=out)
    for replay in range(3):
        got.fill_(replay + 5.0)
        out.fill_(-1.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(out, y), replay
        T.embed_grad(tokens, 2 * dy, torch.empty_like(want))        # eager work between the replays
        torch.cuda.synchronize()


def test_arguments_are_checked():
    tokens = torch.zeros((2, 3), dtype=torch.int64, device="cuda")
    table = torch.zeros((2, 5, 4), device="cuda")
    for bad in (lambda: T.embed(tokens.float(), table), lambda: T.embed(tokens, table.double()), lambda: T.embed(tokens[:1], table),
                lambda: T.embed(tokens, table.transpose(1, 2)), lambda: T.embed(tokens.cpu(), table),
                lambda: T.embed_grad(tokens, table, table), lambda: T.embed_grad(tokens, table[:, :3], table.bfloat16())):
        with pytest.raises(AssertionError):
            bad()
    with pytest.raises(B.ChocoError):
        T.embed(tokens[:, :1].expand(2, 3).contiguous(), table, out=torch.zeros((2, 1, 4), device="cuda").expand(2, 3, 4))
