"""The gates' gradient of linear attention, dg_t = e^g_t <E_t, S_{t-1}>, against 64 bits step by step: it is as near for a gate that is almost
closed as for an open one.

Tolerances.  With S and E of the same formulas on absolute values, what goes past a step has the magnitude M_t = e^g_t <|E_t|, |S_{t-1}|>.  A
product that counts in it goes through fewer than dk + dv + steps + 64 additions and products in fp32 on its way (rows with rows, states, steps
of a chunk), and its weight, 2^x with |x| < 127 of a rounded x, is off by less than 128 2^-24: together terms 2^-24 M_t.  Where operands are
numbers of 16 bits, states enter as pieces that leave at most 2^-22 of them, twice.  Weights, and states by them, that are less than 2^-126, fp32's
least normal number, are nothing: of what would pass with all gates open, 2^-120 at most.
With inputs that are not negative M_t is dg_t itself, and the bound a relative one."""
import pytest
import torch

from paper_1907_09356_amd import train as T
from tests.test_gpu_linear_attention import BF16, F16, F32, make, reference, whole

pytestmark = pytest.mark.gpu


def check_gates(q, k, v, g, h0, lengths, dy, dlast, relative=None):
    B, N, H = q.shape[0], q.shape[1], g.shape[-1]
    n = whole(lengths, B, N)
    exact = reference(q, k, v, g, h0, n, dy, dlast)
    if min(float(x.min()) for x in (q, k, v, h0, dy, dlast)) >= 0:
        size = exact["steps_dg"]
    else:
        size = reference(q.abs(), k.abs(), v.abs(), g, h0.abs(), n, dy.abs(), dlast.abs())["steps_dg"]
    opened = reference(q.abs(), k.abs(), v.abs(), torch.zeros_like(g), h0.abs(), n, dy.abs(), dlast.abs())["steps_dg"]
    saved = T.linear_attention(q, k, v, g, h0=h0, lengths=lengths, save=True)[2]
    dg = T.linear_attention_grad(q, k, v, g, saved, dy, lengths=lengths, dlast=dlast)[3]
    part = (q.shape[3] + v.shape[3] + N + 192) * 2.0 ** -24 + (0.0 if q.dtype == F32 else 2.0 ** -21)
    want = exact["steps_dg"]
    if g.dim() == 1:
        want, size, opened = (x.sum((0, 1)) for x in (want, size, opened))
    allowed = part * size + 2.0 ** -120 * opened
    off = (dg.double() - want).abs()
    assert bool((off <= allowed).all()), (float((off / allowed).max()), off.max().item())
    if relative:      # the bound says something: nothing at all would not pass
        assert float(allowed.norm()) <= relative * float(want.norm())


def positive(args):
    q, k, v, g, h0, lengths, dy, dlast = args
    return q.abs(), k.abs(), v.abs(), g, h0.abs(), lengths, dy.abs(), dlast.abs()


@pytest.mark.parametrize("value", [-0.05, -1.0, -5.0, -10.0, -20.0, -50.0, -80.0])
@pytest.mark.parametrize("N", [2, 3, 8, 40, 64, 65, 130, 257, 600])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_gates_that_let_little_through(value, N, dtype):
    q, k, v, g, h0, _, dy, dlast = make(2, N, 2, 32, 24, dtype, seed=N)
    args = q, k, v, torch.full_like(g, value), h0, None, dy, dlast
    near = value < -60      # e^-80 is 2^-115, and 2^-120 of what open gates let through no small part of what goes through it
    check_gates(*args, relative=None if near else 0.1)
    check_gates(*positive(args), relative=None if near else 1e-3)


@pytest.mark.parametrize("N", [3, 8, 50, 70, 200, 256, 300, 1025])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_closed_gates_among_open_ones(N, dtype):
    # each gate is open, nearly closed, or lets nothing through
    q, k, v, g, h0, lengths, dy, dlast = make(3, N, 2, 24, 40, dtype, seed=N + 1, ragged=True)
    gen = torch.Generator(device="cuda").manual_seed(N)
    kind = torch.rand(g.shape, device="cuda", generator=gen)
    g = torch.where(kind < 0.04, -30.0, torch.where(kind < 0.06, -8.0, torch.where(kind < 0.07, -torch.inf, -0.002)))
    args = q, k, v, g, h0, lengths, dy, dlast
    check_gates(*args)
    check_gates(*positive(args), relative=1e-3)


@pytest.mark.parametrize("at", [0, 1, 63, 64, 100, 127, 128, 191, 192, 255, 256, 319, 511, 599])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_closed_gate_wherever_it_is(at, dtype):
    # what passes it comes from steps of its tile, its chunk, its piece of 256 steps and from beyond on either side
    q, k, v, g, h0, _, dy, dlast = make(1, 600, 2, 40, 16, dtype, seed=at)
    g = torch.full_like(g, -2.0 ** -9)
    g[:, at] = -25.0
    args = q, k, v, g, h0, None, dy, dlast
    check_gates(*args)
    check_gates(*positive(args), relative=1e-3)


@pytest.mark.parametrize("dk, dv", [(1, 1), (50, 50), (64, 130), (130, 64), (128, 128), (129, 31), (256, 200), (7, 256)])
@pytest.mark.parametrize("N", [2, 5, 100, 330])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes_of_heads(dk, dv, N, dtype):
    q, k, v, g, h0, lengths, dy, dlast = make(2, N, 2, dk, dv, dtype, seed=dk + dv, ragged=True)
    if dtype == F16:
        dy, dlast = dy / 16, dlast / 16
    args = q, k, v, g, h0, lengths, dy, dlast
    check_gates(*args)
    check_gates(*positive(args), relative=1e-3)


@pytest.mark.parametrize("heads", [(6, 6, 6), (1, 1, 1), (2, 2, 6), (6, 3, 3), (1, 6, 2)])
@pytest.mark.parametrize("gate", ["step", "head"])
@pytest.mark.parametrize("N", [3, 90, 300])
def test_shared_heads_and_ragged_batches(heads, gate, N):
    for dtype in (F32, BF16):
        q, k, v, g, h0, _, dy, dlast = make(5, N, 6, 24, 40, dtype, seed=sum(heads), heads=heads, gate=gate)
        lengths = torch.tensor([0, 1, N, N // 2, N - 1], dtype=torch.int32, device="cuda")
        args = q, k, v, g, h0, lengths, dy, dlast
        check_gates(*args)
        check_gates(*positive(args), relative=1e-3)


@pytest.mark.parametrize("N", [1, 8, 64, 100, 515])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_a_first_state_or_a_gradient_of_the_last(N, dtype):
    q, k, v, g, h0, lengths, dy, dlast = make(3, N, 2, 33, 20, dtype, seed=N, ragged=True)
    zero = torch.zeros_like(h0)
    for first, last in ((None, dlast), (h0, None), (None, None)):
        saved = T.linear_attention(q, k, v, g, h0=first, lengths=lengths, save=True)[2]
        dg = T.linear_attention_grad(q, k, v, g, saved, dy, lengths=lengths, dlast=last)[3]
        saved = T.linear_attention(q, k, v, g, h0=zero if first is None else h0, lengths=lengths, save=True)[2]
        assert torch.equal(dg, T.linear_attention_grad(q, k, v, g, saved, dy, lengths=lengths, dlast=zero if last is None else dlast)[3])


@pytest.mark.parametrize("N", [1, 4, 60, 700])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_number_for_each_head_gathers_its_steps(N, dtype):
    # the same gates given step by step have the same gradients, whose sums of up to 256 steps are rounded once and added up in 64 bits
    q, k, v, g, h0, lengths, dy, dlast = make(3, N, 4, 24, 24, dtype, gate="head", ragged=True)
    both = []
    for gates in (g, g.expand(3, N, 4), g.expand(3, N, 4).contiguous()):
        saved = T.linear_attention(q, k, v, gates, h0=h0, lengths=lengths, save=True)[2]
        both.append(T.linear_attention_grad(q, k, v, gates, saved, dy, lengths=lengths, dlast=dlast)[3].double())
    assert torch.equal(both[1], both[2])
    assert bool(((both[0] - both[1].sum((0, 1))).abs() <= 2.0 ** -23 * both[1].abs().sum((0, 1))).all())


def test_values_that_are_not_finite_stay_in_their_sequence_and_head():
    for N in (6, 100, 400):
        q, k, v, g, h0, _, dy, dlast = make(2, N, 3, 16, 16, F32, seed=N)
        grads = []
        for bad in (False, True):
            k2 = k.clone()
            if bad:
                k2[1, N // 2, 1, 3] = torch.nan
            saved = T.linear_attention(q, k2, v, g, h0=h0, save=True)[2]
            grads.append(T.linear_attention_grad(q, k2, v, g, saved, dy, dlast=dlast)[3])
        keep = torch.ones_like(g, dtype=torch.bool)
        keep[1, :, 1] = False
        assert torch.equal(grads[0][keep], grads[1][keep]) and bool(grads[1][1, N // 2 + 1:, 1].isnan().all())


@pytest.mark.parametrize("N", [2, 8, 70, 600])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("heads", [(4, 4, 4), (2, 1, 4), (4, 4, 1)])
def test_the_other_gradients_do_not_depend_on_whether_the_gates_is_asked_for(heads, dtype, N):
    q, k, v, g, h0, lengths, dy, dlast = make(3, N, 4, 40, 24, dtype, heads=heads, ragged=True)
    saved = T.linear_attention(q, k, v, g, h0=h0, lengths=lengths, save=True)[2]
    want = T.linear_attention_grad(q, k, v, g, saved, dy, lengths=lengths, dlast=dlast)
    got = [torch.zeros_like(x) for x in (q.contiguous(), k.contiguous(), v.contiguous())]
    dh0 = torch.zeros_like(h0)
    cfg, nbytes, _ = T._linear_config(1, g, (q, k, v, dy, *got))
    workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
    T._enqueue(q, "choco_linear_backward", cfg, q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(), lengths.data_ptr(), saved.data_ptr(),
               dy.data_ptr(), dlast.data_ptr(), *(x.data_ptr() for x in got), None, dh0.data_ptr(), workspace.data_ptr(), nbytes)
    for name, a, b in zip(("dq", "dk", "dv", "dh0"), got + [dh0], want[:3] + want[4:]):
        assert torch.equal(a, b), name


@pytest.mark.parametrize("N", [5, 40, 300])
@pytest.mark.parametrize("gate", ["step", "head"])
def test_captured_and_replayed_beside_eager_calls(N, gate):
    q, k, v, g, h0, lengths, dy, dlast = make(3, N, 2, 32, 64, F32, gate=gate, ragged=True)
    other = make(3, N, 2, 32, 64, F32, gate=gate, seed=8)

    def work(q, k, v, g, h0, lengths, dy, dlast):
        saved = T.linear_attention(q, k, v, g, h0=h0, lengths=lengths, save=True)[2]
        return T.linear_attention_grad(q, k, v, g, saved, dy, lengths=lengths, dlast=dlast)

    want = [x.clone() for x in work(q, k, v, g, h0, lengths, dy, dlast)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        work(q, k, v, g, h0, lengths, dy, dlast)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = work(q, k, v, g, h0, lengths, dy, dlast)
    for _ in range(3):
        for x in got:
            x.zero_()
        work(*other)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_rows_far_apart():
    # 2^26 entries: the last begins beyond 2^32 bytes
    N, gap = 33, 1 << 26
    flat = torch.zeros(N * gap, dtype=BF16, device="cuda")
    q, k, v, g, h0, _, dy, dlast = make(1, N, 1, 16, 24, BF16)
    saved = T.linear_attention(q, k, v, g, h0=h0, save=True)[2]
    want = T.linear_attention_grad(q, k, v, g, saved, dy, dlast=dlast)
    for i in range(4):
        parts = [q, k, v, dy]
        far = flat.as_strided(parts[i].shape, (0, gap, parts[i].shape[3], 1))
        far.copy_(parts[i])
        parts[i] = far
        got = T.linear_attention_grad(*parts[:3], g, saved, parts[3], dlast=dlast)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
