"""The launches of linear attention and of orthogonalised matrices, over a stand-in for the HIP runtime, without a GPU."""
import pytest

from tests.launches import recorded

HEAD = """
import ctypes
from paper_1907_09356_amd import train as T
P = 0x10000
def launches(code):
    assert code == B.OK, code
    rows = [line.split() for line in stub.stub_launches().decode().splitlines()]
    return [[name] + [[int(x) for x in dims.split("x")] for dims in (grid, block)] + [int(lds)] for name, grid, block, lds in rows]
"""


def run(code):
    return recorded(HEAD + code)


def fits(launch):
    return launch[1][0] * launch[2][0] < 2 ** 32


# ---- linear attention ----
LINEAR = """
def strides(steps, heads, dim):
    return (ctypes.c_int64 * 3)(steps * heads * dim, heads * dim, dim)
def linear(batch, steps, heads, dk, dv, kind, gate=1, q_heads=None, k_heads=None, v_heads=None):
    hq, hk, hv = q_heads or heads, k_heads or heads, v_heads or heads
    s = dict(q=(hq, dk), k=(hk, dk), v=(hv, dv), y=(heads, dv), g=(heads, 1), dq=(hq, dk), dk=(hk, dk), dv=(hv, dv))
    return T.LinearConfig(batch=batch, steps=steps, heads=heads, q_heads=hq, k_heads=hk, v_heads=hv, dim_k=dk, dim_v=dv, type=kind,
                          gate_steps=gate, **{name + "_stride": strides(steps, *v) for name, v in s.items()})
def forward(c, h0=P, last=P, saved=P):
    stub.stub_clear()
    return launches(T.lib().choco_linear_forward(ctypes.byref(c), P, P, P, P, h0, None, P, last, saved, P, 1 << 50))
def backward(c, saved=P, dlast=P, dg=P, dh0=P):
    stub.stub_clear()
    return launches(T.lib().choco_linear_backward(ctypes.byref(c), P, P, P, P, None, saved, P, dlast, P, P, P, dg, dh0, P, 1 << 50))
"""


@pytest.mark.parametrize("dk, dv", [(16, 24), (50, 50), (33, 7), (8, 1), (1, 8)])
@pytest.mark.parametrize("steps", [1, 3, 100])
def test_what_is_launched_depends_on_sizes_and_not_on_the_states_addresses(dk, dv, steps):
    # lanes' columns set the order of sums, so they may not follow from where a state lies
    out = run(LINEAR + """
c = linear(2, %d, 3, %d, %d, T.F32)
out = [[forward(c, P + a, P + b, P + e), backward(c, P + a, P + b, dh0=P + e)] for a, b, e in ((0, 0, 0), (4, 0, 0), (0, 4, 0), (0, 0, 4), (8, 8, 8))]
""" % (steps, dk, dv))
    for other in out[1:]:
        assert other == out[0]


# ---- orthogonalised matrices ----
@pytest.mark.parametrize("batch", [4_194_303, 4_194_304, 5_000_001, 16_777_215, 40_000_000])
def test_stacks_of_small_matrices_are_divided_where_a_launch_ends(batch):
    # a workgroup of 1024 threads takes a matrix, and a grid holds less than 2^32 threads
    out = run("""
c = T.OrthogonalizeConfig(batch=%d, rows=8, cols=8, type=T.F32, iterations=5, x_stride=(ctypes.c_int64 * 2)(64, 8), y_stride=(ctypes.c_int64 * 2)(64, 8))
out = launches(T.lib().choco_orthogonalize(ctypes.byref(c), P, P, None, 0))
""" % batch)
    assert all(name == "k_muon_whole<float,false>" and block == [1024, 1, 1] for name, _, block, _ in out)
    assert all(fits(launch) for launch in out)
    assert sum(grid[0] for _, grid, _, _ in out) == batch
    assert len(out) == 1 or len(out) <= 2 * -(-batch // (2 ** 22 - 1))


def test_rounds_of_many_small_matrices_are_divided_where_a_launch_ends():
    n, count = 65535, 70
    out = run("""
import numpy as np
n, count = %d, %d
cfg, keep = T.make_muon_config(n, 2 * count, 2 * count, (np.arange(count) * 2, [1] * count, [2] * count))
need, a = ctypes.c_size_t(), ctypes.c_void_p()
assert T.lib().choco_muon_workspace_bytes(ctypes.byref(cfg), ctypes.byref(need)) == B.OK
ws = np.zeros(need.value + 256, dtype=np.uint8)
base = (ws.ctypes.data + 255) // 256 * 256
assert T.lib().choco_muon_init(ctypes.byref(cfg), P, base, need.value, ctypes.byref(a)) == B.OK
out = launches(T.lib().choco_muon_step(a, P, T.F32, 0.1, None))
""" % (n, count))
    assert all(fits(launch) for launch in out)
    assert sum(grid[0] for _, grid, _, _ in out) == n * count


def test_the_shapes_that_are_compared_with_64_bits_take_every_form():
    from tests.test_gpu_newton_schulz import BOTH, LARGE, SIXTY_FOUR, WHOLE
    out = run("""
out = []
for batch, rows, cols in %s:
    c = T.OrthogonalizeConfig(batch=batch, rows=rows, cols=cols, type=T.F32, iterations=1, x_stride=(ctypes.c_int64 * 2)(rows * cols, cols),
                              y_stride=(ctypes.c_int64 * 2)(rows * cols, cols))
    stub.stub_clear()
    out.append([launch[0] for launch in launches(T.lib().choco_orthogonalize(ctypes.byref(c), P, P, P, 1 << 50))])
""" % (WHOLE + SIXTY_FOUR + LARGE + BOTH))
    forms = [["k_muon_whole<float,false>"]] * len(WHOLE)
    for shapes, gram, apply in ((SIXTY_FOUR, 64, 64), (LARGE, 128, 128), (BOTH, 64, 128)):
        forms += [["k_muon_squares<float,false>", "k_muon_start<float,false>", "k_muon_product<0,%d>" % gram, "k_muon_product<1,%d>" % gram,
                   "k_muon_product<2,%d>" % apply]] * len(shapes)
    assert out == forms, [(a, b) for a, b in zip(out, forms) if a != b]
