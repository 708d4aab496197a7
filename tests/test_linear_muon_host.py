"""Host-side checks of linear attention, orthogonalised matrices and their optimiser that need no GPU: refusals before any
device work.  The pointers handed over are never dereferenced: a call that these tests expect to be refused returns before a launch,
one that they expect to pass has nothing to do."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

from paper_1907_09356_amd import binding as B
from paper_1907_09356_amd import train as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000     # an aligned address


def test_structures_have_the_compilers_sizes():
    source = ('#include "choco_train.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", sizeof(choco_linear_config), '
              'sizeof(choco_orthogonalize_config), sizeof(choco_muon_config)); return 0; }\n')
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "s.c"), os.path.join(tmp, "s")
        open(src, "w").write(source)
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"), src, "-o", exe])
        sizes = [int(v) for v in subprocess.check_output([exe]).split()]
    assert sizes == [ctypes.sizeof(T.LinearConfig), ctypes.sizeof(T.OrthogonalizeConfig), ctypes.sizeof(T.MuonConfig)]


# ---- linear attention ----
def linear_cfg(**over):
    kw = dict(batch=2, steps=5, heads=4, q_heads=2, k_heads=4, v_heads=1, dim_k=8, dim_v=6, type=T.F32, gate_steps=1)
    strides = dict(q=(80, 16, 8), k=(160, 32, 8), v=(30, 6, 6), y=(120, 24, 6), g=(20, 4, 1), dq=(80, 16, 8), dk=(160, 32, 8), dv=(30, 6, 6))
    for name, v in over.items():
        if name in strides:
            strides[name] = v
        else:
            kw[name] = v
    return T.LinearConfig(**kw, **{name + "_stride": (ctypes.c_int64 * 3)(*v) for name, v in strides.items()})


def linear_codes(c, nbytes=1 << 50, **over):
    p = dict(q=P, k=P, v=P, g=P, h0=P, lengths=P, y=P, last=P, saved=P, dy=P, dlast=P, dq=P, dk=P, dv=P, dg=P, dh0=P, ws=P)
    p.update(over)
    L = T.lib()
    return (L.choco_linear_forward(ctypes.byref(c), p["q"], p["k"], p["v"], p["g"], p["h0"], p["lengths"], p["y"], p["last"], p["saved"],
                                   p["ws"], nbytes),
            L.choco_linear_backward(ctypes.byref(c), p["q"], p["k"], p["v"], p["g"], p["lengths"], p["saved"], p["dy"], p["dlast"],
                                    p["dq"], p["dk"], p["dv"], p["dg"], p["dh0"], p["ws"], nbytes))


@pytest.mark.parametrize("over", [
    dict(batch=-1), dict(batch=2 ** 31), dict(steps=-1), dict(steps=2 ** 31), dict(heads=-1), dict(heads=3), dict(q_heads=0), dict(k_heads=3),
    dict(v_heads=-1), dict(q_heads=8), dict(dim_k=0), dict(dim_k=257), dict(dim_v=0), dict(dim_v=257), dict(type=3), dict(type=-1),
    dict(gate_steps=2), dict(batch=2 ** 22), dict(q=(-1, 16, 8)), dict(k=(160, -1, 8)), dict(v=(30, 6, -6)), dict(g=(20, -4, 1)),
    dict(q=(2 ** 61, 16, 8)), dict(v=(2 ** 60, 2 ** 60, 6)),
])
def test_linear_attention_refuses_bad_sizes(over):
    assert linear_codes(linear_cfg(**over)) == (B.E_INVAL, B.E_INVAL)


@pytest.mark.parametrize("over, codes", [
    (dict(y=(120, 24, 5)), 0), (dict(y=(120, 23, 6)), 0), (dict(y=(0, 24, 6)), 0), (dict(y=(24, 24, 6)), 0),
    (dict(dq=(80, 8, 8)), 1), (dict(dk=(160, 32, 7)), 1), (dict(dv=(29, 6, 6)), 1), (dict(dv=(0, 6, 6)), 1),
])
def test_linear_attention_refuses_outputs_that_overlap(over, codes):
    assert linear_codes(linear_cfg(**over))[codes] == B.E_INVAL


def test_linear_attention_refuses_bad_pointers():
    c = linear_cfg()
    for over in (dict(q=0), dict(k=0), dict(v=0), dict(g=0), dict(q=P + 2), dict(k=P + 1), dict(v=P + 2), dict(g=P + 2), dict(lengths=P + 1)):
        assert linear_codes(c, **over) == (B.E_INVAL, B.E_INVAL), over
    for over in (dict(y=0), dict(y=P + 2), dict(h0=P + 2), dict(last=P + 1), dict(saved=P + 2)):
        assert linear_codes(c, **over)[0] == B.E_INVAL, over
    for over in (dict(saved=0), dict(dy=0), dict(dq=0), dict(dk=0), dict(dv=0), dict(dq=P + 2), dict(dg=P + 2), dict(dh0=P + 1), dict(dlast=P + 2),
                 dict(ws=0), dict(ws=P + 4)):
        assert linear_codes(c, **over)[1] == B.E_INVAL, over
    L, out = T.lib(), ctypes.c_size_t()
    assert L.choco_linear_workspace_bytes(None, 0, ctypes.byref(out)) == B.E_INVAL
    assert L.choco_linear_workspace_bytes(ctypes.byref(c), 0, None) == B.E_INVAL
    assert L.choco_linear_saved_bytes(ctypes.byref(c), None) == B.E_INVAL
    for back, steps in ((0, 100_000), (1, 5), (1, 5000)):
        big = linear_cfg(steps=steps, **{k: (10 ** 7, 40, 8) for k in ("q", "k", "v", "y", "dq", "dk", "dv")})
        assert L.choco_linear_workspace_bytes(ctypes.byref(big), back, ctypes.byref(out)) == B.OK
        if out.value:
            assert linear_codes(big, nbytes=out.value - 1)[back] == B.E_NOMEM


def test_linear_attention_refuses_what_no_launch_holds():
    c = linear_cfg(batch=2 ** 21, steps=2 ** 30, **{k: (2 ** 38, 32, 8) for k in ("q", "k", "v", "y", "g", "dq", "dk", "dv")})
    assert linear_codes(c) == (B.E_UNSUPPORTED, B.E_UNSUPPORTED)
    out = ctypes.c_size_t()
    assert T.lib().choco_linear_saved_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_UNSUPPORTED
    assert T.lib().choco_linear_workspace_bytes(ctypes.byref(c), 0, ctypes.byref(out)) == B.E_UNSUPPORTED


def test_linear_attention_with_nothing_to_do():
    assert linear_codes(linear_cfg(batch=0)) == (B.OK, B.OK)
    assert linear_codes(linear_cfg(heads=0)) == (B.OK, B.OK)
    out = ctypes.c_size_t()
    for back in (0, 1):
        assert T.lib().choco_linear_workspace_bytes(ctypes.byref(linear_cfg(steps=0)), back, ctypes.byref(out)) == B.OK


def test_linear_attention_checks_its_tensors():
    q = torch.zeros(2, 5, 4, 8)
    for bad in (dict(g=torch.zeros(3)), dict(k=torch.zeros(2, 5, 4, 7)), dict(g=torch.zeros(4, dtype=torch.float64)), dict()):
        kw = dict(k=q, v=q, g=torch.zeros(4))
        kw.update(bad)
        with pytest.raises(AssertionError):
            T.linear_attention(q, **kw)


# ---- orthogonalised matrices ----
def stack_cfg(**over):
    kw = dict(batch=2, rows=6, cols=8, type=T.F32, iterations=5)
    strides = dict(x=(48, 8), y=(48, 8))
    for name, v in over.items():
        if name in strides:
            strides[name] = v
        else:
            kw[name] = v
    return T.OrthogonalizeConfig(**kw, **{name + "_stride": (ctypes.c_int64 * 2)(*v) for name, v in strides.items()})


@pytest.mark.parametrize("over", [
    dict(batch=-1), dict(batch=2 ** 31), dict(rows=-1), dict(rows=65537), dict(cols=-1), dict(cols=65537), dict(type=3), dict(iterations=0),
    dict(iterations=33), dict(x=(-1, 8)), dict(x=(48, -1)), dict(x=(2 ** 61, 8)), dict(y=(48, 7)), dict(y=(47, 8)), dict(y=(0, 8)), dict(y=(48, -8)),
])
def test_orthogonalize_refuses_bad_sizes(over):
    c, out = stack_cfg(**over), ctypes.c_size_t()
    assert T.lib().choco_orthogonalize(ctypes.byref(c), P, P, P, 1 << 50) == B.E_INVAL
    assert T.lib().choco_orthogonalize_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_INVAL


def test_orthogonalize_refuses_bad_pointers_and_does_nothing_where_nothing_is():
    L, c, out = T.lib(), stack_cfg(rows=300, cols=400, x=(120_000, 400), y=(120_000, 400)), ctypes.c_size_t()
    assert L.choco_orthogonalize_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.OK and out.value > 0
    for x, y, ws in ((0, P, P), (P, 0, P), (P, P, 0), (P + 2, P, P), (P, P + 2, P), (P, P, P + 128)):
        assert L.choco_orthogonalize(ctypes.byref(c), x, y, ws, out.value) == B.E_INVAL
    assert L.choco_orthogonalize(ctypes.byref(c), P, P, P, out.value - 1) == B.E_NOMEM
    assert L.choco_orthogonalize(None, P, P, P, 0) == B.E_INVAL
    for over in (dict(batch=0), dict(rows=0), dict(cols=0)):
        assert L.choco_orthogonalize(ctypes.byref(stack_cfg(**over)), 0, 0, 0, 0) == B.OK


def test_orthogonalize_checks_its_tensors():
    for bad in (torch.zeros(4, 4), torch.zeros(1, 4, 4)):       # no stack; not on a GPU
        with pytest.raises(AssertionError):
            T.orthogonalize(bad)


# ---- the optimiser ----
def muon_code(matrices=((0, 48), (6, 3), (8, 4)), n=2, d=64, ld=64, x=P, ws=P, nbytes=1 << 50, **kw):
    cfg, keep = T.make_muon_config(n, d, ld, matrices, **kw)
    out, a = ctypes.c_size_t(), ctypes.c_void_p()
    code = T.lib().choco_muon_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out))
    if code == B.OK:
        code = T.lib().choco_muon_init(ctypes.byref(cfg), x, ws, min(nbytes, out.value - (nbytes == -1)) if nbytes >= 0 else out.value - 1, ctypes.byref(a))
        assert a.value is None
    return code


@pytest.mark.parametrize("over", [
    dict(n=0), dict(n=65536), dict(d=0), dict(ld=63), dict(ld=62), dict(matrices=((0, 47), (6, 3), (8, 4))), dict(matrices=((0, 53), (6, 3), (8, 4))),
    dict(matrices=((-1,), (2,), (2,))), dict(matrices=((0,), (-1,), (2,))), dict(matrices=((0,), (2,), (-1,))), dict(matrices=((0,), (65537,), (1,))),
    dict(matrices=((), (), ())), dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")), dict(iterations=0), dict(iterations=33),
    dict(weight_decay=-1.0), dict(weight_decay=float("inf")), dict(lr_scale=float("nan")),
    dict(x=0), dict(x=P + 2), dict(ws=0), dict(ws=P + 128),
])
def test_muon_refuses(over):
    assert muon_code(**over) == B.E_INVAL


def test_muon_refuses_a_small_workspace_and_missing_handles():
    assert muon_code(nbytes=-1) == B.E_NOMEM
    L, p, count = T.lib(), ctypes.c_void_p(), ctypes.c_size_t()
    assert L.choco_muon_init(None, P, P, 0, None) == B.E_INVAL
    assert L.choco_muon_step(None, P, T.F32, 0.1, None) == B.E_INVAL
    assert L.choco_muon_state(None, ctypes.byref(p), ctypes.byref(count)) == B.E_INVAL
    assert L.choco_muon_set_stream(None, None) == B.E_INVAL
    assert L.choco_muon_destroy(None) == B.OK


def test_muon_workspace_is_bounded_by_rounds():
    # 64 workers' 4096 x 1024 matrices: operands of a round stay below 2 GB, the momenta are what grows
    sizes = []
    for n in (32, 64):
        cfg, keep = T.make_muon_config(n, 4096 * 1024, 4096 * 1024, ([0], [4096], [1024]))
        out = ctypes.c_size_t()
        assert T.lib().choco_muon_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out)) == B.OK
        sizes.append(out.value - n * 4096 * 1024 * 4)
    assert sizes[0] <= 1.01 * 2 ** 31 and abs(sizes[1] - sizes[0]) <= 2 ** 20
    assert np.isfinite(sizes).all()
