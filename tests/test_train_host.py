"""Host-side checks of include/choco_train.h that need no GPU: exports, and refusals before any device work.
The pointers handed over are never dereferenced: a call that these tests expect to be refused returns before a launch,
one that they expect to pass has nothing to do."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_1907_09356_amd import binding as B
from paper_1907_09356_amd import train as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000     # an aligned address


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "choco_train.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(choco_[a-z_0-9]+)\s*\(", text)))
    raw = ctypes.CDLL(B.LIB_PATH)
    for name in names:
        assert hasattr(raw, name), "missing export " + name
    assert sorted(T.EXPORTS) == names


def test_structures_have_the_compilers_sizes():
    # (a field too many or of another width on one side shows here)
    source = ('#include "choco_train.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu", sizeof(choco_embed_config), '
              'sizeof(choco_recur_config), sizeof(choco_adamw_config)); return 0; }\n')
    import subprocess
    import tempfile
    with tempfile.TemporaryDirectory() as tmp:
        src, exe = os.path.join(tmp, "s.c"), os.path.join(tmp, "s")
        open(src, "w").write(source)
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"), src, "-o", exe])
        sizes = [int(v) for v in subprocess.check_output([exe]).split()]
    assert sizes == [ctypes.sizeof(T.EmbedConfig), ctypes.sizeof(T.RecurConfig), ctypes.sizeof(T.AdamwConfig)]


# ---- embedding ----
def embed_cfg(**over):
    kw = dict(n=2, tokens=5, vocab=100, dim=8, token_type=T.I64, table_type=T.F32, row_type=T.F32, token_stride=5,
              table_stride=800, row_stride=40, row_ld=8, scale=1.0)
    kw.update(over)
    return T.EmbedConfig(**kw)


def embed_codes(c, tokens=P, table=P, rows=P, accumulate=0, ws=P, nbytes=1 << 40):
    L = T.lib()
    return (L.choco_embed_forward(ctypes.byref(c), tokens, table, rows),
            L.choco_embed_backward(ctypes.byref(c), tokens, rows, table, accumulate, ws, nbytes))


@pytest.mark.parametrize("over", [
    dict(n=-1), dict(n=65536), dict(tokens=-1), dict(tokens=2 ** 31), dict(vocab=0), dict(vocab=2 ** 31), dict(dim=-1),
    dict(dim=2 ** 31), dict(token_type=2), dict(table_type=3), dict(row_type=-1), dict(token_stride=4), dict(table_stride=799),
    dict(row_stride=39), dict(row_ld=7), dict(table_stride=2 ** 60), dict(row_stride=2 ** 62),
])
def test_embed_refuses_bad_sizes(over):
    c = embed_cfg(**over)
    assert embed_codes(c) == (B.E_INVAL, B.E_INVAL)
    out = ctypes.c_size_t()
    assert T.lib().choco_embed_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_INVAL


def test_embed_refuses_bad_pointers():
    c = embed_cfg()
    for over in (dict(tokens=0), dict(table=0), dict(rows=0), dict(tokens=P + 4), dict(table=P + 2), dict(rows=P + 1)):
        assert embed_codes(c, **over) == (B.E_INVAL, B.E_INVAL), over
    assert T.lib().choco_embed_forward(None, P, P, P) == B.E_INVAL
    assert T.lib().choco_embed_workspace_bytes(ctypes.byref(c), None) == B.E_INVAL
    out = ctypes.c_size_t()
    for tokens in (5, 5000, 200_000):
        big = embed_cfg(tokens=tokens, token_stride=tokens, row_stride=8 * tokens)
        assert T.lib().choco_embed_workspace_bytes(ctypes.byref(big), ctypes.byref(out)) == B.OK
        if out.value:
            assert embed_codes(big, nbytes=out.value - 1)[1] == B.E_NOMEM
            assert embed_codes(big, ws=0)[1] == B.E_INVAL
            assert embed_codes(big, ws=P + 8)[1] == B.E_INVAL


def test_embed_with_nothing_to_do():
    assert embed_codes(embed_cfg(n=0), 0, 0, 0) == (B.OK, B.OK)
    assert embed_codes(embed_cfg(dim=0), 0, 0, 0) == (B.OK, B.OK)
    assert embed_codes(embed_cfg(tokens=0), 0, 0, 0, accumulate=1) == (B.OK, B.OK)
    assert embed_codes(embed_cfg(tokens=0), 0, 0, 0)[1] == B.E_INVAL       # the gradient would have to be cleared


# ---- recurrence ----
def recur_cfg(**over):
    kw = dict(batch=2, steps=5, dim=8, type=T.F32)
    strides = {name: (40, 8) for name in ("f", "u", "o", "y", "df", "du", "do")}
    for k, v in over.items():
        if k in strides:
            strides[k] = v
        else:
            kw[k] = v
    return T.RecurConfig(**kw, **{k + "_stride": (ctypes.c_int64 * 2)(*v) for k, v in strides.items()})


def recur_codes(c, **over):
    p = dict(f=P, u=P, o=P, h0=P, lengths=P, y=P, last=P, saved=P, dy=P, dlast=P, df=P, du=P, do=P, dh0=P)
    p.update(over)
    L = T.lib()
    return (L.choco_recur_forward(ctypes.byref(c), p["f"], p["u"], p["o"], p["h0"], p["lengths"], p["y"], p["last"], p["saved"],
                                  P, 1 << 40),
            L.choco_recur_backward(ctypes.byref(c), p["f"], p["u"], p["o"], p["lengths"], p["saved"], p["dy"], p["dlast"],
                                   p["df"], p["du"], p["do"], p["dh0"], P, 1 << 40))


@pytest.mark.parametrize("over", [
    dict(batch=-1), dict(batch=2 ** 31), dict(steps=-1), dict(steps=2 ** 31), dict(dim=-1), dict(dim=2 ** 31), dict(type=3),
    dict(batch=2 ** 30, dim=2 ** 11), dict(batch=2 ** 30, steps=2 ** 11), dict(f=(-1, 8)), dict(u=(40, -8)), dict(o=(2 ** 61, 8)),
    dict(f=(2 ** 60, 2 ** 60)),
])
def test_recurrence_refuses_bad_sizes(over):
    assert recur_codes(recur_cfg(**over)) == (B.E_INVAL, B.E_INVAL)


def test_recurrence_refuses_outputs_whose_entries_share_a_place():
    assert recur_codes(recur_cfg(y=(40, 7)))[0] == B.E_INVAL        # (dy is only read)
    assert recur_codes(recur_cfg(y=(39, 8)))[0] == B.E_INVAL
    assert recur_codes(recur_cfg(y=(0, 8)))[0] == B.E_INVAL
    for name in ("df", "du", "do"):
        assert recur_codes(recur_cfg(**{name: (40, 7)}))[1] == B.E_INVAL
        assert recur_codes(recur_cfg(**{name: (15, 8)}))[1] == B.E_INVAL


def test_recurrence_refuses_bad_pointers():
    c = recur_cfg()
    for name in ("f", "u"):
        assert recur_codes(c, **{name: 0}) == (B.E_INVAL, B.E_INVAL)
    for name in ("f", "u", "o", "lengths", "saved"):
        assert recur_codes(c, **{name: P + 2}) == (B.E_INVAL, B.E_INVAL)
    for name in ("y",):
        assert recur_codes(c, **{name: 0})[0] == B.E_INVAL
    for name in ("h0", "last", "y"):
        assert recur_codes(c, **{name: P + 2})[0] == B.E_INVAL
    for name in ("saved", "dy", "df", "du", "do"):
        assert recur_codes(c, **{name: 0})[1] == B.E_INVAL
    for name in ("dy", "dlast", "df", "du", "do", "dh0"):
        assert recur_codes(c, **{name: P + 2})[1] == B.E_INVAL
    out = ctypes.c_size_t()
    assert T.lib().choco_recur_saved_bytes(None, ctypes.byref(out)) == B.E_INVAL
    assert T.lib().choco_recur_saved_bytes(ctypes.byref(c), None) == B.E_INVAL
    assert T.lib().choco_recur_workspace_bytes(ctypes.byref(c), None) == B.E_INVAL


def test_recurrence_refuses_a_small_workspace():
    c = recur_cfg(batch=1, steps=50_000, dim=64, **{k: (50_000 * 64, 64) for k in ("f", "u", "o", "y", "df", "du", "do")})
    out = ctypes.c_size_t()
    assert T.lib().choco_recur_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.OK
    if out.value:
        L = T.lib()
        for ws, nbytes, code in ((P, out.value - 1, B.E_NOMEM), (0, out.value, B.E_INVAL), (P + 4, out.value, B.E_INVAL)):
            assert L.choco_recur_forward(ctypes.byref(c), P, P, P, P, None, P, P, P, ws, nbytes) == code
            assert L.choco_recur_backward(ctypes.byref(c), P, P, P, None, P, P, P, P, P, P, P, ws, nbytes) == code


def test_more_than_a_launch_holds_is_unsupported():
    big = 2 ** 31 - 1
    out = ctypes.c_size_t()
    c = recur_cfg(batch=500, steps=big, dim=4096, **{k: (big * 4096, 4096) for k in ("f", "u", "o", "y", "df", "du", "do")})
    assert recur_codes(c) == (B.E_UNSUPPORTED, B.E_UNSUPPORTED)
    assert T.lib().choco_recur_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_UNSUPPORTED
    c = embed_cfg(n=1, tokens=big, vocab=10, dim=big, token_stride=big, table_stride=10 * big, row_stride=big * big, row_ld=big)
    assert embed_codes(c) == (B.E_INVAL, B.E_INVAL)                    # an array of more than 2^60 entries
    c = embed_cfg(n=1, tokens=2 ** 30, vocab=10, dim=2 ** 28, token_stride=2 ** 30, table_stride=10 * 2 ** 28, row_stride=2 ** 58,
                  row_ld=2 ** 28)
    assert embed_codes(c)[1] == B.E_UNSUPPORTED
    assert T.lib().choco_embed_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_UNSUPPORTED
    c = embed_cfg(n=1, tokens=2 ** 30, vocab=10, dim=64, token_stride=2 ** 30, row_stride=2 ** 36, row_ld=64)
    assert embed_codes(c)[0] == B.E_UNSUPPORTED


def test_kept_states_are_only_counted_for_what_a_launch_holds():
    big = 2 ** 31 - 1
    out = ctypes.c_size_t(7)
    for batch, steps, dim in ((511, big, big), (500, big, 4096), (1, big, 2 ** 20)):
        c = recur_cfg(batch=batch, steps=steps, dim=dim)
        assert T.lib().choco_recur_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_UNSUPPORTED
        assert T.lib().choco_recur_saved_bytes(ctypes.byref(c), ctypes.byref(out)) == B.E_UNSUPPORTED
    assert out.value == 7


def test_recurrence_with_nothing_to_do():
    assert recur_codes(recur_cfg(batch=0)) == (B.OK, B.OK)
    assert recur_codes(recur_cfg(dim=0)) == (B.OK, B.OK)
    out = ctypes.c_size_t(7)
    assert T.lib().choco_recur_saved_bytes(ctypes.byref(recur_cfg(steps=0)), ctypes.byref(out)) == B.OK and out.value == 0
    assert T.lib().choco_recur_saved_bytes(ctypes.byref(recur_cfg(steps=17)), ctypes.byref(out)) == B.OK
    assert out.value == -(-17 // T.SAVE_STEPS) * 2 * 8 * 4


# ---- AdamW ----
def adamw_code(n=2, d=1000, ld=0, x=P, ws=P, nbytes=1 << 40, **kw):
    c, keep = T.make_adamw_config(n, d, ld, **kw)
    need, a = ctypes.c_size_t(), ctypes.c_void_p(1)
    asked = T.lib().choco_adamw_workspace_bytes(ctypes.byref(c), ctypes.byref(need))
    if asked == B.OK:
        return asked
    rc = T.lib().choco_adamw_init(ctypes.byref(c), x, ws, nbytes, ctypes.byref(a))
    assert rc == asked and a.value is None
    return rc


@pytest.mark.parametrize("over", [
    dict(n=0), dict(n=65536), dict(d=0), dict(d=2 ** 31), dict(ld=996), dict(ld=1001), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)),
    dict(betas=(0.9, 1 - 1e-12)), dict(betas=(float("nan"), 0.9)), dict(eps=0.0), dict(eps=-1e-8), dict(eps=1e-60), dict(eps=float("inf")),
    dict(state_bits=16), dict(weight_decay=-0.1), dict(weight_decay=float("nan")), dict(lr_scale=float("inf")),
    dict(tensors=([0, 3], [4, 5])), dict(tensors=([0, 990], [4, 11])), dict(tensors=([-1], [4])), dict(tensors=([0], [-1])),
    dict(tensors=([500, 0], [10, 10])), dict(tensors=([2 ** 62], [2 ** 62])),
])
def test_adamw_refuses_bad_configurations(over):
    assert adamw_code(**over) == B.E_INVAL


@pytest.mark.parametrize("beta2", [0.0, 0.9, 0.999, 0.99999])
def test_adamw_refuses_an_eps_that_the_second_moments_range_outweighs(beta2):
    least = 2.0 ** -60 / (1 - beta2) ** 0.5
    for eps in (1e-39, 1e-30, least / 2, float("nan")):
        assert adamw_code(betas=(0.9, beta2), eps=eps) == B.E_INVAL
    for eps in (least, 1e-15, 1e-8):
        assert adamw_code(betas=(0.9, beta2), eps=eps) == B.OK


def test_adamw_accepts_any_disjoint_tensors():
    for bits in (32, 8):
        assert adamw_code(state_bits=bits) == B.OK
        assert adamw_code(state_bits=bits, tensors=([0, 1, 1, 999], [1, 0, 500, 1]), weight_decay=[0, 1, 2, 3]) == B.OK
        assert adamw_code(state_bits=bits, d=2 ** 31 - 2 ** 19) == B.OK
        assert adamw_code(state_bits=bits, tensors=([1000], [0])) == B.OK


def test_adamw_with_more_tensors_than_a_launch_holds_is_unsupported():
    # a tensor of one entry, a gap of one, ...: a tile each, of which a workgroup takes four
    for count, code in ((2 ** 25 + 1, B.E_UNSUPPORTED), (2 ** 25 - 8, B.OK)):
        assert adamw_code(d=2 * count, tensors=(np.arange(0, 2 * count, 2), np.ones(count, dtype=np.int64))) == code


def test_adamw_workspace_in_bytes_per_entry():
    def need(bits):
        c, keep = T.make_adamw_config(4, 1 << 20, state_bits=bits)
        out = ctypes.c_size_t()
        assert T.lib().choco_adamw_workspace_bytes(ctypes.byref(c), ctypes.byref(out)) == B.OK
        return out.value / (4 << 20)
    assert 8.0 <= need(32) < 8.1
    assert 2.0 + 8 / 256 <= need(8) < 2.1


def test_adamw_refuses_bad_pointers():
    L = T.lib()
    c, keep = T.make_adamw_config(2, 1000)
    a = ctypes.c_void_p(1)
    need = ctypes.c_size_t()
    assert L.choco_adamw_workspace_bytes(ctypes.byref(c), ctypes.byref(need)) == B.OK
    assert L.choco_adamw_workspace_bytes(ctypes.byref(c), None) == B.E_INVAL
    assert L.choco_adamw_workspace_bytes(None, ctypes.byref(need)) == B.E_INVAL
    for x, ws, nbytes, code in ((0, P, need.value, B.E_INVAL), (P, 0, need.value, B.E_INVAL), (P + 4, P, need.value, B.E_INVAL),
                                (P, P + 16, need.value, B.E_INVAL), (P, P, need.value - 1, B.E_NOMEM)):
        assert L.choco_adamw_init(ctypes.byref(c), x, ws, nbytes, ctypes.byref(a)) == code and a.value is None
    assert L.choco_adamw_init(ctypes.byref(c), P, P, need.value, None) == B.E_INVAL
    t = ctypes.c_uint64()
    assert L.choco_adamw_step(None, P, T.F32, 0.1, None) == B.E_INVAL
    assert L.choco_adamw_moments(None, P, P) == B.E_INVAL
    assert L.choco_adamw_get_step(None, ctypes.byref(t)) == B.E_INVAL
    assert L.choco_adamw_set_step(None, 3) == B.E_INVAL
    assert L.choco_adamw_state(None, ctypes.byref(a), ctypes.byref(need)) == B.E_INVAL
    assert L.choco_adamw_destroy(None) == B.OK


def test_adamw_refuses_to_set_the_stream_of_nothing():
    assert T.lib().choco_adamw_set_stream(None, None) == B.E_INVAL


# ---- the binding's calls, written down instead of made ----
class OnDevice(torch.Tensor):
    """A tensor in host memory that says it is on a device."""
    is_cuda = True
    number = 0

    def get_device(self):
        return self.number


def on_device(t):
    return torch.Tensor._make_subclass(OnDevice, t)


@pytest.fixture
def calls(monkeypatch):
    """[(name, arguments)] of the library's calls; calls.current: the current stream; calls.devices: the device that was
    current at each."""
    class Calls(list):
        current, device = 0, 0

    made = Calls()
    made.devices = []

    class Device:
        def __init__(self, number):
            self.number = number

        def __enter__(self):
            self.before, made.device = made.device, self.number

        def __exit__(self, *error):
            made.device = self.before

    class Library:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, args))
                made.devices.append((name, made.device))
                return B.OK
            call.__name__ = name
            return call

    monkeypatch.setattr(T, "lib", Library)
    monkeypatch.setattr(T, "_stream", lambda t: made.current)
    monkeypatch.setattr(T, "_current_device", lambda: made.device, raising=False)
    monkeypatch.setattr(torch.cuda, "device", Device)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: on_device(empty(*a, **kw)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: made.current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: made.append(("record_stream", (t.data_ptr(), stream))),
                        raising=False)
    for plan in (T._embed_plan, T._recur_plan):
        plan.cache_clear()
    yield made
    for plan in (T._embed_plan, T._recur_plan):      # (made with a library that asks for no workspace)
        plan.cache_clear()


def test_an_optimiser_launches_on_the_stream_that_is_current(calls):
    X = on_device(torch.zeros((2, 64)))
    opt = T.AdamW(X, 60, state_bits=8)
    for current in (0, 7, 7, 9):
        calls.current = current
        for use in (lambda: opt.step(X, 0.1), opt.moments):
            before = len(calls)
            use()
            launch = [i for i, c in enumerate(calls) if c[0] in ("choco_adamw_step", "choco_adamw_moments")][-1]
            assert launch >= before
            streams = [c[1][1] for c in calls[:launch] if c[0] == "choco_adamw_set_stream"]
            assert (streams[-1] if streams else opt.cfg.stream or 0) == current
            if current != 0:        # the workspace's memory is not handed out again before that stream is done
                assert ("record_stream", (opt.workspace.data_ptr(), current)) in calls


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_are_not_the_state_itself(calls, bits):
    X = on_device(torch.zeros((2, 64)))
    opt = T.AdamW(X, 60, state_bits=bits)
    opt.moments()
    m, v = opt.moments()
    name, (handle, m_at, v_at) = calls[-1]
    assert name == "choco_adamw_moments" and (m_at, v_at) == (m.data_ptr(), v.data_ptr())
    own = opt.workspace.untyped_storage().data_ptr()
    assert own not in (m.untyped_storage().data_ptr(), v.untyped_storage().data_ptr())


@pytest.mark.parametrize("number,current", [(0, 0), (1, 0), (0, 1), (2, 2)])
def test_calls_are_made_with_the_tensors_device_current(calls, monkeypatch, number, current):
    monkeypatch.setattr(OnDevice, "number", number)
    calls.device = current
    tokens = on_device(torch.zeros((2, 3), dtype=torch.int64))
    table, rows = on_device(torch.zeros((2, 5, 4))), on_device(torch.zeros((2, 3, 4)))
    T.embed(tokens, table, out=rows)
    T.embed_grad(tokens, rows, table)
    state = on_device(torch.zeros((2, 4)))
    T.recurrence(rows, rows, h_last=state, out=rows)
    T.recurrence_grad(rows, rows, on_device(torch.zeros((1, 2, 4))), rows)
    X = on_device(torch.zeros((2, 64)))
    opt = T.AdamW(X, 60, state_bits=8)
    opt.step(X, 0.1)
    opt.moments()
    names = ["choco_embed_forward", "choco_embed_backward", "choco_recur_forward", "choco_recur_backward", "choco_adamw_init",
             "choco_adamw_step", "choco_adamw_moments"]
    at = [(name, device) for name, device in calls.devices if name in names]
    assert at == [(name, number) for name in names]
    assert calls.device == current
