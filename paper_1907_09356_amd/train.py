"""ctypes binding of include/choco_train.h: embedding lookup and gradient, gated linear recurrence, AdamW.

Argument marshalling only, like `binding`: torch provides device memory and the stream, every computation runs in the
HIP library.  Functions and methods enqueue on torch's current stream of the tensors' device.  As with torch's own operations, work of
one stream that needs that of another has to wait for it, and a tensor that is used on another stream than the one it was
made on has to be kept until that stream is done with it (an `AdamW` sees to its own workspace).  Nothing here is recorded by
torch's automatic differentiation: results do not require a gradient, and the gradients are calls of their own.
"""
import ctypes
import functools

import numpy as np
import torch

from . import binding
from .binding import _check

F32, BF16, F16 = 0, 1, 2
I32, I64 = 0, 1
SAVE_STEPS, BLOCK = 8, 256
TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
TOKEN_TYPES = {torch.int32: I32, torch.int64: I64}

EXPORTS = [
    "choco_embed_workspace_bytes", "choco_embed_forward", "choco_embed_backward", "choco_recur_saved_bytes",
    "choco_recur_workspace_bytes", "choco_recur_forward", "choco_recur_backward", "choco_adamw_workspace_bytes",
    "choco_adamw_init", "choco_adamw_step", "choco_adamw_moments", "choco_adamw_state", "choco_adamw_set_stream",
    "choco_adamw_get_step", "choco_adamw_set_step", "choco_adamw_destroy", "choco_train_last_hip_error",
]

_i32, _i64, _u64, _f32, _f64 = ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_float, ctypes.c_double
_vp, _size = ctypes.c_void_p, ctypes.c_size_t


class EmbedConfig(ctypes.Structure):
    _fields_ = [("n", _i32), ("tokens", _i64), ("vocab", _i64), ("dim", _i64), ("token_type", _i32), ("table_type", _i32),
                ("row_type", _i32), ("token_stride", _i64), ("table_stride", _i64), ("row_stride", _i64), ("row_ld", _i64),
                ("scale", _f32), ("stream", _vp)]


class RecurConfig(ctypes.Structure):
    _fields_ = [("batch", _i64), ("steps", _i64), ("dim", _i64), ("type", _i32)] + [
        (name + "_stride", _i64 * 2) for name in ("f", "u", "o", "y", "df", "du", "do")] + [("stream", _vp)]


class AdamwConfig(ctypes.Structure):
    _fields_ = [("n", _i32), ("d", _i64), ("ld", _i64), ("ntensors", _i32), ("start_host", ctypes.POINTER(_i64)),
                ("len_host", ctypes.POINTER(_i64)), ("weight_decay_host", ctypes.POINTER(_f32)),
                ("lr_scale_host", ctypes.POINTER(_f32)), ("beta1", _f64), ("beta2", _f64), ("eps", _f64),
                ("state_bits", _i32), ("seed", _u64), ("stream", _vp)]


_lib = None


def lib():
    """The loaded HIP library.  Raises if it has not been built."""
    global _lib
    if _lib is None:
        L = binding.lib()
        embed, recur, adamw, size = (ctypes.POINTER(t) for t in (EmbedConfig, RecurConfig, AdamwConfig, _size))
        L.choco_embed_workspace_bytes.argtypes = [embed, size]
        L.choco_embed_forward.argtypes = [embed, _vp, _vp, _vp]
        L.choco_embed_backward.argtypes = [embed, _vp, _vp, _vp, ctypes.c_int, _vp, _size]
        L.choco_recur_saved_bytes.argtypes = [recur, size]
        L.choco_recur_workspace_bytes.argtypes = [recur, size]
        L.choco_recur_forward.argtypes = [recur] + [_vp] * 9 + [_size]
        L.choco_recur_backward.argtypes = [recur] + [_vp] * 12 + [_size]
        L.choco_adamw_workspace_bytes.argtypes = [adamw, size]
        L.choco_adamw_init.argtypes = [adamw, _vp, _vp, _size, ctypes.POINTER(_vp)]
        L.choco_adamw_step.argtypes = [_vp, _vp, _i32, _f32, _vp]
        L.choco_adamw_moments.argtypes = [_vp, _vp, _vp]
        L.choco_adamw_state.argtypes = [_vp, ctypes.POINTER(_vp), size]
        L.choco_adamw_set_stream.argtypes = [_vp, _vp]
        L.choco_adamw_get_step.argtypes = [_vp, ctypes.POINTER(_u64)]
        L.choco_adamw_set_step.argtypes = [_vp, _u64]
        L.choco_adamw_destroy.argtypes = [_vp]
        L.choco_train_last_hip_error.argtypes = []
        for name in EXPORTS:
            getattr(L, name).restype = ctypes.c_int
        _lib = L
    return _lib


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(t):
    return torch._C._cuda_getCurrentRawStream(t.get_device())


_current_device = torch._C._cuda_getDevice


def _enqueue(t, name, *args):
    """A call of the library that works on t's device: made with that device current, as kernels go to the current one."""
    call, device = getattr(lib(), name), t.get_device()
    if device == _current_device():
        code = call(*args)
    else:
        with torch.cuda.device(device):
            code = call(*args)
    if code:
        _check(code, name)


def _scratch(nbytes, like):
    return torch.empty(nbytes, dtype=torch.uint8, device=like.device) if nbytes else None


def _planned(cfg, query):
    """A configuration by reference, and the bytes of workspace that `query` asks for it."""
    need = _size()
    _check(query(ctypes.byref(cfg), ctypes.byref(need)), query.__name__)
    return ctypes.byref(cfg), need.value


# ---- embedding ------------------------------------------------------------------------------------
@functools.lru_cache(maxsize=512)
def _embed_plan(token_shape, token_stride, token_type, table_shape, table_stride, table_type, row_shape, row_stride, row_type,
                scale, stream):
    """The configuration of a call, by what of its tensors goes into it."""
    assert len(token_shape) == 2 and len(table_shape) == 3 and len(row_shape) == 3
    assert token_type in TOKEN_TYPES and table_type in TYPES and row_type in TYPES
    (n, count), (tables, vocab, dim) = token_shape, table_shape
    assert tables == n and row_shape == (n, count, dim)
    assert count <= 1 or token_stride[1] == 1
    assert (dim <= 1 or table_stride[2] == 1) and (vocab <= 1 or table_stride[1] == dim)   # rows of a table lie one behind the other
    assert dim <= 1 or row_stride[2] == 1
    row_ld = row_stride[1] if count > 1 else dim
    return _planned(EmbedConfig(n=n, tokens=count, vocab=vocab, dim=dim, token_type=TOKEN_TYPES[token_type],
                                table_type=TYPES[table_type], row_type=TYPES[row_type],
                                token_stride=token_stride[0] if n > 1 else count,
                                table_stride=table_stride[0] if n > 1 else vocab * dim,
                                row_stride=row_stride[0] if n > 1 else count * row_ld, row_ld=row_ld, scale=scale,
                                stream=stream), lib().choco_embed_workspace_bytes)


def _embed_config(tokens, table, rows, scale):
    assert tokens.is_cuda and table.get_device() == rows.get_device() == tokens.get_device()
    return _embed_plan(tokens.shape, tokens.stride(), tokens.dtype, table.shape, table.stride(), table.dtype, rows.shape,
                       rows.stride(), rows.dtype, scale, _stream(tokens))


def embed(tokens, table, scale=1.0, out_dtype=None, out=None):
    """scale * table[w, tokens[w, r]] for every worker w: (n, R, dim).

    tokens (n, R) of int32 or int64, zero rows for those outside [0, vocab); table (n, vocab, dim), e.g. a tensor's slice of the
    workers' rows, `X[:, a:a + vocab * dim].view(n, vocab, dim)`."""
    if out is None:
        out = torch.empty(tokens.shape + table.shape[2:], dtype=out_dtype or table.dtype, device=table.device)
    cfg, _ = _embed_config(tokens, table, out, float(scale))
    _enqueue(out, "choco_embed_forward", cfg, tokens.data_ptr(), table.data_ptr(), out.data_ptr())
    return out


def embed_grad(tokens, dout, dtable, scale=1.0, accumulate=False):
    """The gradient of `embed` with respect to its table, written (or added) to dtable (n, vocab, dim) of float32,
    e.g. a tensor's slice of the workers' gradient rows."""
    assert dtable.dtype == torch.float32
    cfg, nbytes = _embed_config(tokens, dtable, dout, float(scale))
    ws = _scratch(nbytes, dtable)
    _enqueue(dtable, "choco_embed_backward", cfg, tokens.data_ptr(), dout.data_ptr(), dtable.data_ptr(), 1 if accumulate else 0,
             _ptr(ws), nbytes)
    return dtable


# ---- gated linear recurrence ----------------------------------------------------------------------
@functools.lru_cache(maxsize=512)
def _recur_plan(shape, dtype, strides, stream):
    """The configuration of a call: strides of f, u, o, y (backward: dy), df, du, do, None for one that is not there."""
    assert len(shape) == 3 and dtype in TYPES
    assert shape[2] <= 1 or all(s is None or s[2] == 1 for s in strides)
    cfg = RecurConfig(batch=shape[0], steps=shape[1], dim=shape[2], type=TYPES[dtype], stream=stream)
    for name, s in zip(("f", "u", "o", "y", "df", "du", "do"), strides):
        if s is not None:
            getattr(cfg, name + "_stride")[:] = s[:2]
    return _planned(cfg, lib().choco_recur_workspace_bytes)


def _recur_config(f, *tensors):
    device, dtype, shape = f.get_device(), f.dtype, f.shape
    strides = [f.stride()]
    for t in tensors:
        if t is not None:
            assert t.dtype == dtype and t.shape == shape and t.get_device() == device
            t = t.stride()
        strides.append(t)
    return _recur_plan(shape, dtype, tuple(strides), _stream(f))


def _state(t, f):
    """The address of a state of every sequence, or None."""
    if t is None:
        return None
    assert t.get_device() == f.get_device() and t.dtype == torch.float32 and t.is_contiguous() and t.shape == f.shape[::2]
    return t.data_ptr()


def _lengths(t, f):
    if t is None:
        return None
    assert t.get_device() == f.get_device() and t.dtype == torch.int32 and t.is_contiguous() and t.shape == f.shape[:1]
    return t.data_ptr()


def recurrence(f, u, o=None, h0=None, lengths=None, save=False, out=None, h_last=None):
    """h_t = a_t h_{t-1} + (1 - a_t) u_t with a = sigmoid(f), y = sigmoid(o) h (or h): (y, last states, saved).

    f, u, o (batch, steps, dim) of one type, strided as they come (columns of one projection); h0 (batch, dim) of
    float32, zero without; lengths (batch,) of int32.  save: keep what `recurrence_grad` needs (else None is returned).
    h_last may be h0 itself, as in token by token generation."""
    assert f.is_cuda
    B, T, C = f.shape
    y = f.new_empty((B, T, C)) if out is None else out
    if h_last is None:
        h_last = torch.empty((B, C), dtype=torch.float32, device=f.device) if h0 is None else torch.empty_like(h0)
    saved = None
    if save:
        saved = torch.empty(((T + SAVE_STEPS - 1) // SAVE_STEPS, B, C), dtype=torch.float32, device=f.device)
    cfg, nbytes = _recur_config(f, u, o, y)
    ws = _scratch(nbytes, f)
    _enqueue(f, "choco_recur_forward", cfg, f.data_ptr(), u.data_ptr(), _ptr(o), _state(h0, f), _lengths(lengths, f), y.data_ptr(),
             _state(h_last, f), _ptr(saved), _ptr(ws), nbytes)
    return y, h_last, saved


def recurrence_grad(f, u, saved, dy, o=None, lengths=None, dlast=None):
    """Backward pass of `recurrence`: (df, du, do or None, dh0), the first three columns of one matrix.

    saved as `recurrence(..., save=True)` returned it; dlast the gradient of the last states, zero without."""
    assert f.is_cuda
    B, T, C = f.shape
    assert saved.get_device() == f.get_device() and saved.dtype == torch.float32 and saved.is_contiguous()
    assert saved.shape == ((T + SAVE_STEPS - 1) // SAVE_STEPS, B, C)
    parts = 2 if o is None else 3
    grads = torch.empty((B, T, parts, C), dtype=f.dtype, device=f.device).unbind(2)
    df, du, do = grads[0], grads[1], None if o is None else grads[2]
    dh0 = torch.empty((B, C), dtype=torch.float32, device=f.device)
    cfg, nbytes = _recur_config(f, u, o, dy, df, du, do)
    ws = _scratch(nbytes, f)
    _enqueue(f, "choco_recur_backward", cfg, f.data_ptr(), u.data_ptr(), _ptr(o), _lengths(lengths, f), saved.data_ptr(),
             dy.data_ptr(), _state(dlast, f), df.data_ptr(), du.data_ptr(), _ptr(do), dh0.data_ptr(), _ptr(ws), nbytes)
    return df, du, do, dh0


# ---- AdamW ----------------------------------------------------------------------------------------
def make_adamw_config(n, d, ld=0, tensors=None, weight_decay=None, lr_scale=None, betas=(0.9, 0.999), eps=1e-8, state_bits=32,
                      seed=0, stream=None):
    """Fill a choco_adamw_config.  Returns (config, keepalive) as `binding.make_config` does.  tensors = (start, length)
    arrays; weight_decay and lr_scale a number or one per tensor."""
    cfg = AdamwConfig(n=int(n), d=int(d), ld=int(ld), beta1=float(betas[0]), beta2=float(betas[1]), eps=float(eps),
                      state_bits=int(state_bits), seed=int(seed), stream=stream)
    keep = []

    def array(values, dtype, kind):
        a = np.ascontiguousarray(values, dtype=dtype)
        keep.append(a)
        return a.ctypes.data_as(ctypes.POINTER(kind))

    count = 1
    if tensors is not None:
        start, length = tensors[0], tensors[1]
        assert len(start) == len(length)
        cfg.ntensors = count = len(start)
        cfg.start_host, cfg.len_host = array(start, np.int64, _i64), array(length, np.int64, _i64)
    if weight_decay is not None:
        cfg.weight_decay_host = array(np.broadcast_to(weight_decay, (count,)), np.float32, _f32)
    if lr_scale is not None:
        cfg.lr_scale_host = array(np.broadcast_to(lr_scale, (count,)), np.float32, _f32)
    return cfg, tuple(keep)


class AdamW:
    """AdamW on the parameter rows X (n, ld) of all workers, in place: `step` takes the place of a local update, a gossip
    step of `binding.Choco` on the same X may follow.  tensors: (start, length) arrays, e.g. the first two of a layer table;
    the whole row is one without."""

    def __init__(self, X, d, tensors=None, **kw):
        assert X.is_cuda and X.dtype == torch.float32 and X.is_contiguous() and X.dim() == 2
        self.X, self.d, self.stream = X, int(d), _stream(X)
        self.cfg, keep = make_adamw_config(X.shape[0], d, X.shape[1], tensors, stream=self.stream, **kw)
        need, a = _size(), _vp()
        _check(lib().choco_adamw_workspace_bytes(ctypes.byref(self.cfg), ctypes.byref(need)), "choco_adamw_workspace_bytes")
        self.workspace = torch.empty(need.value + 256, dtype=torch.uint8, device=X.device)
        base = (self.workspace.data_ptr() + 255) // 256 * 256
        _enqueue(X, "choco_adamw_init", ctypes.byref(self.cfg), _ptr(X), base, need.value, ctypes.byref(a))
        del keep
        self.handle = a

    def close(self):
        if getattr(self, "handle", None):
            lib().choco_adamw_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _follow(self):
        """Takes the current stream for the next call; the workspace is then kept from reuse until that stream is done, too."""
        stream = _stream(self.X)
        if stream != self.stream:
            self.workspace.record_stream(torch.cuda.current_stream(self.X.device))
            _check(lib().choco_adamw_set_stream(self.handle, stream), "choco_adamw_set_stream")
            self.stream = stream

    def step(self, G, lr, grad_scale=None):
        """G: gradients (n, ld) of float32 or bfloat16; grad_scale: (n,) of float32 on the device, a factor for each
        worker's gradient (one that is not finite leaves the worker as it is)."""
        assert G.device == self.X.device and G.is_contiguous() and G.shape == self.X.shape and G.dtype in (torch.float32, torch.bfloat16)
        if grad_scale is not None:
            assert grad_scale.device == G.device and grad_scale.dtype == torch.float32
            assert grad_scale.is_contiguous() and grad_scale.shape == G.shape[:1]
        self._follow()
        _enqueue(self.X, "choco_adamw_step", self.handle, _ptr(G), TYPES[G.dtype], float(lr), _ptr(grad_scale))

    def moments(self):
        """(m, v) as they are now, float32 of (n, d), in 8 bits what the codes stand for."""
        m, v = torch.empty_like(self.X), torch.empty_like(self.X)
        self._follow()
        _enqueue(self.X, "choco_adamw_moments", self.handle, m.data_ptr(), v.data_ptr())
        return m[:, :self.d], v[:, :self.d]

    def state(self):
        """The moments as they are held, a view of bytes that moves with the next step: copy it (and `get_step`) to save a run,
        copy back to resume it.  In 32 bits it is m and then v, as choco_train.h says: to look at them without a copy."""
        p, count = _vp(), _size()
        _check(lib().choco_adamw_state(self.handle, ctypes.byref(p), ctypes.byref(count)), "choco_adamw_state")
        at = p.value - self.workspace.data_ptr()
        return self.workspace[at:at + count.value]

    def get_step(self):
        t = _u64()
        _check(lib().choco_adamw_get_step(self.handle, ctypes.byref(t)), "choco_adamw_get_step")
        return t.value

    def set_step(self, t):
        _check(lib().choco_adamw_set_step(self.handle, int(t)), "choco_adamw_set_step")
