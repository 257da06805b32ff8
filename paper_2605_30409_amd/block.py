"""What stands around the recurrence in a block, and at the end of a training step
(include/gdn_block.h): the gated linear map of a feed-forward block and the short causal
convolution in front of the recurrence, both with their gradient and a form for decoding
batches, and the norm and clipping of all gradients.

Thin binding like :mod:`.ops`: argument checks and marshalling only.  Outputs and
workspaces that are not given are allocated on the stream the call runs on.  No call
records an autograd graph: results of inputs that require a gradient do not.  Tensors that
a call is given to write count as modified in place, and while gradients are recorded may not require
one.
"""
import ctypes

import torch

from . import gdn as _gdn
from .ops import _BF16, _F32, _I32, _Tensor, _call, _dims, _element, _fit, _given, _needs, _on, _ptr

ACTIVATIONS = {None: 0, "silu": 1, "gelu": 2, "gelu_tanh": 3}

_fns = None


def _lib():
    global _fns
    if _fns is None:
        L = _gdn.lib()
        vp, i, sz, fl, ll = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float, ctypes.c_int64
        L.gdn_gated_linear_workspace_bytes.restype = sz
        L.gdn_gated_linear_workspace_bytes.argtypes = [i] * 5
        L.gdn_gated_linear_forward.restype = i
        L.gdn_gated_linear_forward.argtypes = [vp] * 4 + [i] * 5 + [vp, sz, vp]
        L.gdn_gated_linear_backward.restype = i
        L.gdn_gated_linear_backward.argtypes = [vp] * 7 + [i] * 5 + [vp, sz, vp]
        L.gdn_short_conv_forward.restype = i
        L.gdn_short_conv_forward.argtypes = [vp, ll, ll] + [vp] * 5 + [i] * 6 + [vp]
        L.gdn_short_conv_workspace_bytes.restype = sz
        L.gdn_short_conv_workspace_bytes.argtypes = [i] * 4
        L.gdn_short_conv_backward.restype = i
        L.gdn_short_conv_backward.argtypes = [vp, ll, ll] + [vp] * 6 + [ll, ll] + [vp] * 3 + [i] * 6 + [vp, sz, vp]
        L.gdn_short_conv_step.restype = i
        L.gdn_short_conv_step.argtypes = [vp, ll, ll] + [vp] * 7 + [i] * 7 + [vp]
        L.gdn_grad_workspace_bytes.restype = sz
        L.gdn_grad_workspace_bytes.argtypes = [i]
        L.gdn_grad_norm.restype = i
        L.gdn_grad_norm.argtypes = [vp] * 3 + [i, vp, vp, sz, vp]
        L.gdn_grad_clip.restype = i
        L.gdn_grad_clip.argtypes = [vp] * 4 + [i, vp, vp, fl, fl, vp, sz, vp]
        _fns = L
    return _fns


def _act(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {list(ACTIVATIONS)}, got {name!r}") from None


def _sizes(text, *sizes):
    """Sizes that the C call takes in 32 bits."""
    if max(sizes) >= 1 << 31:
        raise ValueError(f"{text} must be below 2^31, got {list(sizes)}")


def _workspace(ws, need, dev):
    """The workspace given, checked, a new one, or None where none is needed."""
    if ws is None:
        return torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    if not isinstance(ws, _Tensor):
        raise TypeError(f"ws must be a tensor, got {type(ws).__name__}")
    if ws.device != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    return ws


# ---------------------------------------------------------------------------
# Gated linear map.

def _gated_inputs(x, w_gate, w_up):
    dt, dev = _element("x", x)
    if x.dim() < 1:
        raise ValueError("x must be [..., C], got []")
    rows = x.shape[:-1]
    F, C = _dims("w_gate", w_gate, 2, "[F, C]")
    M = rows.numel()
    if not (_fit(dev.index, dt, (*rows, C), x) and _fit(dev.index, dt, (F, C), w_gate, w_up)):
        _needs(dev, ("x", x, (*rows, C), dt), ("w_gate", w_gate, (F, C), dt), ("w_up", w_up, (F, C), dt))
    _sizes("rows, C and F", M, C, F)
    return dt, dev, rows, M, C, F


def gated_linear_workspace(x, w_gate, backward=False):
    """Workspace tensor for gated_linear (backward: gated_linear_backward) on inputs shaped like these; empty where none is
    needed."""
    F, C = _dims("w_gate", w_gate, 2, "[F, C]")
    M = x.shape[:-1].numel()
    _sizes("rows, C and F", M, C, F)
    n = _lib().gdn_gated_linear_workspace_bytes(M, C, F, 1 if x.dtype == _BF16 else 0, 1 if backward else 0)
    if n == 0 and backward:
        raise ValueError("unsupported shape for the gated linear map")
    return torch.empty(n, dtype=torch.uint8, device=x.device)


def gated_linear(x, w_gate, w_up, *, activation="silu", out=None, ws=None, stream=None):
    """The gated half of a feed-forward block, both projections, activation and product in one kernel:

        h = act(x w_gate^T) o (x w_up^T)

    x [..., C], w_gate and w_up [F, C] (two halves of one [2 F, C] weight, say), all bf16 or all fp32;
    activation "silu", "gelu", "gelu_tanh" or None.  Any number of rows; a decoding batch takes a kernel that
    streams the weights.  Returns h [..., F] like x."""
    if stream is not None:
        with _on(stream, x):
            return gated_linear(x, w_gate, w_up, activation=activation, out=out, ws=ws)
    dt, dev, rows, M, C, F = _gated_inputs(x, w_gate, w_up)
    written = ()
    if out is None:
        out = torch.empty((*rows, F), dtype=dt, device=dev)
    else:
        _needs(dev, ("out", out, (*rows, F), dt))
        written = (out,)
    bf16 = 1 if dt is _BF16 else 0
    need = (_fns or _lib()).gdn_gated_linear_workspace_bytes(M, C, F, bf16, 0)
    if need or ws is not None:
        ws = _workspace(ws, need, dev)
    _call("gdn_gated_linear_forward", dev, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), out.data_ptr(), M, C, F,
          _act(activation), bf16, _ptr(ws), 0 if ws is None else ws.numel(), written=written)
    return out


def gated_linear_backward(x, w_gate, w_up, dh, *, activation="silu", dx=None, dw_gate=None, dw_up=None, ws=None, stream=None):
    """Gradient of ``gated_linear`` from dh = dL/dh [..., F] like x, with the forward call's inputs; nothing
    else of that call is needed.  Returns (dx, dw_gate, dw_up), each like its input."""
    if stream is not None:
        with _on(stream, x):
            return gated_linear_backward(x, w_gate, w_up, dh, activation=activation, dx=dx, dw_gate=dw_gate, dw_up=dw_up, ws=ws)
    dt, dev, rows, M, C, F = _gated_inputs(x, w_gate, w_up)
    _needs(dev, ("dh", dh, (*rows, F), dt))
    written = [t for t in (dx, dw_gate, dw_up) if t is not None]
    dx = _given("dx", dx, x)
    dw_gate = _given("dw_gate", dw_gate, w_gate)
    dw_up = _given("dw_up", dw_up, w_up)
    bf16 = 1 if dt is _BF16 else 0
    ws = _workspace(ws, _lib().gdn_gated_linear_workspace_bytes(M, C, F, bf16, 1), dev)
    _call("gdn_gated_linear_backward", dev, x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), dh.data_ptr(), dx.data_ptr(),
          dw_gate.data_ptr(), dw_up.data_ptr(), M, C, F, _act(activation), bf16, _ptr(ws), 0 if ws is None else ws.numel(),
          written=written)
    return dx, dw_gate, dw_up


# ---------------------------------------------------------------------------
# Short convolution.

def _strided(name, t, shape, dt, dev):
    """[B, T, C] with whole rows: strides from sequence to sequence and from token to token, in elements (0 where there
    is no other)."""
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a tensor, got {type(t).__name__}")
    if t.dtype != dt:
        raise TypeError(f"{name} must have dtype {dt}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    B, T, C = shape
    sb, st, sc = t.stride()
    if sc != 1 and C > 1:
        raise ValueError(f"{name}'s channels must be next to each other, got strides {list(t.stride())}")
    return (sb if B > 1 else 0), (st if T > 1 else 0)


def _taps(w, bias, C, dev):
    Cw, W = _dims("w", w, 2, "[C, W]")
    if not _fit(dev.index, _F32, (C, W), w):
        _needs(dev, ("w", w, (C, W), _F32))
    if not 2 <= W <= 4:
        raise ValueError(f"w must have 2 to 4 taps, got {W}")
    if bias is not None and not _fit(dev.index, _F32, (C,), bias):
        _needs(dev, ("bias", bias, (C,), _F32))
    return W


def _conv_inputs(x, w, bias, state):
    dt, dev = _element("x", x)
    B, T, C = _dims("x", x, 3, "[B, T, C]")
    _sizes("B, T and C", B, T, C)
    xb, xt = _strided("x", x, x.shape, dt, dev)
    W = _taps(w, bias, C, dev)
    if state is not None:
        _needs(dev, ("state", state, (B, W - 1, C), dt))
    return dt, dev, B, T, C, W, xb, xt


def short_conv(x, w, bias=None, state=None, *, activation="silu", out=None, state_out=None, want_state=True, stream=None):
    """The short causal convolution of each channel in front of the recurrence, with its activation:

        y_t = act(bias + sum_i w[:, i] x_{t - W + 1 + i})

    x [B, T, C], bf16 or fp32, may be a part of a packed projection: its rows have to be whole, the
    strides from token to token and from sequence to sequence are free.  w [C, W] with 2 to 4 taps and bias [C] (or
    None) fp32; state [B, W - 1, C] like x holds the inputs before the first token (None: zeros).
    activation as in gated_linear.  Returns (y [B, T, C], state_out [B, W - 1, C]: the inputs before the next
    token; None without want_state).  state_out may be state."""
    if stream is not None:
        with _on(stream, x):
            return short_conv(x, w, bias, state, activation=activation, out=out, state_out=state_out, want_state=want_state)
    dt, dev, B, T, C, W, xb, xt = _conv_inputs(x, w, bias, state)
    written = [t for t in (out, state_out) if t is not None]
    if out is None:
        out = torch.empty((B, T, C), dtype=dt, device=dev)
    else:
        _needs(dev, ("out", out, (B, T, C), dt))
    if state_out is not None:
        _needs(dev, ("state_out", state_out, (B, W - 1, C), dt))
    elif want_state:
        state_out = torch.empty((B, W - 1, C), dtype=dt, device=dev)
    _lib()
    _call("gdn_short_conv_forward", dev, x.data_ptr(), xb, xt, w.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(),
          _ptr(state_out), B, T, C, W, _act(activation), 1 if dt is _BF16 else 0, written=written)
    return out, state_out


def short_conv_workspace(x, w):
    """Workspace tensor for short_conv_backward on inputs shaped like these."""
    B, T, C = _dims("x", x, 3, "[B, T, C]")
    _sizes("B, T and C", B, T, C)
    n = _lib().gdn_short_conv_workspace_bytes(B, T, C, w.shape[-1])
    if n == 0:
        raise ValueError("unsupported shape for the short convolution")
    return torch.empty(n, dtype=torch.uint8, device=x.device)


def short_conv_backward(x, w, bias, state, dy, dstate_out=None, *, activation="silu", dx=None, dw=None, dbias=None,
                        dstate=None, want_dstate=True, ws=None, stream=None):
    """Gradient of ``short_conv`` from dy = dL/dy [B, T, C] and dstate_out = dL/d(state_out) [B, W - 1, C], both like x
    (dstate_out None: zero), with the forward call's inputs (bias and state may be None there and here).  dx, if given,
    may be a part of a packed gradient, [B, T, ..] or [T, B, ..] in memory.  Returns (dx, dw [C, W] fp32, dbias [C] fp32
    or None without bias, dstate [B, W - 1, C] like x or None without want_dstate)."""
    if stream is not None:
        with _on(stream, x):
            return short_conv_backward(x, w, bias, state, dy, dstate_out, activation=activation, dx=dx, dw=dw, dbias=dbias,
                                       dstate=dstate, want_dstate=want_dstate, ws=ws)
    dt, dev, B, T, C, W, xb, xt = _conv_inputs(x, w, bias, state)
    _needs(dev, ("dy", dy, (B, T, C), dt))
    if dstate_out is not None:
        _needs(dev, ("dstate_out", dstate_out, (B, W - 1, C), dt))
    written = [t for t in (dx, dw, dbias, dstate) if t is not None]
    if dx is None:
        dx = torch.empty((B, T, C), dtype=dt, device=dev)
    ob, ot = _strided("dx", dx, (B, T, C), dt, dev)
    dw = _given("dw", dw, w)
    if bias is not None:
        dbias = _given("dbias", dbias, bias)
    elif dbias is not None:
        raise ValueError("dbias without bias")
    if dstate is not None:
        _needs(dev, ("dstate", dstate, (B, W - 1, C), dt))
    elif want_dstate:
        dstate = torch.empty((B, W - 1, C), dtype=dt, device=dev)
    ws = _workspace(ws, _lib().gdn_short_conv_workspace_bytes(B, T, C, W), dev)
    _call("gdn_short_conv_backward", dev, x.data_ptr(), xb, xt, w.data_ptr(), _ptr(bias), _ptr(state), dy.data_ptr(),
          _ptr(dstate_out), dx.data_ptr(), ob, ot, dw.data_ptr(), _ptr(dbias), _ptr(dstate), B, T, C, W, _act(activation),
          1 if dt is _BF16 else 0, _ptr(ws), 0 if ws is None else ws.numel(), written=written)
    return dx, dw, dbias, dstate


def short_conv_step(x, w, bias, state, *, slots=None, lengths=None, activation="silu", out=None, state_out=None, stream=None):
    """``short_conv`` for up to L new tokens of N sequences, whose last W - 1 inputs are kept in a pool: what ``step``
    is to ``forward``, with its slots and lengths.

    x [N, L, C] strided as there; state [P, W - 1, C] like x, updated in place unless state_out, a pool of
    the same shape, is given.  slots [N] int32 names each row's slot (None: row n has slot n), lengths [N] int32 how
    many of its L tokens are there (None: all).  A negative slot is padding: nothing of its row is written.
    Tokens past a row's length, and slots that no row names, are left as they were (an out that is allocated here is zero
    there).  A slot beyond the pool, or named by an earlier row too, makes the row's out NaN and writes no state.
    Returns (out [N, L, C], state_out)."""
    if stream is not None:
        with _on(stream, x):
            return short_conv_step(x, w, bias, state, slots=slots, lengths=lengths, activation=activation, out=out,
                                   state_out=state_out)
    dt, dev = _element("x", x)
    N, L, C = _dims("x", x, 3, "[N, L, C]")
    P = _dims("state", state, 3, "[P, W - 1, C]")[0]
    _sizes("N, L, P and C", N, L, P, C)
    xb, xt = _strided("x", x, x.shape, dt, dev)
    W = _taps(w, bias, C, dev)
    if state_out is None:
        state_out = state
    index, pool = dev.index, (P, W - 1, C)
    if not (_fit(index, dt, pool, state) and (state_out is state or _fit(index, dt, pool, state_out))
            and (out is None or _fit(index, dt, (N, L, C), out)) and (slots is None or _fit(index, _I32, (N,), slots))
            and (lengths is None or _fit(index, _I32, (N,), lengths))):
        _needs(dev, ("state", state, pool, dt), ("state_out", state_out, pool, dt))
        for name, t, shape, dtype in (("slots", slots, (N,), _I32), ("lengths", lengths, (N,), _I32), ("out", out, (N, L, C), dt)):
            if t is not None:
                _needs(dev, (name, t, shape, dtype))
    written = (state_out, out)
    if out is None:
        written = (state_out,)
        make = torch.empty if slots is None and lengths is None else torch.zeros
        out = make((N, L, C), dtype=dt, device=dev)
    if _fns is None:
        _lib()
    _call("gdn_short_conv_step", dev, x.data_ptr(), xb, xt, w.data_ptr(), _ptr(bias), state.data_ptr(), _ptr(slots),
          _ptr(lengths), out.data_ptr(), state_out.data_ptr(), N, L, P, C, W, _act(activation), 1 if dt is _BF16 else 0,
          written=written)
    return out, state_out


# ---------------------------------------------------------------------------
# Gradient norm and clipping.

def _dense(t):
    """Whether a tensor's elements fill a run of memory, in whatever order."""
    if t.is_contiguous():
        return True
    at = 1
    for stride, size in sorted(zip(t.stride(), t.shape)):
        if size != 1:
            if stride != at:
                return False
            at *= size
    return True


_KINDS = {_BF16, _F32}


def _check_grads(tensors, name):
    dev = None
    for i, t in enumerate(tensors):
        if not isinstance(t, _Tensor):
            raise TypeError(f"{name}[{i}] must be a tensor, got {type(t).__name__}")
        if t.dtype is not _BF16 and t.dtype is not _F32:
            raise TypeError(f"{name}[{i}] must be bfloat16 or float32, got {t.dtype}")
        if not t.is_cuda:
            raise ValueError(f"{name}[{i}] must be on a GPU, got {t.device}")
        if dev is None:
            dev = t.device
        elif t.device != dev:
            raise ValueError(f"{name}[{i}] must be on {dev}, got {t.device}")
        if not _dense(t):
            raise ValueError(f"{name}[{i}] must fill a run of memory, got strides {list(t.stride())}")
    if dev is None:
        raise ValueError(f"{name} holds no tensor")


def _pointers(tensors, n):
    return (ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors])


def _grads(tensors, name="grads"):
    """The list, checked, its device, length, and the C call's arrays of it."""
    if isinstance(tensors, _Tensor):
        raise TypeError(f"{name} must be a sequence of tensors, got one tensor")
    tensors = list(tensors)
    n = len(tensors)
    # (a call is as long as its checks: all of them in one expression where nothing is wrong)
    index = tensors[0].get_device() if n and isinstance(tensors[0], _Tensor) else -1
    if index < 0 or not all([type(t) is _Tensor and t.get_device() == index and t.is_contiguous() for t in tensors]):
        _check_grads(tensors, name)
    dtypes = [t.dtype for t in tensors]
    if not _KINDS.issuperset(dtypes):
        _check_grads(tensors, name)
    return (tensors, tensors[0].device, n, _pointers(tensors, n), (ctypes.c_int64 * n)(*[t.numel() for t in tensors]),
            (ctypes.c_int * n)(*[d is _BF16 for d in dtypes]), dtypes)


def grad_workspace(grads):
    """Workspace tensor for grad_norm and clip_grads on this many tensors."""
    grads = list(grads)
    if not grads:
        raise ValueError("grads holds no tensor")
    return torch.empty(_lib().gdn_grad_workspace_bytes(len(grads)), dtype=torch.uint8, device=grads[0].device)


def grad_norm(grads, *, out=None, ws=None, stream=None):
    """The 2-norm over all elements of a sequence of tensors, bf16 and fp32 in any mixture, of any sizes (0 too) on one
    device, each filling a run of memory: a 0-dimensional fp32 tensor, summed in fp64.  Nothing waits for the GPU."""
    if stream is not None:
        grads = list(grads)
        with _on(stream, grads[0] if grads else None):
            return grad_norm(grads, out=out, ws=ws)
    grads, dev, n, ptrs, sizes, kinds, _ = _grads(grads)
    written = ()
    if out is None:
        out = torch.empty((), dtype=_F32, device=dev)
    else:
        _needs(dev, ("out", out, (), _F32))
        written = (out,)
    ws = _workspace(ws, _lib().gdn_grad_workspace_bytes(n), dev)
    _call("gdn_grad_norm", dev, ptrs, sizes, kinds, n, out.data_ptr(), ws.data_ptr(), ws.numel(), written=written)
    return out


def clip_grads(grads, max_norm, *, norm=None, eps=1e-6, out=None, ws=None, stream=None):
    """Scales all tensors of a sequence (as in ``grad_norm``) by min(1, max_norm / (norm + eps)), in place or, if out, a
    sequence of tensors like them, is given, into those (out[i] may be grads[i]).  norm: a 0-dimensional fp32 tensor that holds
    the norm, of shards that several processes join, say; None: that of grads.  No tensor may overlap
    another.  A norm of NaN makes everything NaN.  Returns (norm, the scaled tensors); nothing waits for the GPU."""
    if stream is not None:
        grads = list(grads)
        with _on(stream, grads[0] if grads else None):
            return clip_grads(grads, max_norm, norm=norm, eps=eps, out=out, ws=ws)
    grads, dev, n, ptrs, sizes, kinds, dtypes = _grads(grads)
    if out is None:
        out, outs = grads, ptrs
    else:
        if isinstance(out, _Tensor):
            raise TypeError("out must be a sequence of tensors, got one tensor")
        out, index = list(out), dev.index
        if len(out) != n:
            raise ValueError(f"out must hold {n} tensors, got {len(out)}")
        if not all([type(o) is _Tensor and o.get_device() == index and o.shape == g.shape and o.is_contiguous() and g.is_contiguous()
                    for g, o in zip(grads, out)]) or [o.dtype for o in out] != dtypes:
            _check_grads(out, "out")
            for i, (g, o) in enumerate(zip(grads, out)):
                if g.device != o.device or g.shape != o.shape or g.dtype != o.dtype or not (
                        g.stride() == o.stride() or (g.is_contiguous() and o.is_contiguous())):
                    raise ValueError(f"out[{i}] must be like grads[{i}]")
        outs = _pointers(out, n)
    max_norm, eps = float(max_norm), float(eps)
    if not max_norm >= 0 or not eps >= 0:
        raise ValueError(f"max_norm and eps must not be negative, got {max_norm} and {eps}")
    given = norm
    if given is None:
        norm = torch.empty((), dtype=_F32, device=dev)
        ws = _workspace(ws, _lib().gdn_grad_workspace_bytes(n), dev)
    else:
        _needs(dev, ("norm", norm, (), _F32))
        ws = None
    _lib()
    _call("gdn_grad_clip", dev, ptrs, outs, sizes, kinds, n, _ptr(given), None if given is not None else norm.data_ptr(),
          max_norm, eps, _ptr(ws), 0 if ws is None else ws.numel(), written=out)
    return norm, out
