"""The operators around the gated delta-rule forward (include/gdn_ops.h): the
recurrent step of a decoding batch, the gradient of the token-wise chunk forward,
and the norms, gate and scaled residual between two blocks with their gradient.

Thin binding like :mod:`.gdn`: argument checks and marshalling only.  Outputs and
workspaces that are not given are allocated on the stream the call runs on.  No call
records an autograd graph: results of inputs that require a gradient do not.  Tensors that
a call is given to write count as modified in place, and while gradients are recorded may not require
one.
"""
import ctypes

import torch

from . import gdn as _gdn
from .gdn import GDN_OK, GdnError

_fns = None
_Tensor, _BF16, _F32, _I32 = torch.Tensor, torch.bfloat16, torch.float32, torch.int32


def _lib():
    global _fns
    if _fns is None:
        L = _gdn.lib()
        vp, i, sz, fl = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_float
        L.gdn_step_forward.restype = i
        L.gdn_step_forward.argtypes = [vp] * 10 + [i] * 8 + [vp]
        L.gdn_chunk_backward_workspace_bytes.restype = sz
        L.gdn_chunk_backward_workspace_bytes.argtypes = [i] * 7
        L.gdn_chunk_backward.restype = i
        L.gdn_chunk_backward.argtypes = [vp] * 14 + [i] * 7 + [vp, sz, vp]
        L.gdn_block_norm_forward.restype = i
        L.gdn_block_norm_forward.argtypes = [vp] * 7 + [i] * 3 + [fl] * 2 + [i, vp]
        L.gdn_block_norm_workspace_bytes.restype = sz
        L.gdn_block_norm_workspace_bytes.argtypes = [i] * 3
        L.gdn_block_norm_backward.restype = i
        L.gdn_block_norm_backward.argtypes = [vp] * 12 + [i] * 3 + [fl] * 2 + [i, vp, sz, vp]
        _fns = L
    return _fns


def _ptr(t):
    return None if t is None else t.data_ptr()


def _raw_stream(index):
    return torch.cuda.current_stream(index).cuda_stream


# (the handle alone: the stream object around it takes as long to make as a launch)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)


_modified = torch.autograd.graph.increment_version


def _call(name, dev, *args, written=()):
    """The C call with the current stream of `dev` behind its other arguments.  written: the
    caller's own tensors among the outputs, whose saved uses autograd is told of."""
    for t in written:
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError("a tensor that requires a gradient cannot be written while gradients are recorded")
    fn = getattr(_fns or _lib(), name)
    index = dev.index
    if torch.cuda.current_device() == index:
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _raw_stream(index))
    if rc != GDN_OK:
        raise GdnError(name, rc)
    if written:
        _modified(written)


def _needs(dev, *specs):
    """_need for each (name, tensor, shape, dtype); one condition where nothing is wrong, since
    a small call is as long as its checks."""
    index = dev.index
    for name, t, shape, dtype in specs:
        if not _fit(index, dtype, shape, t):
            _need(name, t, shape, dtype, dev)


def _fit(index, dtype, shape, *tensors):
    """Whether _need would pass all of these (it may pass others, a tensor's subclass)."""
    for t in tensors:
        if type(t) is not _Tensor or t.dtype is not dtype or t.get_device() != index or t.shape != shape \
                or not t.is_contiguous():
            return False
    return True


def _need(name, t, shape, dtype, dev):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor, got {type(t).__name__}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must have dtype {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _on(stream, t):
    """Context of a call on `stream`, which has to be one of the tensors' device."""
    if isinstance(t, torch.Tensor) and t.device.type == "cuda" and stream.device != t.device:
        raise ValueError(f"stream must be on {t.device}, got {stream.device}")
    return torch.cuda.stream(stream)


def _element(name, t):
    if not isinstance(t, _Tensor):
        raise TypeError(f"{name} must be a tensor, got {type(t).__name__}")
    dt = t.dtype
    if dt is not _BF16 and dt is not _F32:
        raise TypeError(f"{name} must be bfloat16 or float32, got {dt}")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU, got {t.device}")
    return dt, t.device


def _int(name, n):
    """A whole number of the caller's that the C call takes in 32 bits (and ctypes would cut)."""
    i = int(n)
    if i != n or not 0 <= i < 1 << 31:
        raise ValueError(f"{name} must be a whole number below 2^31, got {n}")
    return i


def _dims(name, t, dims, text):
    shape = t.shape if isinstance(t, _Tensor) else ()
    if len(shape) != dims:
        raise ValueError(f"{name} must be {text}, got {list(shape)}")
    return shape


def step(q, k, v, alpha, beta, state, *, slots=None, lengths=None, out=None, state_out=None, stream=None):
    """The recurrent form of ``forward``: up to L new tokens of N sequences, against
    states kept in a pool.

    q, k [N, L, Hk, Dk] and v [N, L, H, Dv], bf16 or fp32, with Hk a divisor of H (H / Hk
    consecutive heads share a key head); alpha, beta [N, L, H] fp32; state
    [P, H, Dk, Dv] fp32.  slots [N] int32 names each row's state (None: row n has
    slot n), lengths [N] int32 how many of its L tokens are there (None: all).  The
    states are updated in place unless state_out, a pool of the same shape, is
    given.  A negative slot is padding: nothing of its row is written.  Tokens
    past a row's length, and slots that no row names, are left as they were (an out
    that is allocated here is zero there).  A slot beyond the pool, or named by an earlier row too,
    makes the row's out NaN and writes no state.  Returns (out [N, L, H, Dv] like v, state_out)."""
    if stream is not None:
        with _on(stream, q):
            return step(q, k, v, alpha, beta, state, slots=slots, lengths=lengths, out=out, state_out=state_out)
    dt, dev = _element("q", q)
    N, L, Hk, Dk = keys = _dims("q", q, 4, "[N, L, Hk, Dk]")
    Nv, Lv, H, Dv = values = _dims("v", v, 4, "[N, L, H, Dv]")
    P, Hs, Dks, Dvs = pool = _dims("state", state, 4, "[P, H, Dk, Dv]")
    f32, gates, index = _F32, (N, L, H), dev.index
    if state_out is None:
        state_out = state
    # one condition where nothing is wrong: a token's step is as long as its checks
    if not (N == Nv and L == Lv and H == Hs and Dk == Dks and Dv == Dvs and _fit(index, dt, keys, q, k)
            and _fit(index, dt, values, v) and _fit(index, f32, gates, alpha, beta)
            and _fit(index, f32, pool, state) and (state_out is state or _fit(index, f32, pool, state_out))
            and (out is None or _fit(index, dt, values, out))
            and (slots is None or _fit(index, _I32, (N,), slots))
            and (lengths is None or _fit(index, _I32, (N,), lengths))):
        values, pool = (N, L, H, Dv), (P, H, Dk, Dv)
        _needs(dev, ("q", q, keys, dt), ("k", k, keys, dt), ("v", v, values, dt), ("alpha", alpha, gates, f32),
               ("beta", beta, gates, f32), ("state", state, pool, f32), ("state_out", state_out, pool, f32))
        for name, t, shape, dtype in (("slots", slots, (N,), _I32), ("lengths", lengths, (N,), _I32),
                                      ("out", out, values, dt)):
            if t is not None:
                _needs(dev, (name, t, shape, dtype))
    written = (state_out, out)
    if out is None:
        written = (state_out,)
        # every element is written unless a row may be short or padding
        out = torch.empty_like(v) if slots is None and lengths is None else torch.zeros_like(v)
    _call("gdn_step_forward", dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), alpha.data_ptr(), beta.data_ptr(),
          state.data_ptr(), _ptr(slots), _ptr(lengths), out.data_ptr(), state_out.data_ptr(), N, L, P, Hk, H, Dk, Dv,
          1 if dt is _BF16 else 0, written=written)
    return out, state_out


def backward_workspace(q, v, chunk=_gdn.CHUNK):
    """Workspace tensor for backward on inputs shaped like q [B, T, H, Dk] and v [.., Dv]."""
    B, T, H, Dk = q.shape
    if max(B, T, H) >= 1 << 31:
        raise ValueError(f"B, T and H must be below 2^31, got {list(q.shape)}")
    n = _lib().gdn_chunk_backward_workspace_bytes(B, H, T, Dk, v.shape[-1], _int("chunk", chunk),
                                                  1 if q.dtype == torch.bfloat16 else 0)
    if n == 0:
        raise ValueError("unsupported shape for the GDN chunk backward")
    return torch.empty(n, dtype=torch.uint8, device=q.device)


def backward(q, k, v, alpha, beta, state_in, dout, dstate_out=None, *, dq=None, dk=None, dv=None, dalpha=None,
             dbeta=None, dstate_in=None, want_dstate=True, ws=None, chunk=_gdn.CHUNK, stream=None):
    """Gradient of ``forward``: from dout = dL/d(out) [B, T, H, Dv] like v and dstate_out =
    dL/d(state_out) [B, H, Dk, Dv] fp32 (None: zero), with the forward call's inputs
    (state_in may be None there and here).  Needs nothing else of that call.
    dstate_in may be dstate_out.  Returns (dq, dk, dv like q, dalpha, dbeta [B, T, H] fp32,
    dstate_in [B, H, Dk, Dv] fp32, or None without want_dstate)."""
    if stream is not None:
        with _on(stream, q):
            return backward(q, k, v, alpha, beta, state_in, dout, dstate_out, dq=dq, dk=dk, dv=dv, dalpha=dalpha,
                            dbeta=dbeta, dstate_in=dstate_in, want_dstate=want_dstate, ws=ws, chunk=chunk)
    dt, dev = _element("q", q)
    B, T, H, Dk = _dims("q", q, 4, "[B, T, H, Dk]")
    Dv = _dims("v", v, 4, "[B, T, H, Dv]")[3]
    f32 = torch.float32
    keys, values, gates = (B, T, H, Dk), (B, T, H, Dv), (B, T, H)
    if not (_fit(dev.index, dt, keys, q, k) and _fit(dev.index, dt, values, v, dout)
            and _fit(dev.index, f32, gates, alpha, beta)):
        _needs(dev, ("q", q, keys, dt), ("k", k, keys, dt), ("v", v, values, dt), ("dout", dout, values, dt),
               ("alpha", alpha, gates, f32), ("beta", beta, gates, f32))
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out)):
        if t is not None:
            _needs(dev, (name, t, (B, H, Dk, Dv), f32))
    written = [t for t in (dq, dk, dv, dalpha, dbeta, dstate_in) if t is not None]
    dq = _given("dq", dq, q)
    dk = _given("dk", dk, k)
    dv = _given("dv", dv, v)
    dalpha = _given("dalpha", dalpha, alpha)
    dbeta = _given("dbeta", dbeta, beta)
    if dstate_in is not None:
        _needs(dev, ("dstate_in", dstate_in, (B, H, Dk, Dv), f32))
    elif want_dstate:
        dstate_in = torch.empty((B, H, Dk, Dv), dtype=f32, device=dev)
    if ws is None:
        ws = backward_workspace(q, v, chunk)
    elif ws.device != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    _call("gdn_chunk_backward", dev, q.data_ptr(), k.data_ptr(), v.data_ptr(), alpha.data_ptr(), beta.data_ptr(),
          _ptr(state_in), dout.data_ptr(), _ptr(dstate_out), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
          dalpha.data_ptr(), dbeta.data_ptr(), _ptr(dstate_in), B, H, T, Dk, Dv, _int("chunk", chunk),
          1 if dt == torch.bfloat16 else 0, ws.data_ptr(), ws.numel(), written=written)
    return dq, dk, dv, dalpha, dbeta, dstate_in


def block_norm_workspace(rows, channels, gate_tokens, device):
    """Workspace tensor for block_norm_backward on `rows` tokens of `channels`."""
    return _block_norm_ws(_int("rows", rows), _int("channels", channels), _int("gate_tokens", gate_tokens), device)


def _block_norm_ws(rows, channels, gate_tokens, device):
    n = _lib().gdn_block_norm_workspace_bytes(rows, channels, gate_tokens)
    if n == 0:
        raise ValueError("unsupported shape for the block norm")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _block_inputs(x, y, gate, w_post, w_pre, gate_tokens):
    dt, dev = _element("x", x)
    B, T, C = _dims("x", x, 3, "[B, T, C]")
    gt = gate_tokens if type(gate_tokens) is int else _int("gate_tokens", gate_tokens)   # (one that divides T fits)
    if gt < 1 or T % gt:
        raise ValueError("T must be a whole number of runs of gate_tokens tokens")
    if max(B * T, C) >= 1 << 31:      # (the C call's sizes are 32-bit)
        raise ValueError(f"B T and C must be below 2^31, got {B * T} and {C}")
    f32 = torch.float32
    if not (_fit(dev.index, dt, (B, T, C), x, y) and _fit(dev.index, f32, (C,), w_post, w_pre)):
        _needs(dev, ("x", x, (B, T, C), dt), ("y", y, (B, T, C), dt), ("w_post", w_post, (C,), f32),
               ("w_pre", w_pre, (C,), f32))
    if gate is not None:
        _needs(dev, ("gate", gate, (B, T // gt, C), dt))
    return dt, dev, B, T, C, gt


def _given(name, t, like):
    """An output: the one given, checked, or a new one like another tensor of the call."""
    if t is None:
        return torch.empty_like(like)
    _needs(like.device, (name, t, like.shape, like.dtype))
    return t


def block_norm(x, y, gate, w_post, w_pre, *, gate_tokens=1, res_scale=1.0, eps=1e-6, r=None, u=None, stream=None):
    """The border between two blocks: with the residual stream x and a block's output y
    (both [B, T, C], bf16 or fp32),

        r = res_scale x + gate o RMSNorm(y; w_post),     u = RMSNorm(r; w_pre).

    gate [B, T / gate_tokens, C] (like x, or None for ones) has one row for each run of
    gate_tokens consecutive tokens: 1 per token, T per sample; w_post, w_pre [C]
    fp32; C at most 8192.  r (the next residual stream) and u (the next block's
    input) are allocated unless given; r may be x or y, u may be y.  Returns (r, u)."""
    if stream is not None:
        with _on(stream, x):
            return block_norm(x, y, gate, w_post, w_pre, gate_tokens=gate_tokens, res_scale=res_scale, eps=eps, r=r, u=u)
    dt, dev, B, T, C, gt = _block_inputs(x, y, gate, w_post, w_pre, gate_tokens)
    written = [t for t in (r, u) if t is not None]
    r = _given("r", r, x)
    u = _given("u", u, x)
    _call("gdn_block_norm_forward", dev, x.data_ptr(), y.data_ptr(), _ptr(gate), w_post.data_ptr(), w_pre.data_ptr(),
          r.data_ptr(), u.data_ptr(), B * T, C, gt, float(res_scale), float(eps), 1 if dt == torch.bfloat16 else 0,
          written=written)
    return r, u


def block_norm_backward(x, y, gate, w_post, w_pre, du, dr=None, *, gate_tokens=1, res_scale=1.0, eps=1e-6, dx=None,
                        dy=None, dgate=None, dw_post=None, dw_pre=None, ws=None, stream=None):
    """Gradient of ``block_norm`` from du = dL/du and dr = dL/dr ([B, T, C] like x; dr None:
    zero).  The other arguments are those of the forward call.  dx may be dr or du, dy
    may be y or the other of them.  Returns (dx, dy, dgate, dw_post, dw_pre); dgate is
    None where gate is."""
    if stream is not None:
        with _on(stream, x):
            return block_norm_backward(x, y, gate, w_post, w_pre, du, dr, gate_tokens=gate_tokens, res_scale=res_scale,
                                       eps=eps, dx=dx, dy=dy, dgate=dgate, dw_post=dw_post, dw_pre=dw_pre, ws=ws)
    dt, dev, B, T, C, gt = _block_inputs(x, y, gate, w_post, w_pre, gate_tokens)
    _needs(dev, ("du", du, (B, T, C), dt))
    if dr is not None:
        _needs(dev, ("dr", dr, (B, T, C), dt))
    written = [t for t in (dx, dy, dgate, dw_post, dw_pre) if t is not None]
    dx = _given("dx", dx, x)
    dy = _given("dy", dy, y)
    if gate is not None:
        dgate = _given("dgate", dgate, gate)
    elif dgate is not None:
        raise ValueError("dgate without gate")
    dw_post = _given("dw_post", dw_post, w_post)
    dw_pre = _given("dw_pre", dw_pre, w_pre)
    if ws is None:
        ws = _block_norm_ws(B * T, C, gt, dev)
    elif ws.device != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous uint8 tensor on {dev}")
    _call("gdn_block_norm_backward", dev, x.data_ptr(), y.data_ptr(), _ptr(gate), w_post.data_ptr(), w_pre.data_ptr(),
          du.data_ptr(), _ptr(dr), dx.data_ptr(), dy.data_ptr(), _ptr(dgate), dw_post.data_ptr(), dw_pre.data_ptr(),
          B * T, C, gt, float(res_scale), float(eps), 1 if dt == torch.bfloat16 else 0, ws.data_ptr(), ws.numel(),
          written=written)
    return dx, dy, dgate, dw_post, dw_pre
