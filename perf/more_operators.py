"""Timed calls of the gated linear map, the short convolution and gradient clipping.

``gated``           the gated half of a feed-forward block: two projections, an
                    activation and their product; and its gradient.
``conv``            the short causal convolution in front of the recurrence, over
                    prompts and frames; and its gradient.
``conv_step``       the same for one or a few tokens per sequence, against windows
                    kept in a pool of slots.
``clip``            the norm over all gradients of a step, and their clipping.

Where ``own`` is false the operators run in their plain form, elementary torch
operations in fp32 (long sums in fp64); where it is true, as the package's calls.
Sizes are those of the package's own workloads (16 heads of 128 channels, frames
of 3520 tokens) and of decoding batches of one to 256 sequences.
"""
import math

import torch

own = False

_GATED = dict(op="gated", dtype="bf16", M=1, C=2048, F=8192, act="silu", dir="fwd")
_CONV = dict(op="conv", dtype="bf16", B=1, T=0, C=2048, parts=1, part=0, W=4, act="silu", bias=True, state=True, dir="fwd")
_STEP = dict(op="conv_step", dtype="bf16", N=1, L=1, P=1, C=6144, W=4, act="silu", bias=True, pad=0, ragged=False)
_CLIP = dict(op="clip", blocks=1, C=2048, F=8192, f32_every=0, scale=1.0, max_norm=1.0)


def listed():
    return [
        # one user's token: the weights go through the chip once
        dict(_GATED, name="gated-one"),
        # an ordinary decoding batch
        dict(_GATED, name="gated-batch", M=64),
        # three latent frames of 1280x704 video in one call
        dict(_GATED, name="gated-frames", M=10560),
        # one frame in training
        dict(_GATED, name="gated-frame-grad", M=3520, act="gelu_tanh", dir="bwd"),
        # sizes that no tile divides, fp32, both directions
        dict(_GATED, name="gated-odd-f32", dtype="f32", M=333, C=1283, F=2711, act="gelu", dir="both"),
        # one stream's token through the queries', keys' and values' window: all latency
        dict(_STEP, name="conv-step-one"),
        # drafted tokens of a decoding batch, lengths zero to four, some rows of padding
        dict(_STEP, name="conv-step-batch", N=64, L=4, P=80, pad=3, ragged=True),
        # three frames, the keys' part of a packed projection
        dict(_CONV, name="conv-frames", T=10560, parts=3, part=1),
        # the same in training
        dict(_CONV, name="conv-frames-grad", T=10560, parts=3, part=1, dir="bwd"),
        # an odd width and length, three taps, fp32, both directions, nothing before the first token
        dict(_CONV, name="conv-odd-f32", dtype="f32", B=3, T=1171, C=333, W=3, act="none", state=False, dir="both"),
        # the gradients of a small head: few tensors of odd sizes, two types
        dict(_CLIP, name="clip-small", C=131, F=333, f32_every=3),
        # the gradients of four blocks
        dict(_CLIP, name="clip-blocks", blocks=4, f32_every=0, scale=0.01, max_norm=0.5),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """Another case of the same ranges: 1 to 10560 rows of 64 to 4096 channels through
    64 to 12288 hidden ones, 1 to 256 decoding rows, 1 to 4 blocks' gradients."""
    op = rng.choice(["gated", "gated", "gated", "conv", "conv", "conv_step", "clip"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    act = rng.choice(["silu", "silu", "gelu", "gelu_tanh"])
    if op == "gated":
        C, F = _log_int(rng, 64, 4096), _log_int(rng, 64, 12288)
        if rng.random() < 0.7:
            C, F = max(64, C // 64 * 64), max(64, F // 64 * 64)
        way = rng.choice(["fwd", "fwd", "bwd", "both"])
        room = 10560 * 2048 * 8192 // (C * F * (1 if way == "fwd" else 4) * (6 if dtype == "f32" else 1))
        return dict(_GATED, dtype=dtype, M=_log_int(rng, 1, max(1, min(10560, room))), C=C, F=F, act=act, dir=way)
    W = rng.choice([2, 3, 4, 4])
    if op == "conv":
        B, C = rng.choice([1, 1, 2, 4]), _log_int(rng, 32, 6144)
        if rng.random() < 0.6:
            C = max(32, C // 64 * 64)
        parts = rng.choice([1, 1, 2, 3])
        return dict(_CONV, dtype=dtype, B=B, T=_log_int(rng, 1, min(10560, 10560 * 2048 // (B * C))), C=C, parts=parts,
                    part=rng.randrange(parts), W=W, act=rng.choice([act, "none"]), bias=rng.random() < 0.5,
                    state=rng.random() < 0.6, dir=rng.choice(["fwd", "bwd", "both"]))
    if op == "conv_step":
        N, L = _log_int(rng, 1, 256), rng.choice([1, 1, 1, rng.randint(2, 8)])
        return dict(_STEP, dtype=dtype, N=N, L=L, P=N + rng.randint(0, 16), C=_log_int(rng, 32, 8192), W=W, act=act,
                    bias=rng.random() < 0.5, pad=rng.choice([0, 0, rng.randint(0, N // 4)]),
                    ragged=L > 1 and rng.random() < 0.7)
    C, F = _log_int(rng, 32, 2048), _log_int(rng, 32, 8192)
    return dict(_CLIP, blocks=rng.randint(1, 4), C=C, F=F, f32_every=rng.choice([0, 1, 2, 5]),
                scale=rng.choice([1.0, 0.01, 1e-4]), max_norm=rng.choice([1.0, 0.5, 1e3]))


# ---------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _clip_shapes(case):
    """A block's gradients: projections, feed-forward, convolution and norm weights."""
    C, F = case["C"], case["F"]
    return [(C, C), (C, C), (C, C), (C, C), (C, 4), (C,), (C,), (F, C), (F, C), (C, F)] * case["blocks"]


def _clip_dtypes(case):
    every = case["f32_every"]
    return [torch.float32 if len(s) == 1 or (every and i % every == 0) else torch.bfloat16
            for i, s in enumerate(_clip_shapes(case))]


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    s = dict(case=dict(c))
    if c["op"] == "clip":
        s["grads"] = [(c["scale"] * randn(*n)).to(d) for n, d in zip(_clip_shapes(c), _clip_dtypes(c))]
        s["out"] = [torch.empty_like(g) for g in s["grads"]]
        return s
    dt, C = _dtype(c), c["C"]
    if c["op"] == "gated":
        M, F = c["M"], c["F"]
        s["x"] = randn(M, C).to(dt)                                      # a norm's output
        s["w_gate"], s["w_up"] = ((randn(F, C) / math.sqrt(C)).to(dt) for _ in range(2))
        if c["dir"] != "fwd":
            s["dh"] = randn(M, F).to(dt)
        return s
    W = c["W"]
    s["w"] = randn(C, W) / math.sqrt(W)
    s["bias"] = 0.2 * randn(C) if c["bias"] else None
    if c["op"] == "conv_step":
        N, L, P = c["N"], c["L"], c["P"]
        s["x"] = randn(N, L, C).to(dt)
        s["pool"] = randn(P, W - 1, C).to(dt)
        s["new"] = s["pool"].clone()                                     # windows after the tokens; other slots stay
        slots = torch.randperm(P, generator=gen, device=dev)[:N].to(torch.int32)
        if c["pad"]:
            slots[N - c["pad"]:] = -1                                    # a batch of fixed size that is not full
        s["slots"] = slots
        s["lengths"] = None
        if c["ragged"]:
            s["lengths"] = torch.randint(0, L + 1, (N,), generator=gen, device=dev, dtype=torch.int32)
        s["out"] = torch.zeros(N, L, C, dtype=dt, device=dev)
        return s
    B, T = c["B"], c["T"]
    s["packed"] = randn(B, T, c["parts"] * C).to(dt)
    s["x"] = s["packed"][..., c["part"] * C:(c["part"] + 1) * C]
    s["state"] = randn(B, W - 1, C).to(dt) if c["state"] else None
    if c["dir"] != "fwd":
        s["dy"] = randn(B, T, C).to(dt)
        s["dstate"] = randn(B, W - 1, C).to(dt) if c["state"] else None
    return s


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "gated":
        return _plain_gated(s)
    if c["op"] == "conv":
        return _plain_conv(s)
    return _plain_conv_step(s) if c["op"] == "conv_step" else _plain_clip(s)


def _own(s):
    import paper_2605_30409_amd as gdn
    c = s["case"]
    if c["op"] == "clip":
        return gdn.clip_grads(s["grads"], c["max_norm"], out=s["out"])
    res = ()
    if c["op"] == "gated":
        if c["dir"] != "bwd":
            res += (gdn.gated_linear(s["x"], s["w_gate"], s["w_up"], activation=c["act"]),)
        if c["dir"] != "fwd":
            res += gdn.gated_linear_backward(s["x"], s["w_gate"], s["w_up"], s["dh"], activation=c["act"])
        return res
    act = None if c["act"] == "none" else c["act"]
    if c["op"] == "conv_step":
        return gdn.short_conv_step(s["x"], s["w"], s["bias"], s["pool"], slots=s["slots"], lengths=s["lengths"],
                                   activation=act, out=s["out"], state_out=s["new"])
    if c["dir"] != "bwd":
        res += gdn.short_conv(s["x"], s["w"], s["bias"], s["state"], activation=act)
    if c["dir"] != "fwd":
        dx, dw, dbias, dstate = gdn.short_conv_backward(s["x"], s["w"], s["bias"], s["state"], s["dy"], s["dstate"],
                                                        activation=act)
        res += (dx, dw) + ((dbias,) if c["bias"] else ()) + (dstate,)
    return res


def work(case):
    c = case
    if c["op"] == "clip":
        sizes = [math.prod(n) for n in _clip_shapes(c)]
        by = sum(2 * n * d.itemsize for n, d in zip(sizes, _clip_dtypes(c)))
        return {"bytes": by + 4, "flops": 3 * sum(sizes)}
    esz, C = _dtype(c).itemsize, c["C"]
    if c["op"] == "gated":
        M, F = c["M"], c["F"]
        by = fl = 0
        if c["dir"] != "bwd":
            by += (M * C + 2 * F * C + M * F) * esz
            fl += 4 * M * C * F
        if c["dir"] != "fwd":                        # the two projections again, and their gradients
            by += (2 * M * C + 4 * F * C + M * F) * esz
            fl += 12 * M * C * F
        return {"bytes": by, "flops": fl}
    W = c["W"]
    weights = 4 * C * (W + (1 if c["bias"] else 0))
    if c["op"] == "conv_step":
        rows = c["N"] - c["pad"]
        tok = rows * c["L"] / (2.0 if c["ragged"] else 1.0)
        return {"bytes": (2 * tok + 2 * rows * (W - 1)) * C * esz + weights, "flops": (2 * W + 5) * tok * C}
    n, edge = c["B"] * c["T"] * C, c["B"] * (W - 1) * C * esz
    by = fl = 0
    if c["dir"] != "bwd":
        by += 2 * n * esz + edge * (2 if c["state"] else 1) + weights
        fl += (2 * W + 5) * n
    if c["dir"] != "fwd":
        by += 3 * n * esz + edge * (3 if c["state"] else 1) + 2 * weights
        fl += (6 * W + 12) * n
    return {"bytes": by, "flops": fl}


# ---------------------------------------------------------------------------
# Plain forms.

def _act(z, act):
    if act == "none":
        return z
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))


def _act_slope(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1.0 + z * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (z + 0.044715 * z * z * z))
    return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * k * (1.0 + 3 * 0.044715 * z * z)


def _plain_gated(s):
    c, dt = s["case"], s["x"].dtype
    x, wg, wu = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    g, u = x @ wg.T, x @ wu.T
    a = _act(g, c["act"])
    res = ()
    if c["dir"] != "bwd":
        res += ((a * u).to(dt),)
    if c["dir"] != "fwd":
        dh = s["dh"].float()
        dg, du = dh * u * _act_slope(g, c["act"]), dh * a
        res += ((dg @ wg + du @ wu).to(dt), (dg.T @ x).to(dt), (du.T @ x).to(dt))
    return res


def _window(x, state, W):
    """Inputs with what stands before them, [B, T + W - 1, C] in fp32."""
    if state is None:
        state = torch.zeros_like(x[:, :1]).expand(-1, W - 1, -1)
    return torch.cat([state.float(), x.float()], 1)


def _taps(xe, w, bias):
    z = (xe.unfold(1, w.shape[1], 1) * w).sum(-1)
    return z if bias is None else z + bias


def _plain_conv(s):
    c, dt = s["case"], s["x"].dtype
    T, W, w = c["T"], c["W"], s["w"]
    xe = _window(s["x"], s["state"], W)
    z = _taps(xe, w, s["bias"])
    res = ()
    if c["dir"] != "bwd":
        res += (_act(z, c["act"]).to(dt), xe[:, T:].to(dt))
    if c["dir"] != "fwd":
        dz = s["dy"].float() * _act_slope(z, c["act"])
        edge = torch.zeros_like(xe[:, :W - 1])
        dxe = (torch.cat([edge, dz, edge], 1).unfold(1, W, 1) * w.flip(1)).sum(-1)
        if s["dstate"] is not None:
            dxe[:, T:] += s["dstate"].float()
        dw = (dz.unsqueeze(-1) * xe.unfold(1, W, 1)).sum((0, 1), dtype=torch.float64).float()
        res += (dxe[:, W - 1:].to(dt), dw)
        if s["bias"] is not None:
            res += (dz.sum((0, 1), dtype=torch.float64).float(),)
        res += (dxe[:, :W - 1].to(dt),)
    return res


def _plain_conv_step(s):
    c, dt = s["case"], s["x"].dtype
    W, L, n = c["W"], c["L"], c["N"] - c["pad"]                          # padding stands at the end
    at = s["slots"][:n].long()
    xe = _window(s["x"][:n], s["pool"][at], W)
    y = _act(_taps(xe, s["w"], s["bias"]), c["act"]).to(dt)
    length = torch.full((n,), L, device=xe.device) if s["lengths"] is None else s["lengths"][:n].long()
    on = torch.arange(L, device=xe.device) < length[:, None]
    s["out"][:n] = torch.where(on.unsqueeze(-1), y, s["out"][:n])
    last = length[:, None] + torch.arange(W - 1, device=xe.device)
    s["new"][at] = xe.gather(1, last.unsqueeze(-1).expand(-1, -1, c["C"])).to(dt)
    return s["out"], s["new"]


def _plain_clip(s):
    c = s["case"]
    squares = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]])
    norm = squares.sum().sqrt()
    scale = (c["max_norm"] / (norm + 1e-6)).clamp_max(1.0).float()
    return norm.float(), [o.copy_(g.float() * scale) for g, o in zip(s["grads"], s["out"])]


# ---------------------------------------------------------------------------
# The same results in fp64, from the definitions.

def _exact_act(z, act):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-(8 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "clip":
        return _exact_clip(s)
    if c["op"] == "conv_step":
        return _exact_conv_step(s)
    res = ()
    if c["op"] == "gated":
        x, wg, wu = (s[n].double().requires_grad_() for n in ("x", "w_gate", "w_up"))
        h = _exact_act(torch.matmul(x, wg.t()), c["act"]) * torch.matmul(x, wu.t())
        if c["dir"] != "bwd":
            res += (h.detach(),)
        if c["dir"] != "fwd":
            res += torch.autograd.grad(h, (x, wg, wu), s["dh"].double())
        return res
    x, w = s["x"].double().requires_grad_(), s["w"].double().requires_grad_()
    B, T, C, W = c["B"], c["T"], c["C"], c["W"]
    state = torch.zeros(B, W - 1, C, device=x.device) if s["state"] is None else s["state"]
    state = state.double().requires_grad_()
    bias = None if s["bias"] is None else s["bias"].double().requires_grad_()
    xe = torch.cat([state, x], 1)
    z = torch.zeros_like(x)
    for i in range(W):
        z = z + xe[:, i:i + T] * w[:, i]
    y = _exact_act(z if bias is None else z + bias, c["act"])
    if c["dir"] != "bwd":
        res += (y.detach(), xe[:, T:].detach())
    if c["dir"] != "fwd":
        loss = (y * s["dy"].double()).sum()
        if s["dstate"] is not None:
            loss = loss + (xe[:, T:] * s["dstate"].double()).sum()
        res += torch.autograd.grad(loss, (x, w) + (() if bias is None else (bias,)) + (state,))
    return res


def _exact_conv_step(s):
    """Sequence by sequence, token by token."""
    c = s["case"]
    out, new, w = s["out"].double(), s["pool"].double(), s["w"].double()
    bias = 0.0 if s["bias"] is None else s["bias"].double()
    lengths = [c["L"]] * c["N"] if s["lengths"] is None else s["lengths"].tolist()
    for n, (slot, m) in enumerate(zip(s["slots"].tolist(), lengths)):
        for t in range(m if slot >= 0 else 0):
            win = torch.cat([new[slot], s["x"][n, t:t + 1].double()])
            out[n, t] = _exact_act((win.T * w).sum(1) + bias, c["act"])
            new[slot] = win[1:]
    return out, new


def _exact_clip(s):
    total = sum(float(torch.linalg.vector_norm(g.double())) ** 2 for g in s["grads"])
    norm = torch.tensor(math.sqrt(total), dtype=torch.float64, device="cuda")
    scale = min(1.0, s["case"]["max_norm"] / (math.sqrt(total) + 1e-6))
    return norm, [g.double() * scale for g in s["grads"]]
