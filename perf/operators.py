"""Timed calls of the recurrent step, the gradient and the block norm.

``step``            a decoding batch: one or a few tokens per sequence against
                    recurrent states kept in a pool of slots.
``backward``        the gradient of the token-wise chunk forward.
``block_norm``      the border between two blocks: norm of the block's output,
                    gate, scaled residual, norm of the sum; and its gradient.

Where ``own`` is false the operators run in their plain form, elementary torch
operations in fp32 (decays from fp64 logarithms); where it is true, as the
package's calls.  Sizes are those of the package's own workloads (heads of 64 and
128, 16 to 32 of them, frames of 3520 tokens) and of decoding batches of one to
256 sequences.
"""
import math

import torch

own = False

_STEP = dict(op="step", dtype="bf16", N=1, L=1, P=1, Hk=16, H=16, Dk=128, Dv=128, pad=0, ragged=False, mu=-3.0)
_BACK = dict(op="backward", dtype="bf16", B=1, T=0, H=16, Dk=128, Dv=128, mu=0.0, state=True)
_NORM = dict(op="norm", dtype="bf16", B=1, T=0, C=2048, gate_tokens=1, dir="fwd", res_scale=1.0)


def listed():
    return [
        # one user's stream, one token: all latency
        dict(_STEP, name="step-one"),
        # an ordinary decoding batch, key heads shared by two value heads, three rows of padding
        dict(_STEP, name="step-batch", N=64, P=80, H=32, pad=3),
        # a full server: a gigabyte of states through the chip for one token each
        dict(_STEP, name="step-server", N=256, P=272, H=32),
        # a few drafted tokens per sequence, lengths zero to five, fp32, narrow heads
        dict(_STEP, name="step-draft-f32", dtype="f32", N=13, L=5, P=16, Hk=20, H=20, Dk=64, Dv=64, ragged=True),
        # the smallest training call, five chunks with a ragged tail
        dict(_BACK, name="backward-tiny-f32", dtype="f32", T=257, H=2, Dk=64, Dv=64, state=False),
        # one latent frame of 1280x704 video
        dict(_BACK, name="backward-frame", T=3520),
        # three frames in one call, heads that remember for long
        dict(_BACK, name="backward-stream3", T=10560, mu=-3.0),
        # a batch of narrow heads that forget fast
        dict(_BACK, name="backward-batch-d64", B=4, T=3520, H=20, Dk=64, Dv=64, mu=2.0),
        # fp32 with a length that is no multiple of the chunk
        dict(_BACK, name="backward-ragged-f32", dtype="f32", T=3557, mu=-3.0),
        # three frames, a gate row per frame, forward
        dict(_NORM, name="norm-frames", T=10560, gate_tokens=3520),
        # the same in training
        dict(_NORM, name="norm-frames-grad", T=10560, gate_tokens=3520, dir="bwd", res_scale=0.5),
        # an odd width with a gate of each token's own, both directions, fp32
        dict(_NORM, name="norm-odd-f32", dtype="f32", B=2, T=333, C=1283, dir="both", res_scale=0.5),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    """Another case of the same ranges: 1 to 256 sequences of 1 to 8 tokens, 1 to
    10560 tokens of training, rows of 32 to 8192 channels."""
    op = rng.choice(["step", "step", "backward", "backward", "norm"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    Dk, Dv = rng.choice([(128, 128), (128, 128), (64, 64), (128, 64), (64, 128)])
    if op == "step":
        group = rng.choice([1, 1, 2, 4])
        Hk = _log_int(rng, 1, 32 // group)
        N = _log_int(rng, 1, 256)
        L = rng.choice([1, 1, 1, rng.randint(2, 8)])
        return dict(_STEP, dtype=dtype, N=N, L=L, P=N + rng.randint(0, 16), Hk=Hk, H=Hk * group, Dk=Dk, Dv=Dv,
                    pad=rng.choice([0, 0, rng.randint(0, N // 4)]), ragged=L > 1 and rng.random() < 0.7,
                    mu=rng.choice([0.0, -3.0]))
    if op == "backward":
        B, H = rng.choice([1, 1, 2, 4]), _log_int(rng, 1, 32)
        room = (3557 if dtype == "f32" else 10560) * 16 * 128 // (B * H * max(Dk, Dv))
        return dict(_BACK, dtype=dtype, B=B, T=_log_int(rng, 1, min(room, 10560)), H=H, Dk=Dk, Dv=Dv,
                    mu=rng.choice([0.0, 2.0, -3.0]), state=rng.random() < 0.7)
    B, C = rng.choice([1, 1, 2, 4]), _log_int(rng, 32, 8192)
    if rng.random() < 0.6:
        C = max(32, C // 64 * 64)
    rows = _log_int(rng, 1, min(3520, 10560 * 2048 // (B * C)))          # tokens to a gate row
    G = rng.randint(1, max(1, min(6, 10560 * 2048 // (B * C * rows))))
    each = rng.random() < 0.25
    return dict(_NORM, dtype=dtype, B=B, T=rows * G, C=C, gate_tokens=1 if each else rows,
                dir=rng.choice(["fwd", "bwd", "both"]), res_scale=rng.choice([1.0, 0.5]))


# ---------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def randn(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def unit(*shape):
        x = randn(*shape)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)

    s = dict(case=dict(c))
    if c["op"] == "norm":
        B, T, C = c["B"], c["T"], c["C"]
        s["x"] = (2.0 * randn(B, T, C)).to(dt)
        s["y"] = (randn(B, T, C) * torch.exp(randn(B, T, 1))).to(dt)     # block outputs of varying scale
        s["gate"] = (0.5 * randn(B, T // c["gate_tokens"], C)).to(dt)
        s["w_post"], s["w_pre"] = 1.0 + 0.2 * randn(C), 1.0 + 0.2 * randn(C)
        if c["dir"] != "fwd":
            s["du"], s["dr"] = randn(B, T, C).to(dt), randn(B, T, C).to(dt)
        return s
    lead = (c["N"], c["L"]) if c["op"] == "step" else (c["B"], c["T"])
    H, Dk, Dv = c["H"], c["Dk"], c["Dv"]
    Hk = c.get("Hk", H)
    s["q"], s["k"] = unit(*lead, Hk, Dk), unit(*lead, Hk, Dk)
    s["v"] = randn(*lead, H, Dv).to(dt)
    s["alpha"] = torch.exp(-torch.nn.functional.softplus(randn(*lead, H) + c["mu"]))
    s["beta"] = torch.sigmoid(randn(*lead, H))
    if c["op"] == "backward":
        s["state"] = 0.1 * randn(c["B"], H, Dk, Dv) if c["state"] else None
        s["dout"] = randn(*lead, H, Dv).to(dt)
        s["dstate"] = 0.1 * randn(c["B"], H, Dk, Dv) if c["state"] else None
        return s
    N, P = c["N"], c["P"]
    s["pool"] = 0.1 * randn(P, H, Dk, Dv)
    s["new"] = s["pool"].clone()                     # states after the tokens; other slots stay
    slots = torch.randperm(P, generator=gen, device=dev)[:N].to(torch.int32)
    if c["pad"]:
        slots[N - c["pad"]:] = -1                    # a batch of fixed size that is not full
    s["slots"] = slots
    s["lengths"] = None
    if c["ragged"]:
        s["lengths"] = torch.randint(0, c["L"] + 1, (N,), generator=gen, device=dev, dtype=torch.int32)
    s["out"] = torch.zeros(*lead, H, Dv, dtype=dt, device=dev)
    return s


def run(s):
    c = s["case"]
    if own:
        return _own(s)
    if c["op"] == "step":
        return _plain_step(s)
    if c["op"] == "backward":
        return _plain_backward(s)
    res = ()
    if c["dir"] != "bwd":
        res += _plain_norm(s)
    if c["dir"] != "fwd":
        res += _plain_norm_grad(s)
    return res


def _own(s):
    import paper_2605_30409_amd as gdn
    c = s["case"]
    if c["op"] == "step":
        return gdn.step(s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["pool"], slots=s["slots"],
                        lengths=s["lengths"], out=s["out"], state_out=s["new"])
    if c["op"] == "backward":
        return gdn.backward(s["q"], s["k"], s["v"], s["alpha"], s["beta"], s["state"], s["dout"], s["dstate"])
    res = ()
    args = (s["x"], s["y"], s["gate"], s["w_post"], s["w_pre"])
    kw = dict(gate_tokens=c["gate_tokens"], res_scale=c["res_scale"])
    if c["dir"] != "bwd":
        res += gdn.block_norm(*args, **kw)
    if c["dir"] != "fwd":
        res += gdn.block_norm_backward(*args, s["du"], s["dr"], **kw)
    return res


def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "norm":
        n, C = c["B"] * c["T"], c["C"]
        g = n // c["gate_tokens"]
        by = fl = 0
        if c["dir"] != "bwd":                        # x, y in; r, u out
            by += (4 * n + g) * C * esz + 8 * C
            fl += 11 * n * C
        if c["dir"] != "fwd":                        # x, y, du, dr in; dx, dy out
            by += (6 * n + 2 * g) * C * esz + 16 * C
            fl += 30 * n * C
        return {"bytes": by, "flops": fl}
    H, Dk, Dv = c["H"], c["Dk"], c["Dv"]
    if c["op"] == "step":
        rows = c["N"] - c["pad"]
        tok = rows * c["L"] / (2.0 if c["ragged"] else 1.0)
        by = tok * (2 * c["Hk"] * Dk + 2 * H * Dv) * esz + 8 * tok * H + 8 * rows * H * Dk * Dv
        return {"bytes": by, "flops": 6 * tok * H * Dk * Dv}
    n = c["B"] * c["T"] * H
    by = n * (4 * Dk + 3 * Dv) * esz + 16 * n + (12 if c["state"] else 4) * c["B"] * H * Dk * Dv
    # per token: prediction and update; q dO^T, G^T k, G u, H du, k du^T, H dO and <G, H>
    return {"bytes": by, "flops": 18 * n * Dk * Dv}


# ---------------------------------------------------------------------------
# Plain forms.

def _plain_step(s):
    c = s["case"]
    rep = c["H"] // c["Hk"]
    q, k = (s[n].float().repeat_interleave(rep, 2) for n in ("q", "k"))
    v, alpha, beta = s["v"].float(), s["alpha"], s["beta"]
    live = s["slots"] >= 0
    at = s["slots"].clamp_min(0).long()
    S = s["pool"][at]                                                    # [N, H, Dk, Dv]
    for t in range(c["L"]):
        on = live if s["lengths"] is None else live & (t < s["lengths"])
        kt, qt = k[:, t].unsqueeze(-1), q[:, t].unsqueeze(-1)
        A = alpha[:, t, :, None, None] * S
        u = beta[:, t].unsqueeze(-1) * (v[:, t] - (A * kt).sum(2))
        A = A + kt * u.unsqueeze(2)
        o = (A * qt).sum(2).to(s["out"].dtype)
        S = torch.where(on[:, None, None, None], A, S)
        s["out"][:, t] = torch.where(on[:, None, None], o, s["out"][:, t])
    n = c["N"] - c["pad"]                                                # padding stands at the end
    s["new"][at[:n]] = S[:n]
    return s["out"], s["new"]


def _chunks(x, NC, fill=0.0):
    """[B, T, H, ...] to fp32 chunks [B, H, NC, 64, ...], the tail filled."""
    B, T, H = x.shape[:3]
    y = torch.full((B, NC * 64, H) + tuple(x.shape[3:]), fill, dtype=torch.float32, device=x.device)
    y[:, :T] = x
    y = y.reshape((B, NC, 64, H) + tuple(x.shape[3:]))
    return y.movedim(3, 1).contiguous()


def _tokens(x, T):
    """Chunks back to [B, T, H, ...]."""
    y = x.movedim(1, 3)
    return y.reshape((y.shape[0], -1) + tuple(y.shape[3:]))[:, :T]


def _plain_backward(s):
    c = s["case"]
    T, NC = c["T"], (c["T"] + 63) // 64
    q, k, v, do = (_chunks(s[n], NC) for n in ("q", "k", "v", "dout"))
    b = _chunks(s["beta"], NC).unsqueeze(-1)
    a = _chunks(s["alpha"], NC, 1.0)
    g = torch.cumsum(torch.log(a.clamp_min(1e-38)).double(), -1)         # decay since the chunk's start
    g = torch.cat([torch.zeros_like(g[..., :1]), g], -1)                 # g[0]: before the first token
    low = torch.ones(64, 64, device=q.device).tril()
    D = torch.exp((g[..., 1:, None] - g[..., None, 1:]).clamp_max(0.0)).float() * low
    gam = torch.exp(g[..., 1:]).float().unsqueeze(-1)
    tail = torch.exp(g[..., -1:] - g[..., 1:]).float().unsqueeze(-1)
    gC = gam[..., -1:, :]
    skk, sqk = k @ k.mT, q @ k.mT
    strict = D.tril(-1)
    M = -(strict * skk * b.mT)                                           # (I - M)^-1, M^64 = 0
    R = torch.eye(64, device=q.device) + M
    for _ in range(5):
        M = M @ M
        R = R + M @ R
    zero = torch.zeros(c["B"], c["H"], c["Dk"], c["Dv"], device=q.device)
    H = zero if s["state"] is None else s["state"]
    Hs, es = [], []
    for i in range(NC):                                                  # states forward
        e = R[:, :, i] @ (v[:, :, i] - gam[:, :, i] * (k[:, :, i] @ H))
        Hs.append(H)
        es.append(e)
        H = gC[:, :, i] * H + k[:, :, i].mT @ (tail[:, :, i] * b[:, :, i] * e)
    H, e = torch.stack(Hs, 2), torch.stack(es, 2)
    att = (sqk * D).mT @ do
    G = zero if s["dstate"] is None else s["dstate"]
    Gs, dvs = [None] * NC, [None] * NC
    for i in reversed(range(NC)):                                        # gradients of the states backward
        dv = R[:, :, i].mT @ (b[:, :, i] * (att[:, :, i] + tail[:, :, i] * (k[:, :, i] @ G)))
        Gs[i], dvs[i] = G, dv
        G = gC[:, :, i] * G + q[:, :, i].mT @ (gam[:, :, i] * do[:, :, i]) - k[:, :, i].mT @ (gam[:, :, i] * dv)
    dstate, G, dv = G, torch.stack(Gs, 2), torch.stack(dvs, 2)
    Z, F = do @ e.mT, dv @ e.mT
    PQ, PV, PE = do @ H.mT, dv @ H.mT, e @ G.mT
    G1, G2 = Z * D * b.mT, F * strict * b.mT
    dq = gam * PQ + G1 @ k
    dk = G1.mT @ q + tail * b * PE - gam * PV - (G2 + G2.mT) @ k
    kpe = (k * PE).sum(-1)
    db = (D * sqk * Z).sum(-2) - (strict * skk * F).sum(-2) + tail.squeeze(-1) * kpe
    # dalpha_t: what of later rows i >= t depends on earlier columns j < t, each
    # through the decays on either side of alpha_t; column 0 is the entry state,
    # the last row the exit state
    X = torch.zeros(q.shape[:3] + (65, 65), device=q.device)
    X[..., :64, 1:] = b.mT * (sqk * Z - skk * F) * low.tril(-1)
    X[..., :64, 0] = (q * PQ).sum(-1) - (k * PV).sum(-1)
    X[..., 64, 1:] = b.squeeze(-1) * kpe
    X[..., 64, 0] = (G * H).sum((-1, -2))
    since = torch.cat([g[..., 1:], g[..., -1:]], -1)                     # of row i
    past = torch.ones(65, 64, device=q.device).tril()                    # i >= t
    before = torch.ones(64, 65, device=q.device).tril()                  # j < t
    left = torch.exp((since[..., :, None] - g[..., None, 1:]).clamp_max(0.0)).float() * past
    right = torch.exp((g[..., :-1, None] - g[..., None, :]).clamp_max(0.0)).float() * before
    da = (left * (X @ right.mT)).sum(-2)
    return tuple(_tokens(x, T).to(s["q"].dtype) for x in (dq, dk, dv)) + (_tokens(da, T), _tokens(db, T), dstate)


def _norm_parts(s):
    c = s["case"]
    x, y = s["x"].float(), s["y"].float()
    gate = s["gate"].float().repeat_interleave(c["gate_tokens"], 1)
    iy = torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6)
    n = y * iy * s["w_post"]
    r = c["res_scale"] * x + gate * n
    ir = torch.rsqrt((r * r).mean(-1, keepdim=True) + 1e-6)
    return y, gate, iy, n, r, ir


def _plain_norm(s):
    y, gate, iy, n, r, ir = _norm_parts(s)
    return r.to(s["x"].dtype), (r * ir * s["w_pre"]).to(s["x"].dtype)


def _plain_norm_grad(s):
    c = s["case"]
    y, gate, iy, n, r, ir = _norm_parts(s)
    du, dr = s["du"].float(), s["dr"].float()
    rh, yh = r * ir, y * iy
    d = du * s["w_pre"]
    g = dr + ir * (d - rh * (d * rh).mean(-1, keepdim=True))             # gradient of r
    dn = gate * g
    d2 = dn * s["w_post"]
    dy = iy * (d2 - yh * (d2 * yh).mean(-1, keepdim=True))
    B, T, C = g.shape
    dgate = (n * g).reshape(B, T // c["gate_tokens"], c["gate_tokens"], C).sum(2)
    dt = s["x"].dtype
    return ((c["res_scale"] * g).to(dt), dy.to(dt), dgate.to(dt), (dn * yh).sum((0, 1)), (du * rh).sum((0, 1)))


# ---------------------------------------------------------------------------
# The same results in fp64, from the definitions.

def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "step":
        return _exact_step(s)
    if c["op"] == "backward":
        return _exact_backward(s)
    x, y = s["x"].double().requires_grad_(), s["y"].double().requires_grad_()
    gate, wp, wr = (s[n].double().requires_grad_() for n in ("gate", "w_post", "w_pre"))
    rows = torch.arange(c["T"], device=x.device) // c["gate_tokens"]
    n = wp * y / ((y ** 2).sum(-1, keepdim=True) / c["C"] + 1e-6) ** 0.5
    r = c["res_scale"] * x + gate[:, rows] * n
    u = wr * r / ((r ** 2).sum(-1, keepdim=True) / c["C"] + 1e-6) ** 0.5
    res = ()
    if c["dir"] != "bwd":
        res += (r.detach(), u.detach())
    if c["dir"] != "fwd":
        loss = (u * s["du"].double()).sum() + (r * s["dr"].double()).sum()
        res += torch.autograd.grad(loss, (x, y, gate, wp, wr))
    return res


def _exact_step(s):
    """Sequence by sequence, token by token."""
    c = s["case"]
    out, new = s["out"].double(), s["pool"].double()
    slots = s["slots"].tolist()
    lengths = [c["L"]] * c["N"] if s["lengths"] is None else s["lengths"].tolist()
    head = torch.arange(c["H"], device=out.device) // (c["H"] // c["Hk"])
    for n, (slot, m) in enumerate(zip(slots, lengths)):
        for t in range(m if slot >= 0 else 0):
            k, q = s["k"][n, t, head].double(), s["q"][n, t, head].double()
            S = s["alpha"][n, t].double()[:, None, None] * new[slot]
            err = s["v"][n, t].double() - torch.matmul(k[:, None], S)[:, 0]
            S = S + s["beta"][n, t].double()[:, None, None] * k[:, :, None] * err[:, None]
            new[slot] = S
            out[n, t] = torch.matmul(q[:, None], S)[:, 0]
    return out, new


def _exact_backward(s):
    """The recurrence token by token, then its adjoint in reverse."""
    c = s["case"]
    B, T, H, Dk, Dv = c["B"], c["T"], c["H"], c["Dk"], c["Dv"]
    q, k, v, a, b, do = (s[n].double() for n in ("q", "k", "v", "alpha", "beta", "dout"))
    S = torch.zeros(B, H, Dk, Dv, dtype=torch.float64, device=q.device) if s["state"] is None else s["state"].double()
    states = torch.empty(T + 1, B, H, Dk, Dv, dtype=torch.float64, device=q.device)
    states[0] = S
    err = torch.empty_like(v)
    for t in range(T):
        S = a[:, t, :, None, None] * S
        err[:, t] = v[:, t] - (k[:, t].unsqueeze(-1) * S).sum(2)
        S = torch.addcmul(S, k[:, t].unsqueeze(-1), (b[:, t].unsqueeze(-1) * err[:, t]).unsqueeze(2), out=states[t + 1])
    G = torch.zeros_like(S) if s["dstate"] is None else s["dstate"].double()
    dq, dk, dv, da, db = (torch.empty_like(x) for x in (q, k, v, a, b))
    for t in reversed(range(T)):
        kt, qt, dt = k[:, t].unsqueeze(-1), q[:, t].unsqueeze(-1), do[:, t].unsqueeze(2)
        at, bt, et, S = a[:, t, :, None, None], b[:, t].unsqueeze(-1), err[:, t], states[t]
        dq[:, t] = (states[t + 1] * dt).sum(-1)                          # o = S'^T q
        G = torch.addcmul(G, qt, dt)
        du = (G * kt).sum(2)                                             # S' = a S + k (b e)^T
        dk[:, t] = (G * (bt * et).unsqueeze(2)).sum(-1)
        db[:, t] = (du * et).sum(-1)
        de = bt * du                                                     # e = v - (a S)^T k
        dv[:, t] = de
        dk[:, t] -= at.squeeze(-1) * (S * de.unsqueeze(2)).sum(-1)
        G = torch.addcmul(G, kt, de.unsqueeze(2), value=-1.0)            # now of a S
        da[:, t] = (G * S).sum((-1, -2))
        G = at * G
    return dq, dk, dv, da, db, G
