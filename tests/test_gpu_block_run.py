"""GPU: a whole block in training and in serving, from its convolution over the recurrence, the norms and the gated linear
map to the clipped gradients, against one fp64 autograd graph of the same formulas.

Everything is fp32 and every operator is held to its own formulas elsewhere, to some 100 u of absolute terms with
u = 2^-24; through the six of them a gradient is a sum over 70 tokens and 64 channels of products of those errors, and
2000 u of the largest element leaves room for terms that cancel.
"""
import pytest

pytestmark = pytest.mark.gpu

TOL = 2000 * 2.0 ** -24
B, T, H, D, F = 2, 70, 2, 64, 96
C = H * D


def params(seed=3):
    import torch
    g = torch.Generator().manual_seed(seed)

    def rn(*s):
        return torch.randn(s, generator=g)
    p = {n + i: v for i in "qkv" for n, v in (("w_", rn(C, 4) / 2), ("b_", 0.1 * rn(C)))}
    p.update(w_post=1 + 0.2 * rn(C), w_pre=1 + 0.2 * rn(C), w_gate=rn(F, C) / C ** 0.5, w_up=rn(F, C) / C ** 0.5)
    t = dict(packed=rn(B, T, 3 * C) / D ** 0.5, alpha=torch.sigmoid(rn(B, T, H) + 2), beta=torch.sigmoid(rn(B, T, H)), res=rn(B, T, C),
             dh=rn(B, T, F))
    return {n: v.cuda() for n, v in p.items()}, {n: v.cuda() for n, v in t.items()}


def parts(packed):
    return {i: packed[..., n * C:(n + 1) * C] for n, i in enumerate("qkv")}


def forward(gdn, p, t):
    """The block, and what its gradient needs."""
    import torch
    s = {}
    for i, x in parts(t["packed"]).items():
        s[i] = gdn.short_conv(x, p["w_" + i], p["b_" + i], want_state=False)[0].view(B, T, H, D)
    s["o"], _ = gdn.forward(s["q"], s["k"], s["v"], t["alpha"], t["beta"], torch.zeros(B, H, D, D, device="cuda"))
    s["o"] = s["o"].view(B, T, C)
    s["r"], s["u"] = gdn.block_norm(t["res"], s["o"], None, p["w_post"], p["w_pre"])
    return gdn.gated_linear(s["u"], p["w_gate"], p["w_up"]), s


def backward(gdn, p, t, s):
    """Gradients of all weights and of the packed projection, written straight into its parts."""
    import torch
    g = {}
    du, g["w_gate"], g["w_up"] = gdn.gated_linear_backward(s["u"], p["w_gate"], p["w_up"], t["dh"])
    _, do, _, g["w_post"], g["w_pre"] = gdn.block_norm_backward(t["res"], s["o"], None, p["w_post"], p["w_pre"], du)
    d = dict(zip("qkv", gdn.backward(s["q"], s["k"], s["v"], t["alpha"], t["beta"], None, do.view(B, T, H, D))))
    g["packed"] = torch.empty_like(t["packed"])
    for i, x in parts(t["packed"]).items():
        _, g["w_" + i], g["b_" + i], _ = gdn.short_conv_backward(x, p["w_" + i], p["b_" + i], None, d[i].view(B, T, C), want_dstate=False,
                                                                 dx=parts(g["packed"])[i])
    return g


def plain(p, t):
    import torch
    p, t = ({n: v.double().requires_grad_() for n, v in a.items()} for a in (p, t))
    s = {}
    for i, x in parts(t["packed"]).items():
        xe = torch.cat([x.new_zeros(B, 3, C), x], 1)
        z = p["b_" + i] + sum(p["w_" + i][:, j] * xe[:, j:j + T] for j in range(4))
        s[i] = (z * torch.sigmoid(z)).view(B, T, H, D)
    S, o = t["packed"].new_zeros(B, H, D, D), []
    for n in range(T):
        k = s["k"][:, n].unsqueeze(-1)
        S = t["alpha"][:, n, :, None, None] * S
        S = S + t["beta"][:, n, :, None, None] * k * (s["v"][:, n] - (k * S).sum(2)).unsqueeze(2)
        o.append((s["q"][:, n].unsqueeze(-1) * S).sum(2))
    o = torch.stack(o, 1).reshape(B, T, C)
    r = t["res"] + p["w_post"] * o * torch.rsqrt(o.square().mean(-1, keepdim=True) + 1e-6)
    u = p["w_pre"] * r * torch.rsqrt(r.square().mean(-1, keepdim=True) + 1e-6)
    g = u @ p["w_gate"].T
    h = g * torch.sigmoid(g) * (u @ p["w_up"].T)
    names = list(p) + ["packed"]
    grads = torch.autograd.grad((h * t["dh"]).sum(), [p[n] if n in p else t[n] for n in names])
    return h.detach(), dict(zip(names, grads))


def near(name, got, ref):
    assert got.isfinite().all(), name
    d = float((got.double() - ref).abs().max() / ref.abs().max())
    assert d <= TOL, (name, d)


def test_a_training_step(gdn):
    import torch
    p, t = params()
    h, s = forward(gdn, p, t)
    g = backward(gdn, p, t, s)
    ref_h, ref = plain(p, t)
    near("h", h, ref_h)
    assert set(g) == set(ref)
    for n in ref:
        near(n, g[n], ref[n])
    # clipping: the weights' gradients in place, then an update
    grads = [g[n] for n in p]
    want = torch.stack([ref[n].square().sum() for n in p]).sum().sqrt()
    norm, out = gdn.clip_grads(grads, 0.5)
    assert abs(float(norm / want) - 1) < TOL and out[0] is grads[0]
    for n in p:
        near(n, g[n], ref[n] * 0.5 / (want + 1e-6))
    assert abs(float(gdn.grad_norm(grads)) - 0.5) < 1e-5


def test_a_captured_training_step(gdn):
    """Forward, backward and clipping in one graph, replayed on other inputs beside eager steps."""
    import torch
    p, t = params()

    def step():
        h, s = forward(gdn, p, t)
        g = backward(gdn, p, t, s)
        return [h, *gdn.clip_grads([g[n] for n in p], 0.5)[1], g["packed"]]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        assert all(torch.equal(a, b) for a, b in zip(got, step())), i
        t["packed"].mul_(-0.9)
        torch.cuda.synchronize()


def test_a_server(gdn):
    """Prompts, then tokens one and three at a time from pools of windows and states, against the whole call."""
    import torch
    p, t = params(5)
    h, _ = forward(gdn, p, t)
    n0, P = 50, 5
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    windows = {i: torch.zeros(P, 3, C, device="cuda") for i in "qkv"}
    states = torch.zeros(P, H, D, D, device="cuda")
    y = {}
    for i, x in parts(t["packed"]).items():
        y[i], windows[i][slots.long()] = gdn.short_conv(x[:, :n0], p["w_" + i], p["b_" + i])
    a = {i: v.view(B, n0, H, D) for i, v in y.items()}
    _, states[slots.long()] = gdn.forward(a["q"], a["k"], a["v"], t["alpha"][:, :n0].contiguous(), t["beta"][:, :n0].contiguous(), torch.zeros(B, H, D, D, device="cuda"))
    at = n0
    for n in (1, 1, 3, 1, 3, 1):
        a = {}
        for i, x in parts(t["packed"]).items():
            a[i] = gdn.short_conv_step(x[:, at:at + n], p["w_" + i], p["b_" + i], windows[i], slots=slots)[0].view(B, n, H, D)
        o, _ = gdn.step(a["q"], a["k"], a["v"], t["alpha"][:, at:at + n].contiguous(), t["beta"][:, at:at + n].contiguous(), states, slots=slots)
        _, u = gdn.block_norm(t["res"][:, at:at + n].contiguous(), o.view(B, n, C), None, p["w_post"], p["w_pre"])
        near("h", gdn.gated_linear(u, p["w_gate"], p["w_up"]), h[:, at:at + n].double())
        at += n


def test_two_streams_at_once(gdn):
    """Calls on two streams, each with workspaces of its own, do not meet."""
    import torch
    (p, t), (p2, t2) = params(1), params(2)
    want = [backward(gdn, p, t, forward(gdn, p, t)[1]), backward(gdn, p2, t2, forward(gdn, p2, t2)[1])]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(3):
        got = []
        for s, (a, b) in zip(streams, ((p, t), (p2, t2))):
            with torch.cuda.stream(s):
                got.append(backward(gdn, a, b, forward(gdn, a, b)[1]))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert all(torch.equal(w[n], g[n]) for n in w)
