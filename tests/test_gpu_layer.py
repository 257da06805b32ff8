"""GPU: the operators together, as a layer uses them: chunk forward, block norm, their
gradients in reverse, and decoding from the carried state."""
import pytest

pytestmark = pytest.mark.gpu


def inputs(B, T, H, D, seed):
    import torch
    g = torch.Generator().manual_seed(seed)

    def rn(*s):
        return torch.randn(s, generator=g)

    def unit(*s):
        x = rn(*s)
        return x / x.norm(dim=-1, keepdim=True)
    t = dict(q=unit(B, T, H, D), k=unit(B, T, H, D), v=rn(B, T, H, D), alpha=0.8 + 0.2 * torch.rand(B, T, H, generator=g),
             beta=torch.rand(B, T, H, generator=g), x=rn(B, T, H * D), gate=rn(B, 2, H * D), w_post=1 + 0.2 * rn(H * D),
             w_pre=1 + 0.2 * rn(H * D), du=rn(B, T, H * D))
    return {n: x.cuda() for n, x in t.items()}


def plain(p, B, T, H, D):
    """The layer in fp64: recurrence, then the block norm; its output u."""
    import torch
    S = torch.zeros(B, H, D, D, dtype=torch.float64)
    outs = []
    for i in range(T):
        S = p["alpha"][:, i, :, None, None] * S
        e = p["v"][:, i] - (p["k"][:, i].unsqueeze(-1) * S).sum(2)
        S = S + p["k"][:, i].unsqueeze(-1) * (p["beta"][:, i].unsqueeze(-1) * e).unsqueeze(2)
        outs.append((p["q"][:, i].unsqueeze(-1) * S).sum(2))
    y = torch.stack(outs, 1).reshape(B, T, H * D)
    n = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * p["w_post"]
    r = 0.5 * p["x"] + p["gate"].repeat_interleave(T // 2, 1) * n
    return r / (r.square().mean(-1, keepdim=True) + 1e-6).sqrt() * p["w_pre"]


def test_layer_gradient(gdn):
    """fp32: both gradients chained are the gradient of the layer, to 2e-5 (2-norm) of each
    result: the sum of the bounds that the two are held to."""
    import torch
    B, T, H, D = 2, 100, 2, 64
    t = inputs(B, T, H, D, 1)
    y, _ = gdn.forward(t["q"], t["k"], t["v"], t["alpha"], t["beta"])
    border = (t["x"], y.view(B, T, H * D), t["gate"], t["w_post"], t["w_pre"])
    kw = dict(gate_tokens=T // 2, res_scale=0.5)
    r, u = gdn.block_norm(*border, **kw)
    dx, dy, dgate, dwp, dwr = gdn.block_norm_backward(*border, t["du"], **kw)
    dq, dk, dv, da, db, _ = gdn.backward(t["q"], t["k"], t["v"], t["alpha"], t["beta"], None, dy.view(B, T, H, D))
    p = {n: x.double().cpu().requires_grad_(n != "du") for n, x in t.items()}
    ref_u = plain(p, B, T, H, D)
    names = ("q", "k", "v", "alpha", "beta", "x", "gate", "w_post", "w_pre")
    ref = torch.autograd.grad((ref_u * p["du"]).sum(), [p[n] for n in names])
    assert float((u.double().cpu() - ref_u).norm().detach() / ref_u.detach().norm()) <= 2e-5
    for n, a, b in zip(names, (dq, dk, dv, da, db, dx, dgate, dwp, dwr), ref):
        assert float((a.double().cpu() - b).norm() / b.norm()) <= 2e-5, n


def test_layer_decodes_as_it_prefills(gdn):
    """fp32: prefill, then one token at a time through the step and the block norm, against the
    layer over the whole sequence; two fp32 evaluations, each within 1e-4."""
    import torch
    B, T, H, D, n = 2, 90, 2, 64, 4
    t = inputs(B, T, H, D, 2)
    y, _ = gdn.forward(t["q"], t["k"], t["v"], t["alpha"], t["beta"])
    w = (t["w_post"], t["w_pre"])
    _, whole = gdn.block_norm(t["x"], y.view(B, T, H * D), None, *w)
    seq = [t[k] for k in ("q", "k", "v", "alpha", "beta")]
    _, state = gdn.forward(*(x[:, :T - n].contiguous() for x in seq))
    pool = torch.zeros(5, H, D, D, device="cuda")
    slots = torch.tensor([3, 1], dtype=torch.int32, device="cuda")
    pool[slots.long()] = state
    for i in range(T - n, T):
        y, _ = gdn.step(*(x[:, i:i + 1].contiguous() for x in seq), pool, slots=slots)
        _, u = gdn.block_norm(t["x"][:, i:i + 1].contiguous(), y.view(B, 1, H * D), None, *w)
        assert float((u[:, 0] - whole[:, i]).abs().max()) <= 2e-4 * float(whole.abs().max()), i


def test_calls_on_two_streams_at_once(gdn):
    """Each call has a workspace of its own: gradients that run beside each other keep their bits."""
    import torch
    a, b = inputs(2, 700, 3, 64, 3), inputs(2, 700, 3, 64, 4)

    def run(t, stream=None):
        dout = t["du"].view(t["v"].shape)
        g = gdn.backward(t["q"], t["k"], t["v"], t["alpha"], t["beta"], None, dout, stream=stream)
        n = gdn.block_norm_backward(t["x"], t["du"], t["gate"], t["w_post"], t["w_pre"], t["x"], gate_tokens=350,
                                    stream=stream)
        return g + n
    ref = run(a), run(b)
    torch.cuda.synchronize()
    s = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        got = run(a, s[0]), run(b, s[1])
        torch.cuda.synchronize()
        for x, y in zip(got, ref):
            assert all(torch.equal(p, q) for p, q in zip(x, y))
