"""GPU: gradient of the token-wise chunk forward against the recurrence's adjoint in fp64,
token by token, and against differences.

Tolerances, as the 2-norm of the error over that of the result.  fp32 path: every
product is a sum of at most 128 rounded terms, off by about sqrt(128) 2^-24 = 7e-7 of
its size when the roundings are independent; no result passes through more than
some 12 products in a row, 7e-7 sqrt(12) = 2.4e-6 in quadrature, and the bound is four
times that, 1e-5.  bf16 path: operands that are not inputs are fp32 in three planes, with the
same errors, and the bound of fp32 results is the same; bf16 results add half a step,
2^-8 of each value.  No single element may be off by more than 40 times the bound (plus its half
step) relative to the result's rms.
"""
import pytest

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-5, "bf16": 1e-5}
NAMES = ("dq", "dk", "dv", "dalpha", "dbeta", "dstate_in")


def make(B, T, H, Dk, Dv, dtype, seed, mu=0.0, state=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(s, generator=g)

    def unit(*s):
        x = rn(*s)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)
    t = dict(q=unit(B, T, H, Dk), k=unit(B, T, H, Dk), v=rn(B, T, H, Dv).to(dt),
             alpha=torch.exp(-torch.nn.functional.softplus(rn(B, T, H) + mu)), beta=torch.sigmoid(rn(B, T, H)),
             state_in=0.3 * rn(B, H, Dk, Dv) if state else None, dout=rn(B, T, H, Dv).to(dt),
             dstate_out=0.3 * rn(B, H, Dk, Dv) if state else None)
    return {n: None if x is None else x.cuda() for n, x in t.items()}


def host(t):
    return {n: None if x is None else x.double().cpu() for n, x in t.items()}


def recurrence(t):
    """Outputs, errors and all states of the forward, fp64."""
    import torch
    q, k, v, a, b = (t[n] for n in ("q", "k", "v", "alpha", "beta"))
    B, T, H, Dk = q.shape
    S = t["state_in"] if t["state_in"] is not None else torch.zeros(B, H, Dk, v.shape[-1], dtype=torch.float64)
    out, err, states = [], [], [S]
    for i in range(T):
        S = a[:, i, :, None, None] * S
        e = v[:, i] - (k[:, i].unsqueeze(-1) * S).sum(2)
        S = S + k[:, i].unsqueeze(-1) * (b[:, i].unsqueeze(-1) * e).unsqueeze(2)
        out.append((q[:, i].unsqueeze(-1) * S).sum(2))
        err.append(e)
        states.append(S)
    return torch.stack(out, 1), err, states


def adjoint(t):
    import torch
    q, k, v, a, b, do = (t[n] for n in ("q", "k", "v", "alpha", "beta", "dout"))
    _, err, states = recurrence(t)
    G = t["dstate_out"] if t["dstate_out"] is not None else torch.zeros_like(states[0])
    dq, dk, dv, da, db = (torch.empty_like(x) for x in (q, k, v, a, b))
    for i in reversed(range(q.shape[1])):
        ki, bi = k[:, i].unsqueeze(-1), b[:, i].unsqueeze(-1)
        dq[:, i] = (states[i + 1] * do[:, i].unsqueeze(2)).sum(-1)
        G = G + q[:, i].unsqueeze(-1) * do[:, i].unsqueeze(2)
        du = (G * ki).sum(2)
        db[:, i] = (du * err[i]).sum(-1)
        dv[:, i] = bi * du
        aS = a[:, i, :, None, None] * states[i]
        dk[:, i] = (G * (bi * err[i]).unsqueeze(2)).sum(-1) - (aS * dv[:, i].unsqueeze(2)).sum(-1)
        G = G - ki * dv[:, i].unsqueeze(2)
        da[:, i] = (G * states[i]).sum((-1, -2))
        G = a[:, i, :, None, None] * G
    return dq, dk, dv, da, db, G


def compare(got, ref, dtype, label=""):
    import torch
    for name, x, r in zip(NAMES, got, ref):
        half = 2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0
        x = x.double().cpu()
        assert x.isfinite().all(), (label, name)
        d = (x - r).abs()
        rms = float(r.square().mean().sqrt())
        over = (d - half * r.abs()).clamp_min(0.0)
        rel = float(over.norm()) / max(float(r.norm()), 1e-30)
        print(f"[backward] {label} {name}: {rel:.2e}, largest {float(over.max()) / max(rms, 1e-30):.2e}", flush=True)
        assert rel <= TOL[dtype], (label, name, rel)
        assert float(over.max()) <= 40 * TOL[dtype] * rms, (label, name)


def check(gdn, t, dtype, label=""):
    got = gdn.backward(**t)
    compare(got, adjoint(host(t)), dtype, label)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 130, 200])
def test_lengths(gdn, dtype, Dk, Dv, T):
    check(gdn, make(2, T, 3, Dk, Dv, dtype, T + Dk + 2 * Dv), dtype, f"T{T} {Dk}x{Dv} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mu", [2.0, -3.0, -6.0])
def test_decays(gdn, dtype, mu):
    """Heads that forget fast, remember for long, and hardly forget at all, over 5 chunks."""
    check(gdn, make(1, 300, 9, 64, 64, dtype, 11, mu=mu), dtype, f"mu {mu} {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_states(gdn, dtype):
    """state_in and dstate_out None are zeros; want_dstate=False drops dstate_in."""
    import torch
    t = make(1, 140, 2, 128, 64, dtype, 12, state=False)
    got = check(gdn, t, dtype, "no states")
    z = torch.zeros(1, 2, 128, 64, device="cuda")
    full = gdn.backward(**dict(t, state_in=z, dstate_out=z))
    less = gdn.backward(**t, want_dstate=False)
    assert less[5] is None
    assert all(torch.equal(a, b) for a, b in zip(got, full)) and all(torch.equal(a, b) for a, b in zip(got[:5], less[:5]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_at_their_ends(gdn, dtype):
    """alpha of 0 (a state wiped out, several of them in a chunk and on its borders) and 1,
    beta of 0 and 1: nothing is divided by either."""
    t = make(2, 200, 2, 64, 64, dtype, 13, mu=-3.0)
    for i in (0, 5, 6, 63, 64, 100, 127, 199):
        t["alpha"][0, i] = 0.0
    t["alpha"][1] = 1.0
    t["beta"][:, ::3] = 0.0
    t["beta"][:, 1::3] = 1.0
    check(gdn, t, dtype, f"gate ends {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_small_alphas(gdn, dtype):
    """alpha down to 1e-30: the gradient with respect to it does not vanish with it."""
    import torch
    t = make(1, 128, 2, 64, 64, dtype, 14, mu=-3.0)
    t["alpha"][0, ::7] = 10.0 ** -torch.arange(1, 20, dtype=torch.float32, device="cuda")[:, None].clamp_max(30.0)
    check(gdn, t, dtype, f"small alphas {dtype}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_keys(gdn, dtype):
    """One key in every token with beta = 1: each write replaces the one before (T = (I + N)^-1 has
    entries of size 1 on its first subdiagonal, however large N is)."""
    t = make(1, 130, 2, 64, 128, dtype, 15, mu=-3.0)
    t["k"].zero_()
    t["k"][..., 5] = 1.0
    t["beta"].fill_(1.0)
    check(gdn, t, dtype, f"repeated keys {dtype}")


def test_against_differences(gdn):
    """The fp32 gradient along a direction against central differences of the fp64 recurrence
    (step 1e-4: 1e-8 of truncation), good to 1e-5 of the sum of its absolute terms."""
    import torch
    t = make(1, 100, 2, 64, 64, "f32", 16, mu=-1.0)
    got = gdn.backward(**t)
    h = host(t)
    g = torch.Generator().manual_seed(2)

    def loss(p):
        out, _, states = recurrence(p)
        return float((out * p["dout"]).sum() + (states[-1] * p["dstate_out"]).sum())
    for name, gr in zip(("q", "k", "v", "alpha", "beta", "state_in"), got):
        d = torch.randn(h[name].shape, generator=g, dtype=torch.float64)
        terms = gr.double().cpu() * d
        diff = (loss(dict(h, **{name: h[name] + 1e-4 * d})) - loss(dict(h, **{name: h[name] - 1e-4 * d}))) / 2e-4
        assert abs(float(terms.sum()) - diff) <= 1e-5 * float(terms.abs().sum()), name


def test_gradient_of_the_chunk_forward(gdn):
    """The forward kernel's own outputs change along a direction as the gradient says (fp32,
    a step of 2^-7 in v, in which the outputs are linear)."""
    import torch
    t = make(1, 170, 3, 64, 64, "f32", 17, mu=-2.0)
    args = [t[n] for n in ("q", "k", "v", "alpha", "beta", "state_in")]
    o0, s0 = gdn.forward(*args)
    dv = gdn.backward(**t)[2].double()
    d = torch.randn(t["v"].shape, generator=torch.Generator().manual_seed(3)).cuda()
    args[2] = t["v"] + d
    o1, s1 = gdn.forward(*args)
    terms = dv * (args[2].double() - t["v"].double())
    change = ((o1.double() - o0.double()) * t["dout"].double()).sum() + \
        ((s1.double() - s0.double()) * t["dstate_out"].double()).sum()
    # both sides are fp32 evaluations, the forward to 1e-4 of its outputs' largest at most
    size = (o1.abs().max() * t["dout"].double().norm() + s1.abs().max() * t["dstate_out"].double().norm())
    assert abs(float(terms.sum() - change)) <= 1e-4 * float(size)


def test_nan_stays_in_its_head(gdn):
    import torch
    t = make(2, 150, 3, 64, 64, "bf16", 18)
    ref = gdn.backward(**t)
    t["v"][1, 70, 2, 7] = float("nan")
    t["alpha"][0, 3, 1] = float("nan")
    got = gdn.backward(**t)
    for name, a, b in zip(NAMES, ref, got):
        head = 1 if name == "dstate_in" else 2
        for bi in range(2):
            for h in range(3):
                x, y = a[bi].select(head - 1, h), b[bi].select(head - 1, h)
                if (bi, h) == (0, 1) or ((bi, h) == (1, 2) and name in ("dq", "dk", "dalpha", "dbeta")):
                    assert torch.isnan(y).any(), (name, bi, h)
                else:                       # the loss is linear in v: dv and dstate_in do not depend on it
                    assert torch.equal(x, y), (name, bi, h)


def test_given_outputs_and_workspace(gdn):
    """Outputs that are given, dstate_in over dstate_out, and a workspace of NaNs: the same bits."""
    import torch
    t = make(1, 77, 2, 128, 128, "bf16", 19)
    ref = gdn.backward(**t)
    outs = {n: torch.full_like(x, float("nan")) for n, x in zip(NAMES[:5], ref)}
    ws = gdn.backward_workspace(t["q"], t["v"])
    ws.fill_(0xff)
    ds = t["dstate_out"].clone()
    got = gdn.backward(**dict(t, dstate_out=ds), **outs, dstate_in=ds, ws=ws)
    torch.cuda.synchronize()
    assert got[0] is outs["dq"] and got[5] is ds
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_captured(gdn):
    """In a graph, replayed between eager calls on changing inputs; two graphs with workspaces
    of their own."""
    import torch
    t = make(1, 200, 2, 64, 64, "bf16", 20)
    gdn.backward(**t)
    torch.cuda.synchronize()
    runs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = gdn.backward(**t)
        runs.append((graph, res))
    for i in range(3):
        for graph, _ in runs:
            graph.replay()
        ref = gdn.backward(**t)
        torch.cuda.synchronize()
        for _, res in runs:
            assert all(torch.equal(a, b) for a, b in zip(res, ref)), i
        t["dout"].mul_(0.5)
        t["alpha"].mul_(0.9)


def test_side_stream(gdn):
    import torch
    t = make(2, 90, 2, 64, 128, "f32", 21)
    ref = gdn.backward(**t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gdn.backward(**t, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_heads_and_chunks(gdn, dtype):
    """More heads than eight and more chunks than workgroups are placed in a row; one head against
    fp64, and the call of that head alone gives the same bits."""
    import torch
    t = make(1, 1000, 19, 64, 64, dtype, 22, mu=-3.0)
    got = gdn.backward(**t)
    for h in (0, 18):
        one = {n: None if x is None else (x[:, h:h + 1] if n in ("state_in", "dstate_out") else x[:, :, h:h + 1]).contiguous()
               for n, x in t.items()}
        alone = gdn.backward(**one)
        for name, a, b in zip(NAMES, got, alone):
            sel = a[:, h:h + 1] if name == "dstate_in" else a[:, :, h:h + 1]
            assert torch.equal(sel, b), (name, h)
        compare(alone, adjoint(host(one)), dtype, f"head {h} {dtype}")
