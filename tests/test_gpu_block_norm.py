"""GPU: norms, gate and scaled residual between two blocks, forward and gradient,
against the formulas in fp64 and against differences.

Tolerances, with u = 2^-24: a mean of squares is a sum of depth at most 30 (8
channels a thread, 6 steps over a wave, 16 waves), so iy is off by at most 20 u of its
value and n by 23 u; r by 25 u of m_r = |res_scale x| + |gate n|.  With K = rms(m_r) /
rms(r), ir is off by (20 + 25 K) u, u by (50 + 25 K) u of its value in m_r.  The
gradient's terms then go through two more sums of depth 30 and fewer than 30
roundings: at most (200 + 100 K) u of the same formula with every term taken
absolutely.  Sums over n rows add (n + 32) u of the sum of absolute terms.  bf16
results add half a step, 2^-8 of the value.
"""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(B, T, C, gt, dtype, seed, gated=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(s, generator=g)
    t = dict(x=(2 * rn(B, T, C)).to(dt), y=(rn(B, T, C) * torch.exp(rn(B, T, 1))).to(dt),
             gate=rn(B, T // gt, C).to(dt) if gated else None, w_post=1 + 0.3 * rn(C), w_pre=1 + 0.3 * rn(C),
             du=rn(B, T, C).to(dt), dr=rn(B, T, C).to(dt))
    return {n: None if x is None else x.cuda() for n, x in t.items()}


def host(t):
    return {n: None if x is None else x.double().cpu() for n, x in t.items()}


def gates(t, gt):
    import torch
    return torch.ones(()).double() if t["gate"] is None else t["gate"].repeat_interleave(gt, 1)


def parts(t, gt, rs, eps):
    ga = gates(t, gt)
    iy = 1 / (t["y"].square().mean(-1, keepdim=True) + eps).sqrt()
    n = t["y"] * iy * t["w_post"]
    r = rs * t["x"] + ga * n
    ir = 1 / (r.square().mean(-1, keepdim=True) + eps).sqrt()
    m = abs(rs) * t["x"].abs() + (ga * n).abs()
    # K: how much larger the terms of r are than r
    K = (m.square().mean(-1, keepdim=True) / (r.square().mean(-1, keepdim=True) + eps)).sqrt().clamp_min(1.0)
    return ga, iy, n, r, ir, m, K


def close(name, got, ref, tol, dtype):
    half = 2.0 ** -8 if str(dtype).endswith("bfloat16") else U
    d = (got.double().cpu() - ref).abs()
    assert got.double().cpu().isfinite().all(), name
    assert (d <= tol + half * ref.abs()).all(), (name, float((d - half * ref.abs() - tol).max()), float(d.max()))


def check_forward(t, r, u, gt, rs, eps=1e-6):
    h = host(t)
    ga, iy, n, rr, ir, m, K = parts(h, gt, rs, eps)
    close("r", r, rr, 25 * U * m, r.dtype)
    close("u", u, rr * ir * h["w_pre"], (50 + 25 * K) * U * m * ir * h["w_pre"].abs(), u.dtype)


def grad(h, gt, rs, eps, take=lambda x: x, minus=-1.0):
    """The gradient's formulas; take=abs, minus=+1: with every term absolute."""
    ga, iy, n, r, ir, m, K = parts(h, gt, rs, eps)
    hh = (m if minus > 0 else r) * ir
    ga, n, wp, wr = take(ga), take(n), take(h["w_post"]), take(h["w_pre"])
    du, dr, yh = take(h["du"]), take(h["dr"]) if h["dr"] is not None else 0.0, take(h["y"]) * iy
    d = du * wr
    g = dr + ir * (d + minus * hh * (d * hh).mean(-1, keepdim=True))
    d2 = ga * g * wp
    dy = iy * (d2 + minus * yh * (d2 * yh).mean(-1, keepdim=True))
    ng = n * g
    return dict(dx=take(h["x"].new_tensor(rs)) * g, dy=dy, dgate=ng, dw_post=ga * g * yh, dw_pre=du * hh), K


def check_grad(t, got, gt, rs, eps=1e-6):
    import torch
    h = host(t)
    ref, K = grad(h, gt, rs, eps)
    mag, _ = grad(h, gt, rs, eps, torch.abs, 1.0)
    B, T, C = h["x"].shape
    c = (200 + 100 * K) * U
    for name, x in zip(("dx", "dy", "dgate", "dw_post", "dw_pre"), got):
        if name == "dgate" and h["gate"] is None:
            assert x is None
            continue
        r, m = ref[name], mag[name] * c
        if name == "dgate":
            rows = gt
            r, m = (z.expand(B, T, C).reshape(B, T // gt, gt, C).sum(2) for z in (r, m + (rows + 32) * U * mag[name]))
        elif name.startswith("dw"):
            r, m = (z.expand(B, T, C).sum((0, 1)) for z in (r, m + (B * T + 32) * U * mag[name]))
        close(name, x, r, m, x.dtype)


SHAPES = [(1, 1, 1, 1), (1, 1, 8, 1), (2, 3, 7, 3), (1, 5, 64, 5), (3, 4, 65, 2), (1, 6, 512, 1), (2, 10, 513, 5),
          (1, 12, 1000, 4), (1, 3, 1024, 3), (2, 70, 129, 35), (1, 9, 2048, 9), (1, 4, 2051, 2), (1, 3, 4096, 1),
          (1, 2, 8191, 2), (1, 2, 8192, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,C,gt", SHAPES)
def test_forward(gdn, dtype, B, T, C, gt):
    import torch
    t = make(B, T, C, gt, dtype, B + T + C)
    r, u = gdn.block_norm(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], gate_tokens=gt, res_scale=0.5)
    torch.cuda.synchronize()
    check_forward(t, r, u, gt, 0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,C,gt", SHAPES)
def test_gradient(gdn, dtype, B, T, C, gt):
    import torch
    t = make(B, T, C, gt, dtype, 3 * B + T + C)
    got = gdn.block_norm_backward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], t["du"], t["dr"], gate_tokens=gt,
                                  res_scale=-1.5)
    torch.cuda.synchronize()
    check_grad(t, got, gt, -1.5)


@pytest.mark.parametrize("B,T,gt", [(1, 2000, 2000), (1, 2000, 1000), (2, 1500, 1), (1, 2000, 5), (1, 3000, 3), (3, 700, 7),
                                    (1, 1153, 1153), (1, 6000, 6000), (1, 6000, 3000), (2, 4500, 1), (1, 6000, 5),
                                    (1, 9000, 3), (3, 2100, 7), (1, 4609, 4609), (1, 140000, 4)])
def test_strips(gdn, B, T, gt):
    """Many rows: gate rows that span several strips, that fill strips and of one token,
    with a last strip that is short."""
    import torch
    t = make(B, T, 72 if T < 10000 else 16, gt, "f32", T + gt)
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    r, u = gdn.block_norm(*args, gate_tokens=gt)
    got = gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=gt)
    torch.cuda.synchronize()
    check_forward(t, r, u, gt, 1.0)
    check_grad(t, got, gt, 1.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_gate_or_dr(gdn, dtype):
    import torch
    t = make(2, 9, 200, 1, dtype, 5, gated=False)
    t["dr"] = None
    args = (t["x"], t["y"], None, t["w_post"], t["w_pre"])
    r, u = gdn.block_norm(*args, gate_tokens=3)
    got = gdn.block_norm_backward(*args, t["du"], gate_tokens=3)
    torch.cuda.synchronize()
    check_forward(t, r, u, 3, 1.0)
    check_grad(t, got, 3, 1.0)


def test_zero_rows(gdn):
    """Rows of zeros, in y and in both: eps alone is under the root."""
    import torch
    t = make(1, 6, 40, 2, "f32", 8)
    t["y"][:, 1] = 0
    t["y"][:, 4] = 0
    t["x"][:, 4] = 0
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    r, u = gdn.block_norm(*args, gate_tokens=2, eps=1e-4)
    got = gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=2, eps=1e-4)
    torch.cuda.synchronize()
    check_forward(t, r, u, 2, 1.0, 1e-4)
    check_grad(t, got, 2, 1.0, 1e-4)


def test_nan_stays_in_its_row(gdn):
    import torch
    t = make(1, 40, 96, 40, "bf16", 9)
    args = [t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"]]
    r0, u0 = gdn.block_norm(*args, gate_tokens=40)
    bad = t["y"].clone()
    bad[0, 17, 3] = float("nan")
    bad[0, 23, 90] = float("inf")
    args[1] = bad
    r, u = gdn.block_norm(*args, gate_tokens=40)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[17] = keep[23] = False
    assert torch.equal(r[0, keep], r0[0, keep]) and torch.equal(u[0, keep], u0[0, keep])
    assert torch.isnan(r[0, 17]).all() and torch.isnan(u[0, 23]).all()


def test_in_place(gdn):
    """r over x, u over y; dx over dr, dy over du: the same bits."""
    import torch
    t = make(2, 30, 300, 15, "bf16", 10)
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    r, u = gdn.block_norm(*args, gate_tokens=15)
    g = gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=15)
    x, y = t["x"].clone(), t["y"].clone()
    gdn.block_norm(x, y, *args[2:], gate_tokens=15, r=x, u=y)
    du, dr = t["du"].clone(), t["dr"].clone()
    h = gdn.block_norm_backward(*args, du, dr, gate_tokens=15, dx=dr, dy=du)
    torch.cuda.synchronize()
    assert torch.equal(x, r) and torch.equal(y, u)
    assert all(torch.equal(a, b) for a, b in zip(g, h))


def test_against_differences(gdn):
    """The gradient along a direction against central differences of the fp64 forward.
    A step of 1e-4 leaves 1e-8 of truncation and 1e-12 of rounding; the fp32 gradient
    is good to 1e-5 of the sum of its absolute terms."""
    import torch
    gt, rs = 3, 0.7
    t = make(2, 6, 50, gt, "f32", 12)
    got = gdn.block_norm_backward(t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"], t["du"], t["dr"], gate_tokens=gt,
                                  res_scale=rs)
    h = host(t)
    g = torch.Generator().manual_seed(1)
    names = ("x", "y", "gate", "w_post", "w_pre")

    def loss(p):
        _, _, _, r, ir, _, _ = parts(p, gt, rs, 1e-6)
        return float((r * ir * p["w_pre"] * p["du"]).sum() + (r * p["dr"]).sum())
    for name, gr in zip(names, got):
        step = torch.randn(h[name].shape, generator=g, dtype=torch.float64)
        up, down = dict(h), dict(h)
        up[name] = h[name] + 1e-4 * step
        down[name] = h[name] - 1e-4 * step
        terms = gr.double().cpu() * step
        diff = (loss(up) - loss(down)) / 2e-4
        assert abs(float(terms.sum()) - diff) <= 2e-5 * float(terms.abs().sum()), name


def test_captured_and_workspace(gdn):
    """Forward and gradient in one graph with a workspace of its own, replayed between eager
    calls on changing inputs: the eager call's bits."""
    import torch
    t = make(1, 300, 160, 300, "bf16", 14)
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    ws = gdn.block_norm_workspace(300, 160, 300, "cuda")
    ws.fill_(0xff)                                              # NaN in every word
    gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=300)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = gdn.block_norm(*args, gate_tokens=300)
        b = gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=300, ws=ws)
    for i in range(3):
        graph.replay()
        ef = gdn.block_norm(*args, gate_tokens=300)
        eb = gdn.block_norm_backward(*args, t["du"], t["dr"], gate_tokens=300)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(f + b, ef + eb)), i
        t["y"].mul_(1.25)
        t["du"].neg_()


def test_side_stream(gdn):
    import torch
    t = make(1, 64, 96, 8, "f32", 15)
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    ref = gdn.block_norm(*args, gate_tokens=8) + gdn.block_norm_backward(*args, t["du"], gate_tokens=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gdn.block_norm(*args, gate_tokens=8, stream=side) + \
        gdn.block_norm_backward(*args, t["du"], gate_tokens=8, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
