"""GPU: the short convolution, its gradient and its form for decoding batches against the formulas in fp64 and against
differences.

Tolerances, with u = 2^-24: z is a sum of at most 5 terms, off by 6 u of their absolute sum; activations as in
plain_acts; dz = dy slope adds u; dx is a sum of at most 5 terms again; sums over n tokens are off by (n + 64) u of the
sum of absolute terms.  Every result is rounded to its type, half a step.
"""
import pytest

from plain_acts import ACTS, U, act, act_error, close, half, slope, slope_error

pytestmark = pytest.mark.gpu


def make(B, T, C, W, dtype, seed, bias=True, state=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(s, generator=g)
    t = dict(x=rn(B, T, C).to(dt), w=rn(C, W), bias=rn(C) if bias else None, state=rn(B, W - 1, C).to(dt) if state else None,
             dy=rn(B, T, C).to(dt), dstate=rn(B, W - 1, C).to(dt) if state else None)
    return {n: None if v is None else v.cuda() for n, v in t.items()}


def parts(t):
    import torch
    x, w = t["x"].double(), t["w"].double()
    B, T, C = x.shape
    W = w.shape[1]
    s = torch.zeros(B, W - 1, C, device="cuda").double() if t["state"] is None else t["state"].double()
    xe = torch.cat([s, x], 1)
    b = torch.zeros(C, device="cuda").double() if t["bias"] is None else t["bias"].double()
    z = sum(w[:, i] * xe[:, i:i + T] for i in range(W)) + b
    ez = 6 * U * (sum((w[:, i] * xe[:, i:i + T]).abs() for i in range(W)) + b.abs())
    return xe, w, z, ez, T, W


def check_forward(t, y, state, name):
    import torch
    xe, w, z, ez, T, W = parts(t)
    ref = act(z, name)
    close("y", y, ref, act_error(z, ez, name) + 1.01 * half(y.dtype) * ref.abs())
    if state is not None:
        assert torch.equal(state.double(), xe[:, T:])


def check_gradient(t, got, name):
    import torch
    xe, w, z, ez, T, W = parts(t)
    dx, dw, dbias, dstate = got
    r = half(t["x"].dtype)
    dy, s = t["dy"].double(), slope(z, name)
    dz = dy * s
    edz = dy.abs() * slope_error(z, ez, name) + U * dz.abs()
    ref, tol, mag = (torch.zeros_like(xe) for _ in range(3))
    for i in range(W):
        ref[:, i:i + T] += w[:, i] * dz
        tol[:, i:i + T] += w[:, i].abs() * edz
        mag[:, i:i + T] += (w[:, i] * dz).abs()
    if t["dstate"] is not None:
        ref[:, T:] += t["dstate"].double()
        mag[:, T:] += t["dstate"].double().abs()
    tol = tol + 6 * U * mag + 1.01 * r * ref.abs()
    close("dx", dx, ref[:, W - 1:], tol[:, W - 1:])
    if dstate is not None:
        close("dstate", dstate, ref[:, :W - 1], tol[:, :W - 1])
    n = dz.shape[0] * T
    for i in range(W):
        p = dz * xe[:, i:i + T]
        close("dw", dw[:, i], p.sum((0, 1)), (edz * xe[:, i:i + T].abs()).sum((0, 1)) + (n + 64) * U * p.abs().sum((0, 1)))
    if t["bias"] is not None:
        close("dbias", dbias, dz.sum((0, 1)), edz.sum((0, 1)) + (n + 64) * U * dz.abs().sum((0, 1)))
    else:
        assert dbias is None


def both(gdn, t, name, **kw):
    y, state = gdn.short_conv(t["x"], t["w"], t["bias"], t["state"], activation=name)
    check_forward(t, y, state, name)
    check_gradient(t, gdn.short_conv_backward(t["x"], t["w"], t["bias"], t["state"], t["dy"], t["dstate"], activation=name), name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("B,T,C", [(1, 1, 1), (2, 1, 8), (1, 2, 7), (3, 3, 9), (1, 4, 16), (2, 5, 33), (1, 15, 64), (2, 16, 65), (1, 17, 512),
                                   (2, 63, 100), (1, 64, 8), (2, 65, 24), (1, 200, 520), (1, 1030, 12), (3, 700, 515)])
def test_sizes(gdn, dtype, W, B, T, C):
    both(gdn, make(B, T, C, W, dtype, B + T + C), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("bias,state", [(False, False), (True, False), (False, True)])
def test_activations_and_what_may_be_missing(gdn, dtype, name, bias, state):
    both(gdn, make(2, 37, 40, 4, dtype, 7, bias, state), name)


def test_many_rows(gdn):
    """More tokens than a thread's strip takes at once, and many short sequences."""
    both(gdn, make(1, 9000, 72, 4, "bf16", 1), "silu")
    both(gdn, make(70001, 2, 9, 3, "f32", 2), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,at", [(64, 64), (33, 1), (8, 3)])
def test_part_of_a_packed_projection(gdn, dtype, C, at):
    """x and dx with strides, at any element."""
    import torch
    t = make(2, 50, C, 4, dtype, 3)
    packed = torch.full((2, 50, 3 * C + 5), 9, dtype=t["x"].dtype, device="cuda")
    grads = packed.clone()
    view = packed[..., at:at + C]
    view.copy_(t["x"])
    y, state = gdn.short_conv(view, t["w"], t["bias"], t["state"])
    check_forward(t, y, state, "silu")
    got = gdn.short_conv_backward(view, t["w"], t["bias"], t["state"], t["dy"], t["dstate"], dx=grads[..., at:at + C])
    check_gradient(t, got, "silu")
    assert (grads[..., :at] == 9).all() and (grads[..., at + C:] == 9).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,C,at", [(3, 50, 64, 64), (2, 41, 33, 1), (5, 1, 9, 3), (4, 7, 2, 2), (1, 30, 24, 0)])
def test_part_of_a_projection_token_by_token(gdn, dtype, B, T, C, at):
    """x and dx as parts of [T, B, 3 C + 5] buffers, all sequences of a token before the next token."""
    import torch
    t = make(B, T, C, 4, dtype, 4)
    packed = torch.full((T, B, 3 * C + 5), 9, dtype=t["x"].dtype, device="cuda")
    grads = packed.clone()
    view, dx = (a.transpose(0, 1)[..., at:at + C] for a in (packed, grads))
    view.copy_(t["x"])
    y, state = gdn.short_conv(view, t["w"], t["bias"], t["state"])
    check_forward(t, y, state, "silu")
    got = gdn.short_conv_backward(view, t["w"], t["bias"], t["state"], t["dy"], t["dstate"], dx=dx)
    assert got[0].data_ptr() == dx.data_ptr()
    check_gradient(t, got, "silu")
    assert (grads[..., :at] == 9).all() and (grads[..., at + C:] == 9).all()


def test_sequences_of_one_input(gdn):
    """The same tokens for every sequence (stride 0), and tokens in reverse order of memory refused."""
    import torch
    t = make(1, 20, 24, 4, "f32", 3, state=False)
    y, _ = gdn.short_conv(t["x"].expand(3, -1, -1), t["w"], t["bias"])
    one, _ = gdn.short_conv(t["x"], t["w"], t["bias"])
    assert torch.equal(y, one.expand(3, -1, -1))
    with pytest.raises(ValueError, match="channels"):
        gdn.short_conv(t["x"].transpose(1, 2), t["w"][:20], t["bias"][:20])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [9, 64])
def test_calls_that_follow_each_other(gdn, dtype, C):
    """A stream cut anywhere, its state updated in place, is the whole call bit for bit."""
    import torch
    t = make(2, 41, C, 4, dtype, 5)
    y, state = gdn.short_conv(t["x"], t["w"], t["bias"], t["state"])
    s, at, parts_ = t["state"].clone(), 0, []
    for n in (1, 2, 17, 1, 1, 16, 3):
        p, s2 = gdn.short_conv(t["x"][:, at:at + n], t["w"], t["bias"], s, state_out=s)
        assert s2 is s
        parts_.append(p)
        at += n
    assert at == 41 and torch.equal(torch.cat(parts_, 1), y) and torch.equal(s, state)


def test_gradient_against_differences(gdn):
    import torch
    t = make(2, 30, 12, 4, "f32", 6)
    got = [d.double() for d in gdn.short_conv_backward(t["x"], t["w"], t["bias"], t["state"], t["dy"], t["dstate"])]
    names = ("x", "w", "bias", "state")

    def loss(v):
        xe, w, z, _, T, W = parts(dict(t, **v))
        return (act(z, "silu") * t["dy"].double()).sum() + (xe[:, T:] * t["dstate"].double()).sum()
    g = torch.Generator(device="cuda").manual_seed(1)
    for n, d in zip(names, got):
        v = torch.randn(d.shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        diff = (loss({n: t[n].double() + e * v}) - loss({n: t[n].double() - e * v})) / (2 * e)
        # the difference is off by e^2 times third derivatives of size 1, the kernel by some 100 u
        assert abs(float((d * v).sum() - diff)) <= 1e-6 * float((d * v).abs().sum()), n


def test_not_finite_values_reach_their_window_alone(gdn):
    import torch
    t = make(1, 40, 16, 4, "f32", 2)
    t["x"][0, 10, 3] = float("nan")
    t["x"][0, 39, 5] = float("inf")
    y, state = gdn.short_conv(t["x"], t["w"], t["bias"], t["state"], activation=None)
    bad = ~y.isfinite()
    assert bad[0, 10:14, 3].all() and bad[0, 39, 5] and int(bad.sum()) == 5
    assert state[0, 2, 5] == float("inf")


# ---------------------------------------------------------------------------
# Decoding batches.

def step_case(N, L, P, C, W, dtype, seed, bias=True):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    t = dict(x=torch.randn(N, L, C, generator=g).to(dt), w=torch.randn(C, W, generator=g),
             bias=torch.randn(C, generator=g) if bias else None, pool=torch.randn(P, W - 1, C, generator=g).to(dt),
             slots=torch.randperm(P, generator=g)[:N].int(), lengths=torch.randint(0, L + 1, (N,), generator=g).int())
    return {n: None if v is None else v.cuda() for n, v in t.items()}


def check_step(t, out, pool, slots, lengths, name="silu"):
    import torch
    for n in range(t["x"].shape[0]):
        m, s = int(lengths[n]), int(slots[n])
        if s < 0:
            continue
        row = dict(x=t["x"][n:n + 1, :m], w=t["w"], bias=t["bias"], state=t["pool"][s:s + 1])
        if m:
            check_forward(row, out[n:n + 1, :m], pool[s:s + 1], name)
        else:
            assert torch.equal(pool[s], t["pool"][s])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,L,P,C,W", [(1, 1, 1, 1, 2), (1, 1, 3, 8, 4), (3, 2, 5, 7, 3), (4, 5, 4, 100, 4), (5, 3, 9, 512, 2), (2, 8, 2, 513, 4),
                                       (7, 1, 8, 2049, 3)])
def test_step(gdn, dtype, N, L, P, C, W):
    import torch
    t = step_case(N, L, P, C, W, dtype, N + C)
    out = torch.full_like(t["x"], 5)
    new = torch.full_like(t["pool"], 6)
    gdn.short_conv_step(t["x"], t["w"], t["bias"], t["pool"], slots=t["slots"], lengths=t["lengths"], out=out, state_out=new)
    check_step(t, out, new, t["slots"], t["lengths"])
    for n in range(N):
        assert (out[n, int(t["lengths"][n]):] == 5).all()
    rest = [p for p in range(P) if p not in t["slots"].tolist()]
    assert (new[rest] == 6).all()
    # in place, every row its own slot, all tokens there
    pool = t["pool"].clone()
    out, same = gdn.short_conv_step(t["x"], t["w"], None, pool, activation="gelu")
    assert same is pool
    check_step(dict(t, bias=None), out, pool, range(N), [L] * N, "gelu")


def test_step_padding_and_refused_slots(gdn):
    import torch
    t = step_case(70, 2, 80, 24, 4, "bf16", 1)
    slots = t["slots"].clone()
    slots[3], slots[9] = -1, -7                    # padding
    slots[5], slots[69] = slots[2], slots[0]       # named before
    slots[7] = 80                                  # past the pool
    pool = t["pool"].clone()
    out = torch.full_like(t["x"], 5)
    gdn.short_conv_step(t["x"], t["w"], t["bias"], pool, slots=slots, out=out)
    for n in (3, 9):
        assert (out[n] == 5).all()
    for n in (5, 69, 7):
        assert out[n].isnan().all()
    rows = [n for n in range(70) if n not in (3, 9, 5, 69, 7)]
    check_step({k: v[rows] if k == "x" else v for k, v in t.items()}, out[rows], pool, slots[rows], [2] * len(rows))
    free = [p for p in range(80) if p not in slots[rows].tolist()]
    assert torch.equal(pool[free], t["pool"][free])
    out, _ = gdn.short_conv_step(t["x"], t["w"], t["bias"], t["pool"].clone(), slots=slots)
    assert (out[3] == 0).all()


def test_step_follows_a_prompt(gdn):
    """A prompt's state in a pool, then tokens one and two at a time: bit for bit the whole call."""
    import torch
    t = make(3, 30, 40, 4, "bf16", 4, state=False)
    y, state = gdn.short_conv(t["x"], t["w"], t["bias"])
    first, s = gdn.short_conv(t["x"][:, :21], t["w"], t["bias"])
    pool = torch.zeros(5, 3, 40, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([4, 0, 2], dtype=torch.int32, device="cuda")
    pool[slots.long()] = s
    parts_, at = [first], 21
    for n in (1, 1, 2, 1, 4):
        parts_.append(gdn.short_conv_step(t["x"][:, at:at + n], t["w"], t["bias"], pool, slots=slots)[0])
        at += n
    assert torch.equal(torch.cat(parts_, 1), y) and torch.equal(pool[slots.long()], state)


def test_captured_and_on_another_stream(gdn):
    import torch
    t = make(2, 300, 72, 4, "bf16", 9)
    p = step_case(6, 2, 9, 72, 4, "bf16", 2)
    args = (t["x"], t["w"], t["bias"], t["state"])

    def calls(pool, **kw):
        y = gdn.short_conv(*args, **kw)
        d = gdn.short_conv_backward(*args, t["dy"], t["dstate"], **kw)
        s = gdn.short_conv_step(p["x"], p["w"], p["bias"], p["pool"], slots=p["slots"], state_out=pool, **kw)
        return [*y, *d, *s]
    want = calls(p["pool"].clone())
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    pools = [p["pool"].clone() for _ in range(2)]
    torch.cuda.synchronize()
    got = calls(pools[0], stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(pools[1])
    for i in range(4):
        for o in out[:-1]:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i
        t["x"].mul_(-0.5)
        want = calls(p["pool"].clone())
        torch.cuda.synchronize()


def test_outputs_alone_are_written(gdn):
    import torch
    t = make(2, 77, 33, 4, "bf16", 5)

    def guarded(like, dt=None):
        n = like.numel()
        buf = torch.full((n + 1024,), 7, dtype=like.dtype, device="cuda")
        return buf, buf[512:512 + n].view(like.shape)
    b = {n: guarded(v) for n, v in dict(y=t["x"], so=t["state"], dx=t["x"], dw=t["w"], db=t["bias"], ds=t["state"]).items()}
    ws = gdn.short_conv_workspace(t["x"], t["w"])
    b["ws"] = guarded(ws)
    gdn.short_conv(t["x"], t["w"], t["bias"], t["state"], out=b["y"][1], state_out=b["so"][1])
    got = gdn.short_conv_backward(t["x"], t["w"], t["bias"], t["state"], t["dy"], t["dstate"], dx=b["dx"][1], dw=b["dw"][1],
                                  dbias=b["db"][1], dstate=b["ds"][1], ws=b["ws"][1])
    check_forward(t, b["y"][1], b["so"][1], "silu")
    check_gradient(t, got, "silu")
    for n, (buf, _) in b.items():
        assert (buf[:512] == 7).all() and (buf[-512:] == 7).all(), n
