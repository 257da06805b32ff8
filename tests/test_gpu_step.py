"""GPU: the recurrent step of a decoding batch against the recurrence in fp64.

Tolerance: S^T k and S^T q are sums of Dk fp32 products, off by at most (Dk + 2) half
steps of sum |s| |k| <= |column of S| |k|; with |k| <= 1.01 (unit keys, rounded), alpha
and beta in [0, 1] and fewer than 14 further roundings a token, a token adds at
most (Dk + 16) 2^-24 M to the error of a state or output element, where M is the
largest column norm of any state plus the largest |v|; an error already in
the state grows by no more than 1 + beta |k|^2 < 2.1 in the column norm, and
with L <= 5 tokens the sum of those is below 2^5 times one.  A bf16 output adds half
a step, 2^-8 of its value.
"""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def make(N, L, P, Hk, H, Dk, Dv, dtype, seed, dev="cuda"):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def unit(*s):
        x = torch.randn(s, generator=g)
        return (x / x.norm(dim=-1, keepdim=True)).to(dt)
    t = dict(q=unit(N, L, Hk, Dk), k=unit(N, L, Hk, Dk), v=torch.randn(N, L, H, Dv, generator=g).to(dt),
             alpha=torch.rand(N, L, H, generator=g), beta=torch.rand(N, L, H, generator=g),
             state=torch.randn(P, H, Dk, Dv, generator=g))
    slots = torch.randperm(P, generator=g)[:N].to(torch.int32)
    return {n: x.to(dev) for n, x in t.items()}, slots.to(dev)


def reference(t, slots, lengths, out, state):
    """out and state (fp64, host) after the call, and the scale M of the errors."""
    q, k, v, a, b = (t[n].double().cpu() for n in ("q", "k", "v", "alpha", "beta"))
    N, L, Hk, _ = q.shape
    H, P = v.shape[2], state.shape[0]
    M = float(state.norm(dim=2).max() + v.abs().max())
    seen = set()
    for n in range(N):
        s = int(slots[n])
        m = max(0, min(int(lengths[n]), L))
        if s < 0:
            continue
        if s >= P or s in seen:
            out[n, :m] = float("nan")
            continue
        seen.add(s)
        for h in range(H):
            g = h // (H // Hk)
            S = state[s, h].clone()
            for i in range(m):
                S = a[n, i, h] * S
                S = S + b[n, i, h] * k[n, i, g][:, None] * (v[n, i, h] - S.T @ k[n, i, g])
                out[n, i, h] = S.T @ q[n, i, g]
                M = max(M, float(S.norm(dim=0).max() + v.abs().max()))
            state[s, h] = S
    return out, state, M


def check(t, slots, lengths, out, state, before_out, before_state):
    import torch
    N, L = t["q"].shape[:2]
    Dk = t["q"].shape[3]
    sl = slots if slots is not None else torch.arange(N)
    ln = lengths if lengths is not None else torch.full((N,), L)
    ro, rs, M = reference(t, sl.tolist(), ln.tolist(), before_out.double().cpu(), before_state.double().cpu())
    tol = (Dk + 16) * U * M * (1 if L == 1 else 2 ** 5)
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else U
    o, s = out.double().cpu(), state.double().cpu()
    assert torch.equal(torch.isnan(o), torch.isnan(ro))
    fine = ~torch.isnan(ro)
    assert ((o - ro).abs()[fine] <= tol + half * ro.abs()[fine]).all(), float((o - ro).abs()[fine].max())
    assert ((s - rs).abs() <= tol).all(), float((s - rs).abs().max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("N,L,Hk,H", [(1, 1, 1, 1), (3, 1, 2, 6), (5, 4, 3, 3), (7, 2, 1, 5)])
def test_step(gdn, dtype, Dk, Dv, N, L, Hk, H):
    """In place on a pool with slots to spare; the other slots keep their bits."""
    import torch
    t, slots = make(N, L, N + 3, Hk, H, Dk, Dv, dtype, 10 * N + L + Dk + Dv)
    before = t["state"].clone()
    out, st = gdn.step(**t, slots=slots)
    torch.cuda.synchronize()
    assert st is t["state"]
    check(t, slots, None, out, st, torch.zeros_like(out), before)
    rest = torch.ones(N + 3, dtype=torch.bool)
    rest[slots.long().cpu()] = False
    assert torch.equal(st[rest.cuda()], before[rest.cuda()])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lengths_padding_and_refused_rows(gdn, dtype):
    """Lengths of 0, 1 and past L, a padding row, a slot beyond the pool and a slot named
    twice: what is not written keeps its bits, refused rows are NaN."""
    import torch
    N, L, P = 7, 3, 5
    t, _ = make(N, L, P, 2, 4, 64, 128, dtype, 77)
    slots = torch.tensor([4, -1, 0, 5, 4, 2, 1], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([1, 3, 0, 2, 3, 9, -2], dtype=torch.int32, device="cuda")
    out = torch.full((N, L, 4, 128), 7.0, dtype=t["q"].dtype, device="cuda")
    new = torch.full_like(t["state"], 5.0)
    old, before = t["state"].clone(), out.clone()
    gdn.step(**t, slots=slots, lengths=lengths, out=out, state_out=new)
    torch.cuda.synchronize()
    assert torch.equal(t["state"], old)
    assert torch.equal(new[3], torch.full_like(new[3], 5.0))            # no row names slot 3
    assert torch.equal(new[0], old[0]) and torch.equal(new[1], old[1])  # lengths 0 and below
    ref_state = old.clone()
    ref_state[3] = 5.0
    check(t, slots, lengths, out, new, before, ref_state)
    for n, m in enumerate([1, 0, 0, 2, 3, 3, 0]):
        assert torch.equal(out[n, m:], before[n, m:])
    assert torch.isnan(out[3, :2]).all() and torch.isnan(out[4]).all()


def test_same_slot_in_a_wide_batch(gdn):
    """Rows past 64 find an earlier owner in any part of the list."""
    import torch
    N = 200
    t, slots = make(N, 1, N, 1, 1, 64, 64, "f32", 3)
    for late, early in ((199, 0), (130, 64), (65, 1)):
        slots[late] = slots[early]
    before = t["state"].clone()
    out, st = gdn.step(**t, slots=slots)
    torch.cuda.synchronize()
    check(t, slots, None, out, st, torch.zeros_like(out), before)
    assert torch.isnan(out).flatten(1).any(1).nonzero().flatten().tolist() == [65, 130, 199]


def test_gates_at_their_ends(gdn):
    """alpha and beta of exactly 0 and 1."""
    import torch
    t, slots = make(4, 5, 4, 2, 2, 128, 128, "bf16", 5)
    t["alpha"] = t["alpha"].round()
    t["beta"] = t["beta"].round()
    before = t["state"].clone()
    out, st = gdn.step(**t, slots=slots)
    torch.cuda.synchronize()
    check(t, slots, None, out, st, torch.zeros_like(out), before)


def test_continues_the_chunk_forward(gdn):
    """Prefill with forward, then tokens one by one and several at a time: the same
    outputs as the forward over the whole sequence."""
    import torch
    g = torch.Generator().manual_seed(9)
    B, T, H, D, n = 2, 150, 3, 64, 6
    q, k = (torch.nn.functional.normalize(torch.randn(B, T, H, D, generator=g), dim=-1).cuda() for _ in range(2))
    v = torch.randn(B, T, H, D, generator=g).cuda()
    a, b = torch.rand(B, T, H, generator=g).cuda(), torch.rand(B, T, H, generator=g).cuda()
    ref, ref_state = gdn.forward(q, k, v, a, b)

    def cut(lo, hi):
        return [x[:, lo:hi].contiguous() for x in (q, k, v, a, b)]
    out, state = gdn.forward(*cut(0, T - n))
    outs = [out]
    for lo, hi in ((T - n, T - n + 1), (T - n + 1, T - n + 2), (T - n + 2, T)):
        o, state = gdn.step(*cut(lo, hi), state)
        outs.append(o)
    # two fp32 evaluations of one recurrence: each is within 1e-4 of it (the bound
    # that the forward is held to)
    assert (torch.cat(outs, 1) - ref).abs().max() <= 2e-4 * ref.abs().max()
    assert (state - ref_state).abs().max() <= 2e-4 * ref_state.abs().max()


def test_captured(gdn):
    """A captured step, replayed with eager work between: each replay advances the pool
    as an eager call does, bit for bit."""
    import torch
    t, slots = make(6, 1, 8, 2, 4, 128, 128, "bf16", 21)
    lengths = torch.ones(6, dtype=torch.int32, device="cuda")
    eager = {n: x.clone() for n, x in t.items()}
    out = torch.zeros(6, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    ref = torch.zeros_like(out)                         # rows of length 0 keep their last output in both
    gdn.step(**{n: x.clone() for n, x in t.items()}, slots=slots, lengths=lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gdn.step(**t, slots=slots, lengths=lengths, out=out)
    for i in range(4):
        graph.replay()
        gdn.step(**eager, slots=slots, lengths=lengths, out=ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i
        assert torch.equal(t["state"], eager["state"]), i
        lengths[i] = 0                                  # the next replay leaves this row


def test_side_stream(gdn):
    import torch
    t, slots = make(9, 2, 9, 1, 2, 64, 64, "f32", 31)
    ref, rs = gdn.step(**{n: x.clone() for n, x in t.items()}, slots=slots)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, st = gdn.step(**t, slots=slots, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, ref) and torch.equal(st, rs)


def test_fresh_output_is_zero_where_nothing_is_written(gdn):
    """Without out=, tokens past a row's length and padding rows come back as zeros."""
    import torch
    t, slots = make(3, 2, 4, 1, 1, 64, 64, "bf16", 6)
    slots[2] = -1
    torch.full((3, 2, 1, 64), float("nan"), dtype=torch.bfloat16, device="cuda")   # freed memory that is not zero
    out, _ = gdn.step(**t, slots=slots, lengths=torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
    assert not out[0].any() and not out[1, 1].any() and not out[2].any() and out[1, 0].all()


@pytest.mark.parametrize("name", ["q", "k", "v", "alpha", "beta", "state", "slots", "lengths", "out", "state_out"])
def test_arguments(gdn, name):
    """Each argument with a wrong size, a wrong type, on the host, or with gaps is refused by its name;
    a parameter of a module passes, with the bits of its tensor."""
    import torch
    t, slots = make(3, 2, 4, 2, 4, 64, 128, "bf16", 41)
    a = dict(t, slots=slots, lengths=torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"),
             out=torch.zeros_like(t["v"]), state_out=t["state"].clone())
    ref, after = (x.clone() for x in gdn.step(**a))
    x = a[name]
    wrong = [x.new_zeros([n + 1 for n in x.shape]), x.cpu(), x.new_zeros([2 * n for n in x.shape])[tuple(slice(None, None, 2) for _ in x.shape)]]
    for bad in wrong:
        with pytest.raises(ValueError):
            gdn.step(**dict(a, **{name: bad}))
    for bad in (x.double(), None if name in ("q", "k", "v", "alpha", "beta", "state") else 3):
        with pytest.raises((TypeError, ValueError)):
            gdn.step(**dict(a, **{name: bad}))
    if x.is_floating_point():
        a.update(out=torch.zeros_like(ref), state_out=t["state"].clone())
        a[name] = torch.nn.Parameter(a[name], requires_grad=False)
        out, state = gdn.step(**a)
        assert torch.equal(out, ref) and torch.equal(state, after)
