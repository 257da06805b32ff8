"""GPU: the norm of many tensors and their clipping.

Tolerances, with u = 2^-24: squares are exact in fp64 and n of them sum to within n 2^-53, so the norm is off by its
rounding to fp32, u; the factor by 2 u more, a product by u, and a result by half a step of its type.
"""
import math

import pytest

from plain_acts import U, half

pytestmark = pytest.mark.gpu


def make(sizes, seed, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(torch.bfloat16 if i % 2 else torch.float32).cuda() for i, n in enumerate(sizes)]


def exact(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check(ts, norm, out, max_norm, eps=1e-6):
    want = exact(ts)
    assert abs(float(norm) - want) <= 1.01 * U * want
    s = min(1.0, max_norm / (want + eps)) if max_norm < math.inf else 1.0
    for t, o in zip(ts, out):
        ref = t.double() * s
        assert o.dtype == t.dtype and o.shape == t.shape
        assert ((o.double() - ref).abs() <= (5 * U + half(t.dtype)) * ref.abs()).all()


LISTS = [[1], [0], [7, 0, 3], [16384], [16385, 16383, 1], [8, 9, 4097, 100000], [333] * 300, [0] * 200 + [5], [70000, 1] * 70, [40000000, 3]]


@pytest.mark.parametrize("max_norm", [1.0, 1e9])
@pytest.mark.parametrize("sizes", LISTS)
def test_lists(gdn, sizes, max_norm):
    import torch
    ts = make(sizes, len(sizes))
    norm = gdn.grad_norm(ts)
    assert norm.shape == () and norm.dtype == torch.float32
    out = [torch.empty_like(t) for t in ts]
    n2, got = gdn.clip_grads(ts, max_norm, out=out)
    assert float(n2) == float(norm) and all(a is b for a, b in zip(got, out))
    check(ts, norm, out, max_norm)
    here = [t.clone() for t in ts]
    n3, got = gdn.clip_grads(here, max_norm)
    assert float(n3) == float(norm) and all(a is b for a, b in zip(got, here))
    assert all(torch.equal(a, b) for a, b in zip(here, out))
    if max_norm > 1e8:
        assert all(torch.equal(a, b) for a, b in zip(here, ts))


def test_many_launches(gdn):
    """More sums than a workgroup adds up for itself: large tensors over six launches, small ones over forty."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(4)
    for n, size in ((700, 262145), (5000, 3)):
        ts = [torch.randn(size, generator=g, device="cuda", dtype=torch.bfloat16 if i % 2 else torch.float32) for i in range(n)]
        want = math.sqrt(float(torch.stack([t.double().square().sum() for t in ts]).sum()))
        norm, out = gdn.clip_grads(ts, 1.0, out=[torch.empty_like(t) for t in ts])
        assert abs(float(norm) - want) <= 1.01 * U * want and float(gdn.grad_norm(ts)) == float(norm)
        for t, o in list(zip(ts, out))[:: n // 50]:
            ref = t.double() / (want + 1e-6)
            assert ((o.double() - ref).abs() <= (5 * U + half(t.dtype)) * ref.abs()).all()


@pytest.mark.parametrize("n", [8192, 8193, 9000])
def test_sums_of_many_small_tensors(gdn, n):
    """Tensors of three elements, a sum each: 8192 sums are the most that every workgroup of the scaling adds up for itself, more are read from
    the workspace as one norm; over 64 launches and more, in place too and from replays of a graph."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(n)
    flat = [torch.randn(3 * n, generator=g, device="cuda").to(dt) for dt in (torch.bfloat16, torch.float32)]

    def parts(pair):
        return [pair[i % 2][3 * i:3 * i + 3] for i in range(n)]
    used = [torch.arange(3 * n, device="cuda") // 3 % 2 == k for k in (0, 1)]

    def check(norm, out):
        want = math.sqrt(sum(float(f[u].double().square().sum()) for f, u in zip(flat, used)))
        assert abs(float(norm) - want) <= 1.01 * U * want
        for f, u, o in zip(flat, used, out):
            ref = f[u].double() * min(1.0, 1.0 / (want + 1e-6))
            assert ((o[u].double() - ref).abs() <= (5 * U + half(f.dtype)) * ref.abs()).all()
            assert (o[~u] == 9).all()
    outs = [[torch.full_like(f, 9) for f in flat] for _ in range(2)]
    norm, _ = gdn.clip_grads(parts(flat), 1.0, out=parts(outs[0]))
    check(norm, outs[0])
    assert torch.equal(gdn.grad_norm(parts(flat)), norm)
    here = [torch.where(u, f, 9) for f, u in zip(flat, used)]
    n2, _ = gdn.clip_grads(parts(here), 1.0)
    assert torch.equal(n2, norm) and all(torch.equal(a, b) for a, b in zip(here, outs[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n3, _ = gdn.clip_grads(parts(flat), 1.0, out=parts(outs[1]))
    for i in range(3):
        n3.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check(n3, outs[1])
        for f in flat:
            f.mul_(-0.75)
        gdn.clip_grads(parts(here), 1.0)
        torch.cuda.synchronize()


def test_any_element_and_order(gdn):
    """Tensors that start at any element of a flat buffer, and permuted ones."""
    import torch
    flat = [make([5000], i)[0].to(dt) for i, dt in enumerate((torch.bfloat16, torch.float32))]
    keep = [f.clone() for f in flat]
    ts = [f[a:b] for f in flat for a, b in ((1, 2), (3, 700), (701, 4801))] + [make([600], 3)[0].view(20, 30).T]
    was = [t.clone() for t in ts]
    norm, out = gdn.clip_grads(ts, 2.0)
    check(was, norm, ts, 2.0)
    for f, k in zip(flat, keep):
        for a, b in ((0, 1), (2, 3), (700, 701), (4801, 5000)):
            assert torch.equal(f[a:b], k[a:b])


def test_norm_given(gdn):
    import torch
    ts = make([1000, 77], 1)
    was = [t.clone() for t in ts]
    n = torch.tensor(40.0, device="cuda")
    got, _ = gdn.clip_grads(ts, 10.0, norm=n, eps=0.0)
    assert got is n and float(n) == 40.0
    assert all(torch.equal(a, b * 0.25) for a, b in zip(ts, was))


def test_far_values(gdn):
    """Squares that fp32 does not hold, norms of zero, and of values that are not finite."""
    import torch
    big = torch.full((1000,), 1e30, device="cuda")
    tiny = torch.full((1000,), 1e-30, device="cuda")
    assert abs(float(gdn.grad_norm([big])) / (1e30 * math.sqrt(1000)) - 1) < 3 * U
    assert abs(float(gdn.grad_norm([tiny])) / (1e-30 * math.sqrt(1000)) - 1) < 3 * U
    n, _ = gdn.clip_grads([big], 1.0)
    assert float((big * math.sqrt(1000) - 1).abs().max()) < 1e-6
    zero = torch.zeros(50, device="cuda")
    n, _ = gdn.clip_grads([zero], 0.0)
    assert float(n) == 0 and (zero == 0).all()
    a, b = torch.ones(20, device="cuda"), torch.ones(20, device="cuda", dtype=torch.bfloat16)
    b[7] = float("inf")
    n, _ = gdn.clip_grads([a, b], 1.0)
    assert float(n) == math.inf and (a == 0).all() and b[7].isnan() and (b[:7] == 0).all()
    a = torch.ones(20, device="cuda")
    a[3] = float("nan")
    c = torch.ones(20, device="cuda")
    n, _ = gdn.clip_grads([a, c], 1.0)
    assert n.isnan() and c.isnan().all()
    c = torch.ones(20, device="cuda")
    gdn.clip_grads([c], math.inf)
    assert (c == 1).all()
    gdn.clip_grads([b], math.inf)                           # no bound, and a norm that is infinite
    c[3] = math.inf
    gdn.clip_grads([c], math.inf)
    assert (c[:3] == 1).all() and c[3] == math.inf and (c[4:] == 1).all()
    gdn.clip_grads([zero], 0.0, eps=0.0)                    # 0 / 0
    assert (zero == 0).all()
    c[3] = math.nan
    gdn.clip_grads([c], math.inf)
    assert c.isnan().all()


def test_same_bits_every_time_and_in_graphs(gdn):
    import torch
    ts = make([100001, 5, 33333, 16384] * 40, 2)
    ws = gdn.grad_workspace(ts)
    norm, out = gdn.clip_grads(ts, 1.0, out=[torch.empty_like(t) for t in ts], ws=ws)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    n2, o2 = gdn.clip_grads(ts, 1.0, out=[torch.empty_like(t) for t in ts], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(norm, n2) and all(torch.equal(a, b) for a, b in zip(out, o2))
    o3 = [torch.zeros_like(t) for t in ts]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n3, _ = gdn.clip_grads(ts, 1.0, out=o3)
    for i in range(4):
        for o in o3:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, n3) and all(torch.equal(a, b) for a, b in zip(out, o3)), i
        for t in ts[:3]:
            t.mul_(-1.5)
        norm, out = gdn.clip_grads(ts, 1.0, out=[torch.empty_like(t) for t in ts])
        torch.cuda.synchronize()


def test_refusals(gdn):
    import torch
    a, b = make([100, 100], 1)
    with pytest.raises(ValueError, match="no tensor"):
        gdn.grad_norm([])
    with pytest.raises(TypeError, match="sequence"):
        gdn.grad_norm(a)
    with pytest.raises(TypeError, match="bfloat16"):
        gdn.grad_norm([a.half()])
    with pytest.raises(ValueError, match="GPU"):
        gdn.grad_norm([a, a.cpu()])
    with pytest.raises(ValueError, match="run of memory"):
        gdn.grad_norm([a[::2]])
    with pytest.raises(ValueError, match="negative"):
        gdn.clip_grads([a], -1.0)
    with pytest.raises(ValueError, match="negative"):
        gdn.clip_grads([a], float("nan"))
    with pytest.raises(ValueError, match="like"):
        gdn.clip_grads([a], 1.0, out=[b])
    with pytest.raises(gdn.GdnError):                       # twice in place: its factor would count twice
        gdn.clip_grads([a, b, a], 1.0)
    with pytest.raises(gdn.GdnError):
        gdn.clip_grads([a[:60], a[50:]], 1.0)
    with pytest.raises(gdn.GdnError):
        gdn.clip_grads([a[:50]], 1.0, out=[a[20:70]])
    keep = a.clone()
    assert abs(float(gdn.grad_norm([a, a])) - math.sqrt(2) * exact([a])) <= 2 * U * exact([a])
    torch.cuda.synchronize()
    assert torch.equal(a, keep)
    v = a._version
    gdn.clip_grads([a], 1.0)
    assert a._version > v
    with pytest.raises(ValueError, match="gradient"):
        gdn.clip_grads([a.requires_grad_()], 1.0)
