"""GPU: the gated linear map and its gradient against the formulas in fp64 and against differences.

Tolerances, with u = 2^-24: a sum of n products in fp32 is off by at most 2 (n + 16) u of the sum of absolute products
(the matrix cores may cut instead of rounding: two half steps an addition); activations as in plain_acts.  The
gradient's operands dg and du are rounded to the type (half a step of each), and so is every result.
"""
import pytest

from plain_acts import ACTS, U, act, act_error, close, half, slope, slope_error

pytestmark = pytest.mark.gpu


def make(M, C, F, dtype, seed, scale=1.0):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(s, generator=g)
    return [t.to(dt).cuda() for t in (scale * rn(M, C), rn(F, C) / C ** 0.5, rn(F, C) / C ** 0.5, rn(M, F))]


def sums(a, b, n):
    """Error of a @ b over n products, beside that of its operands."""
    return 2 * (n + 16) * U * (a.abs() @ b.abs())


def parts(x, wg, wu):
    x, wg, wu = x.double(), wg.double(), wu.double()
    C = x.shape[1]
    return x, wg, wu, x @ wg.T, x @ wu.T, sums(x, wg.T, C), sums(x, wu.T, C)


def check_forward(t, h, name):
    x, wg, wu, g, u, eg, eu = parts(*t[:3])
    a, ea = act(g, name), act_error(g, eg, name)
    ref = a * u
    close("h", h, ref, ea * (u.abs() + eu) + a.abs() * eu + (U + half(h.dtype)) * 1.01 * ref.abs())


def check_gradient(t, got, name):
    x, wg, wu, g, u, eg, eu = parts(*t[:3])
    dh, r = t[3].double(), half(t[0].dtype)
    M, F = dh.shape
    a, s = act(g, name), slope(g, name)
    ea, es = act_error(g, eg, name), slope_error(g, eg, name)
    dg, du = dh * u * s, dh * a
    edg = dh.abs() * ((u.abs() + eu) * es + s.abs() * eu) + (r + 3 * U) * 1.02 * dg.abs()
    edu = dh.abs() * ea + (r + 2 * U) * 1.02 * du.abs()
    dx = dg @ wg + du @ wu
    close("dx", got[0], dx, edg @ wg.abs() + edu @ wu.abs() + sums(dg, wg, 2 * F) + sums(du, wu, 2 * F) + 1.02 * r * dx.abs())
    for n, d, ed, w in (("dw_gate", dg, edg, got[1]), ("dw_up", du, edu, got[2])):
        ref = d.T @ x
        close(n, w, ref, ed.T @ x.abs() + sums(d.T, x, M) + 1.02 * r * ref.abs())


# rows up to 64 stream the weights; C and F around the tiles' and stages' ends
SMALL = [(1, 64, 16), (1, 1, 1), (1, 2048, 100), (2, 7, 33), (15, 130, 31), (16, 64, 17), (17, 200, 64), (32, 513, 40), (33, 96, 48),
         (48, 1000, 16), (63, 9, 5), (64, 640, 130)]
TILES = [(65, 64, 64), (65, 1, 1), (66, 7, 3), (127, 63, 65), (128, 128, 64), (129, 65, 63), (200, 96, 200), (256, 40, 264), (257, 72, 129),
         (300, 513, 130), (511, 200, 72), (640, 136, 514)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", SMALL + TILES)
def test_forward(gdn, dtype, M, C, F):
    t = make(M, C, F, dtype, M + C + F)
    check_forward(t, gdn.gated_linear(*t[:3]), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", [(1, 1, 1), (1, 64, 64), (3, 130, 7), (64, 65, 33)] + TILES)
def test_gradient(gdn, dtype, M, C, F):
    t = make(M, C, F, dtype, M + 2 * C + F)
    check_gradient(t, gdn.gated_linear_backward(*t), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("M", [5, 100])
def test_activations(gdn, dtype, name, M):
    t = make(M, 72, 136, dtype, M, scale=4.0)
    check_forward(t, gdn.gated_linear(*t[:3], activation=name), name)
    check_gradient(t, gdn.gated_linear_backward(*t, activation=name), name)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", [(3520, 256, 1800), (3333, 264, 1803), (257, 4104, 6200), (6200, 4101, 257)])
def test_large_tiles(gdn, dtype, M, C, F):
    """Enough tiles for the large ones in at least one of the products, whole and with ragged ends."""
    t = make(M, C, F, dtype, M + C)
    check_forward(t, gdn.gated_linear(*t[:3]), "silu")
    check_gradient(t, gdn.gated_linear_backward(*t), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", [(100, 4096, 64), (40, 4096, 128), (64, 4104, 100), (20, 3000, 70), (9000, 72, 130), (70, 2056, 40), (20000, 16, 8)])
def test_contractions_that_are_cut(gdn, dtype, M, C, F):
    """Few tiles and long sums: each contraction in parts that are joined, whole ones and with a tail."""
    t = make(M, C, F, dtype, M + C)
    check_forward(t, gdn.gated_linear(*t[:3]), "silu")
    check_gradient(t, gdn.gated_linear_backward(*t), "silu")


# Sizes that take each variant of the tiles, whole contractions and parts, for more stages than it has buffers (which
# sizes those are, a test on the host looks after).
VARIANTS = [(452, 475, 10), (1, 4104, 8), (1426, 248, 121), (1, 8, 193), (1, 8, 1892), (1, 8, 3785), (4075, 8, 8), (65, 8590, 11), (7634, 8, 8),
            (3223, 168, 383), (386, 800, 774), (5587, 336, 135), (2058, 272, 1067), (261, 641, 1807), (177, 152, 8215), (514, 285, 3278),
            (2006, 1040, 579), (964, 136, 4207), (1801, 2490, 143), (1840, 668, 1148), (454, 201, 8504), (5377, 8, 556), (274, 3788, 1955),
            (657, 5584, 66), (1033, 3745, 136), (4978, 2336, 398), (64, 768, 4159), (9, 8272, 547), (11020, 8, 1171), (2345, 8, 5813),
            (8418, 137, 1409), (67, 3208, 8259), (64, 2048, 8192), (39, 1656, 6441), (57, 872, 5349)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", VARIANTS)
def test_variants(gdn, dtype, M, C, F):
    t = make(M, C, F, dtype, M + C)
    check_forward(t, gdn.gated_linear(*t[:3]), "silu")
    check_gradient(t, gdn.gated_linear_backward(*t), "silu")


def test_halves_of_one_weight_and_leading_dimensions(gdn):
    import torch
    t = make(6, 64, 96, "bf16", 3)
    w = torch.cat(t[1:3])
    h = gdn.gated_linear(t[0].view(2, 3, 64), w[:96], w[96:])
    assert h.shape == (2, 3, 96)
    check_forward(t, h.view(6, 96), "silu")
    one = gdn.gated_linear(t[0][0], w[:96], w[96:])
    assert one.shape == (96,)
    dw = torch.empty_like(w)
    dx, dg, du = gdn.gated_linear_backward(t[0].view(2, 3, 64), w[:96], w[96:], t[3].view(2, 3, 96), dw_gate=dw[:96], dw_up=dw[96:])
    assert dg.data_ptr() == dw.data_ptr() and dx.shape == (2, 3, 64)
    check_gradient(t, (dx.view(6, 64), dw[:96], dw[96:]), "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,C,F", [(6, 33, 31), (100, 33, 31), (70, 7, 5), (80, 1, 3), (300, 129, 131), (90, 64, 31), (90, 31, 64)])
def test_halves_of_one_odd_weight(gdn, dtype, M, C, F):
    """Tensors that start at any element, as halves of a weight and rows of a buffer with odd sizes do."""
    import torch
    t = make(M, C, F, dtype, M + C)
    dt = t[0].dtype

    def behind_a_row(a):
        return torch.cat([torch.full_like(a[:1], 9), a])[1:]
    x, w, dh = behind_a_row(t[0]), torch.cat(t[1:3]), behind_a_row(t[3])
    h = torch.full((M + 2, F), 9, dtype=dt, device="cuda")
    gdn.gated_linear(x, w[:F], w[F:], out=h[1:-1])
    check_forward(t, h[1:-1], "silu")
    dx, dw = torch.full((M + 2, C), 9, dtype=dt, device="cuda"), torch.full((2 * F + 2, C), 9, dtype=dt, device="cuda")
    got = gdn.gated_linear_backward(x, w[:F], w[F:], dh, dx=dx[1:-1], dw_gate=dw[1:F + 1], dw_up=dw[F + 1:-1])
    check_gradient(t, got, "silu")
    for a in (h, dx, dw):
        assert (a[0] == 9).all() and (a[-1] == 9).all()


@pytest.mark.parametrize("name", ACTS[1:])
def test_gradient_against_differences(gdn, name):
    import torch
    t = make(90, 40, 72, "f32", 11)
    got = [d.double() for d in gdn.gated_linear_backward(*t, activation=name)]
    x, wg, wu, dh = (a.double() for a in t)

    def loss(x, wg, wu):
        return (act(x @ wg.T, name) * (x @ wu.T) * dh).sum()
    g = torch.Generator(device="cuda").manual_seed(1)
    for i in range(3):
        v = torch.randn(got[i].shape, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-5
        a = [x, wg, wu]
        hi, lo = list(a), list(a)
        hi[i], lo[i] = a[i] + e * v, a[i] - e * v
        diff = (loss(*hi) - loss(*lo)) / (2 * e)
        # the difference is off by e^2 times third derivatives of size 1, the kernel by some 100 u
        assert abs(float((got[i] * v).sum() - diff)) <= 1e-6 * float((got[i] * v).abs().sum())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [4, 200])
def test_not_finite_rows_stay_by_themselves(gdn, dtype, M):
    """A NaN or an infinity in a row of x reaches that row of h alone."""
    import torch
    t = make(M, 100, 70, dtype, 8)
    t[0][1, 99] = float("nan")
    t[0][3, 0] = float("inf")
    h = gdn.gated_linear(*t[:3])
    assert h[1].isnan().all() and not h[3].isfinite().any()
    rows = [r for r in range(M) if r not in (1, 3)]
    check_forward([t[0][rows], *t[1:3]], h[rows], "silu")


def test_far_values(gdn):
    """Projections far out: the activation is 0 or the projection itself, its slope 0 or 1, not NaN."""
    import torch
    x = torch.tensor([[1e4], [-1e4], [3e7], [-3e7]], device="cuda").repeat(20, 1)
    w, one = torch.ones(3, 1, device="cuda"), torch.ones(80, 3, device="cuda")
    for name in ACTS[1:]:
        for xs, ds in ((x, one), (x[:4], one[:4])):
            h = gdn.gated_linear(xs, w, w, activation=name)
            assert torch.equal(h, torch.where(xs > 0, xs * xs, 0.0).expand(-1, 3))
            dx, dwg, dwu = gdn.gated_linear_backward(xs, w, w, ds, activation=name)
            assert torch.equal(dx, torch.where(xs > 0, 6 * xs, 0.0))


@pytest.mark.parametrize("M,C,F", [(3, 129, 40), (500, 129, 40), (500, 128, 40)])
def test_outputs_alone_are_written(gdn, M, C, F):
    """Guards around every output and the workspace stay as they are."""
    import torch
    t = make(M, C, F, "bf16", 5)

    def guarded(*shape, dt=torch.bfloat16):
        n = 1
        for s in shape:
            n *= s
        buf = torch.full((n + 1024,), 7, dtype=dt, device="cuda")
        return buf, buf[512:512 + n].view(shape)
    bufs = [guarded(M, F), guarded(M, C), guarded(F, C), guarded(F, C)]
    lib = gdn.block._lib()
    n = [lib.gdn_gated_linear_workspace_bytes(M, C, F, 1, b) for b in (0, 1)]
    ws = [guarded(k, dt=torch.uint8) for k in n]
    gdn.gated_linear(*t[:3], out=bufs[0][1], ws=ws[0][1] if n[0] else None)
    gdn.gated_linear_backward(*t, dx=bufs[1][1], dw_gate=bufs[2][1], dw_up=bufs[3][1], ws=ws[1][1])
    check_forward(t, bufs[0][1], "silu")
    check_gradient(t, [b[1] for b in bufs[1:]], "silu")
    for buf, _ in bufs + ws:
        assert (buf[:512] == 7).all() and (buf[-512:] == 7).all()


@pytest.mark.parametrize("M", [8, 300])
def test_captured_and_on_another_stream(gdn, M):
    """The same bits from a stream of one's own and from replays of a graph, with eager calls between them."""
    import torch
    t = make(M, 200, 160, "bf16", 9)
    want = (gdn.gated_linear(*t[:3]), *gdn.gated_linear_backward(*t))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = (gdn.gated_linear(*t[:3], stream=s), *gdn.gated_linear_backward(*t, stream=s))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    ws = [gdn.gated_linear_workspace(t[0], t[1], backward=b) for b in (False, True)]
    out = [torch.zeros_like(a) for a in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gdn.gated_linear(*t[:3], out=out[0], ws=ws[0])
        gdn.gated_linear_backward(*t, dx=out[1], dw_gate=out[2], dw_up=out[3], ws=ws[1])
    for i in range(4):
        for o in out:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), i
        t[0].mul_(-0.5)
        want = (gdn.gated_linear(*t[:3]), *gdn.gated_linear_backward(*t))
        torch.cuda.synchronize()


def test_what_is_written_counts_as_modified(gdn):
    import torch
    t = make(3, 16, 8, "f32", 1)
    out = torch.empty(3, 8, device="cuda")
    v = out._version
    gdn.gated_linear(*t[:3], out=out)
    assert out._version > v
    with pytest.raises(ValueError, match="gradient"):
        gdn.gated_linear(*t[:3], out=out.requires_grad_())
