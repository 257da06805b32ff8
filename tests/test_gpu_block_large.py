"""GPU: offsets past 32 bits, in elements and in bytes, in the operators of gdn_block.h.  Rows from both ends and around
2^31 elements are held to the same bounds as small cases are."""
import pytest

import test_gpu_gated_linear as gated
import test_gpu_short_conv as conv
from plain_acts import U

pytestmark = pytest.mark.gpu


def randn(gen, *shape):
    import torch
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def test_gated_linear(gdn):
    import torch
    M, C, F = 140000, 64, 16384
    g = torch.Generator(device="cuda").manual_seed(1)
    t = [randn(g, M, C), randn(g, F, C) / 8, randn(g, F, C) / 8]
    h = gdn.gated_linear(*t)
    at = [0, 1, 2 ** 31 // F - 1, 2 ** 31 // F, M - 257, M - 1]
    rows = torch.tensor(at, device="cuda")
    gated.check_forward([t[0][rows], *t[1:]], h[rows], "silu")
    dh = torch.zeros(M, F, device="cuda", dtype=torch.bfloat16)      # the weights' gradients: of these rows alone
    dh[rows] = randn(g, len(at), F)
    dx, dwg, dwu = gdn.gated_linear_backward(*t, dh)
    gated.check_gradient([t[0][rows], *t[1:], dh[rows]], (dx[rows], dwg, dwu), "silu")
    keep = torch.ones(M, dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert (dx[keep] == 0).all()


def test_short_conv(gdn):
    import torch
    T, C, W = 70000, 32768, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    x, w, bias = randn(g, 1, T, C), torch.randn(C, W, generator=g, device="cuda"), torch.randn(C, generator=g, device="cuda")
    y, state = gdn.short_conv(x, w, bias)
    for a, b in ((0, 10), (2 ** 31 // C - 5, 2 ** 31 // C + 5), (T - 10, T)):
        s = x[:, a - 3:a] if a else None
        conv.check_forward(dict(x=x[:, a:b], w=w, bias=bias, state=s), y[:, a:b], state if b == T else None, "silu")
    dy = torch.zeros_like(x)
    a, b = 2 ** 31 // C - 5, T - 3
    dy[:, a:] = randn(g, 1, T - a, C)
    dx, dw, dbias, _ = gdn.short_conv_backward(x, w, bias, None, dy)
    assert (dx[:, :a - 3] == 0).all()
    t = dict(x=x[:, a:], w=w[:256].contiguous(), bias=bias[:256].contiguous(), state=x[:, a - 3:a], dy=dy[:, a:], dstate=None)
    cut = {n: v if v is None or n in ("w", "bias") else v[..., :256] for n, v in t.items()}
    conv.check_gradient(cut, (dx[:, a:, :256], dw[:256], dbias[:256], dx[:, a - 3:a, :256]), "silu")


def test_gradient_norm(gdn):
    import torch
    n = 2 ** 31 + 12345
    x = torch.ones(n, device="cuda", dtype=torch.bfloat16)
    norm, _ = gdn.clip_grads([x], 1.0, eps=0.0)
    assert abs(float(norm) / n ** 0.5 - 1) <= 2 * U
    want = torch.tensor(1 / n ** 0.5).bfloat16()
    assert bool((x == want.cuda()).all())
