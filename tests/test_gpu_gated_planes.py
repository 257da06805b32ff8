"""The gated linear map's fp32 products to within some steps of fp32, in every variant: rows of x and of dh with two
values that are not zero, so that few roundings stand between a result and its definition, however long the contraction is.

Tolerances, with u = 2^-24.  An operand is cut into planes of 8 bits: behind the first is less than 2^-7 of it, behind
the second less than 2^-15, so the three products of planes that are left out are below (2 2^-22 + 2^-30) |a b| = 8.1 u |a b|.
The other six are exact and added one by one, each addition off by a step, 2 u, of what is then there, at most 1.02 times the
sum of absolute products; zeros change nothing.  Sums of parts, or of waves, add n u.  For n products that is (9 + 14 n) u of the sum of
absolute ones.  h, dg and du are one product more, u each.
"""
import pytest
import torch

import test_gpu_gated_linear as sizes
from plain_acts import U, close


def make(M, C, F, seed):
    g = torch.Generator().manual_seed(seed)

    def two(rows, n):
        """Two values a row, in places that move from row to row."""
        a = torch.zeros(rows, n)
        at = torch.randint(0, n, (rows, 2), generator=g)
        return a.scatter_(1, at, torch.randn(rows, 2, generator=g))
    return [two(M, C), torch.randn(F, C, generator=g), torch.randn(F, C, generator=g), two(M, F)]


def product(a, ea, b, eb):
    """a @ b, and what it may be off by where the operands are by ea and eb."""
    n = (a != 0).double() @ (b != 0).double()
    return a @ b, ea @ (b.abs() + eb) + a.abs() @ eb + (9 + 14 * n) * U * (a.abs() @ b.abs())


def forward(t):
    x, wg, wu = (a.double() for a in t[:3])
    zx, zw = torch.zeros_like(x), torch.zeros_like(wg.T)
    return (*product(x, zx, wg.T, zw), *product(x, zx, wu.T, zw))


def check_forward(t, h):
    g, eg, u, eu = forward(t)
    close("h", h, g * u, eg * (u.abs() + eu) + g.abs() * eu + 1.01 * U * (g * u).abs())


def check_gradient(t, got):
    g, eg, u, eu = forward(t)
    x, wg, wu, dh = (a.double() for a in t)
    zx, zw = torch.zeros_like(x), torch.zeros_like(wg)
    dg, du = dh * u, dh * g                                 # no activation
    edg, edu = (dh.abs() * e + 1.01 * U * d.abs() for d, e in ((dg, eu), (du, eg)))
    # dx is one sum of both products
    dx, edx = product(torch.cat([dg, du], 1), torch.cat([edg, edu], 1), torch.cat([wg, wu]), torch.cat([zw, zw]))
    close("dx", got[0], dx, edx)
    for name, d, e, w in (("dw_gate", dg, edg, got[1]), ("dw_up", du, edu, got[2])):
        close(name, w, *product(d.T, e.T, x, zx))


@pytest.mark.gpu
@pytest.mark.parametrize("M,C,F", sizes.VARIANTS + sizes.SMALL)
def test_few_products(gdn, M, C, F):
    t = [a.cuda() for a in make(M, C, F, M + C + F)]
    check_forward(t, gdn.gated_linear(*t[:3], activation=None))
    check_gradient(t, gdn.gated_linear_backward(*t, activation=None))


def planes(a):
    out = []
    for _ in range(3):
        p = (a.view(torch.int32) & -65536).view(torch.float32)
        out.append(p.double())
        a = a - p
    return out


SIX = [(2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0)]


@pytest.mark.parametrize("without", [None, *SIX])
def test_the_bound_asks_for_all_six_products_of_planes(without):
    """The same products on the host, planes cut as the kernels do: within a third of the bound; and with one product
    of planes left out far outside it."""
    x, wg, wu, dh = make(64, 96, 80, 1)

    def mul(a, b):
        a, b = planes(a.contiguous()), planes(b.contiguous())
        return sum(a[i] @ b[j] for i, j in SIX if (i, j) != without).float()

    def worst(got, ref, tol):
        return float(((got.double() - ref).abs() / tol.clamp_min(1e-300)).max())
    g, eg, u, eu = forward([x, wg, wu])
    gs, us = mul(x, wg.T), mul(x, wu.T)
    off = [worst(gs, g, eg), worst(us, u, eu)]
    dg = (dh * us).contiguous()
    exact, zero = dg.double(), torch.zeros(80, 64, dtype=torch.float64)
    off.append(worst(mul(dg.T, x), *product(exact.T, zero, x.double(), torch.zeros(64, 96, dtype=torch.float64))))
    assert max(off) < 1 / 3 if without is None else min(off) > 10, off
