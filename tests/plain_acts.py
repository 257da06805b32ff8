"""Activations and slopes in fp64 for the tests of the block's operators, with what fp32 arithmetic may be off by.

With u = 2^-24 and z known to ez: the value is off by at most 1.2 ez (no slope is above 1.2) plus (16 + cond) u of
itself, where cond counts what an exponential or the normal distribution makes of a rounded argument: |z| for silu,
2 z^2 for gelu, five roundings of 2k for its tanh form.  A slope's own slope is below 1.2 as well, and its terms are
below 2 in size."""
import math

import torch

U = 2.0 ** -24
ACTS = [None, "silu", "gelu", "gelu_tanh"]


def half(dtype):
    """Half a step of a type, relative."""
    return torch.finfo(dtype).eps / 2


def act(z, name):
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return z * torch.special.ndtr(z)
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope(z, name):
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def cond(z, name):
    if name is None:
        return torch.zeros_like(z)
    a = z.abs()
    return a + 2 * a ** 2 + 5 * (1.6 * a + 0.0714 * a ** 3)


def act_error(z, ez, name):
    return 1.2 * ez + (16 + cond(z, name)) * U * act(z, name).abs()


def slope_error(z, ez, name):
    return 1.2 * ez + (16 + cond(z, name)) * U * 2 if name else torch.zeros_like(z)


def close(name, got, ref, tol):
    got = got.double().to(ref.device)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert got.isfinite().all(), name
    d = (got - ref).abs()
    assert (d <= tol).all(), (name, float((d - tol).max()), float(d.max()), int((d > tol).sum()))
