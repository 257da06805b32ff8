"""GPU: the variants of the gradient's kernels that calls of many heads and chunks take, in every head
shape, each head with values of its own, against the recurrence's adjoint in fp64 (inputs,
reference and tolerances of test_gpu_backward).

The last launch has four waves from 257 chunks and heads on and eight below; the scan of bf16 heads of
Dk = Dv = 128 loads its operands directly from 17 heads on (at Dv = 64 it has as many workgroups from 33 on)."""
import pytest

from test_gpu_backward import NAMES, TOL, adjoint, compare, host, make
from test_gpu_ops_large import room

pytestmark = pytest.mark.gpu


def head(t, b, h):
    """The tensors of one head, contiguous."""
    return {n: None if x is None else (x[b:b + 1, h:h + 1] if n in ("state_in", "dstate_out") else x[b:b + 1, :, h:h + 1]).contiguous()
            for n, x in t.items()}


def result(got, b, h):
    return [x[b:b + 1, h:h + 1] if n == "dstate_in" else x[b:b + 1, :, h:h + 1] for n, x in zip(NAMES, got)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("B,T,H", [(1, 300, 60), (2, 520, 17)])
def test_many_heads(gdn, dtype, Dk, Dv, B, T, H):
    """300 and 306 chunks and heads, the last chunk short; 60 and 34 heads."""
    t = make(B, T, H, Dk, Dv, dtype, 40 + T + Dk + 2 * Dv, mu=-2.0)
    got = gdn.backward(**t)
    for b, h in ((0, 0), (B - 1, H // 2), (B - 1, H - 1)):
        one = head(t, b, h)
        ref = adjoint(host(one))
        label = f"{B}x{H} {Dk}x{Dv} {dtype} head {b},{h}"
        compare(result(got, b, h), ref, dtype, label)
        compare(gdn.backward(**one), ref, dtype, label + " alone")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("H", [16, 17, 32, 33])
def test_short_sequences_of_many_heads(gdn, dtype, Dk, Dv, H):
    """On both sides of the scans' borders, a chunk and a token, without states."""
    t = make(1, 65, H, Dk, Dv, dtype, 50 + H + Dk + 2 * Dv, mu=-1.0, state=False)
    got = gdn.backward(**t)
    for h in (0, H - 1):
        compare(result(got, 0, h), adjoint(host(head(t, 0, h))), dtype, f"{H} heads {Dk}x{Dv} {dtype} head {h}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("name", ["q", "k", "v", "dout", "state_in", "dstate_out"])
def test_infinities_stay_in_their_head(gdn, dtype, name):
    import torch
    t = make(2, 150, 3, 64, 64, dtype, 60, mu=-1.0)
    ref = gdn.backward(**t)
    t[name][(1, 2, 3, 4) if "state" in name else (1, 70, 2, 7)] = float("inf")
    got = gdn.backward(**t)
    for n, a, b in zip(NAMES, ref, got):
        for i in range(2):
            for h in range(3):
                if (i, h) != (1, 2):
                    x, y = (z[i, h] if n == "dstate_in" else z[i, :, h] for z in (a, b))
                    assert torch.equal(x, y), (n, i, h)
    assert not all(x.isfinite().all() for x in got)


def test_many_chunks_of_different_heads(gdn):
    """The last of 64 heads lies behind element 2^31 of the kept states and byte 2^32 of the workspace.
    Each head has one head's inputs with v and state_in times 2^i and dout and dstate_out times 2^j, (i, j)
    its own, so its results are that head's times 2^j, 2^(i + j): another head's records would be off
    by a factor of two at least.  Tolerance: both calls within the gradient's, and one step of bf16."""
    import torch
    room(96)
    H, T, D = 64, 131153, 128
    one = make(1, T, 1, D, D, "bf16", 34, mu=-3.0)
    ref = gdn.backward(**one)
    assert len({(h % 8, h // 8) for h in range(H)}) == H
    si = torch.tensor([2.0 ** (h % 8 - 4) for h in range(H)], device="cuda")
    sj = torch.tensor([2.0 ** (h // 8 - 4) for h in range(H)], device="cuda")
    by = dict(v=si, state_in=si, dout=sj, dstate_out=sj)
    big = {}
    for n, x in one.items():
        state = n in ("state_in", "dstate_out")
        y = (x.expand(-1, H, -1, -1) if state else x.expand(-1, -1, H, *x.shape[3:])).contiguous()
        if n in by:
            y *= (by[n].view(1, H, 1, 1) if state else by[n].view(1, 1, H, 1)).to(y.dtype)
        big[n] = y
    got = gdn.backward(**big)
    for h in (0, 7, 29, 56, H - 1):
        for name, x, r in zip(NAMES, result(got, 0, h), ref):
            y = x.double() / float(sj[h] if name in ("dv", "dstate_in") else si[h] * sj[h])
            r64 = r.double()
            step = 2.0 ** -7 if r.dtype == torch.bfloat16 else 0.0
            over = ((y - r64).abs() - step * r64.abs()).clamp_min(0.0)
            assert y.isfinite().all() and float(over.norm()) <= 2 * TOL["bf16"] * float(r64.norm()), (name, h)


@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 64), ("bf16", 128)])
def test_as_many_heads_as_are_allowed(gdn, dtype, D):
    """65535 heads, a chunk and two tokens."""
    import torch
    room(100)
    T, H = 66, 65535
    g = torch.Generator(device="cuda").manual_seed(70 + D)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def rn(*s):
        return torch.randn(s, generator=g, device="cuda")
    t = dict(q=torch.nn.functional.normalize(rn(1, T, H, D), dim=-1).to(dt), k=torch.nn.functional.normalize(rn(1, T, H, D), dim=-1).to(dt),
             v=rn(1, T, H, D).to(dt), alpha=torch.sigmoid(rn(1, T, H) + 2.0), beta=torch.sigmoid(rn(1, T, H)), state_in=0.3 * rn(1, H, D, D),
             dout=rn(1, T, H, D).to(dt), dstate_out=0.3 * rn(1, H, D, D))
    got = gdn.backward(**t)
    for h in (0, 32768, H - 1):
        compare(result(got, 0, h), adjoint(host(head(t, 0, h))), dtype, f"{H} heads of {D} {dtype} head {h}")
