"""GPU: gradients whose every step is exact in fp32, so that the result is the exact one, rounded
once.  All gates are 1 and keys are unit vectors, so decays and T hold only 0, 1 and -1; products of
dout with values are 1 + 2^-9 + 2^-17 and its neighbours, which 24 bits hold and 16 do not, and what
reaches dq and dk are their differences of 2^-16."""
import pytest

from test_gpu_backward import adjoint, host

pytestmark = pytest.mark.gpu


def make(tokens, T, H, Dk, Dv, dtype):
    """Head 0, tokens a < b < c: a and b write to one key, c reads it and writes beside it:
    dq_c and dk_c are sums over a and b of opposite terms.  Head 1: b and c read beside the key of a with
    opposite douts: dk_a is such a sum.  Further heads repeat these two; other tokens are zeros."""
    import torch
    a, b, c = tokens
    t = {n: torch.zeros(1, T, H, d) for n, d in (("q", Dk), ("k", Dk), ("v", Dv), ("dout", Dv))}
    value = torch.tensor([1.0, 2.0 ** -9, 2.0 ** -17])
    at = [3, Dv // 2, Dv - 1]
    q, k, v, do = (t[n][0] for n in ("q", "k", "v", "dout"))
    k[a, 0::2, 7] = k[b, 0::2, 7] = 1
    k[c, 0::2, Dk - 1] = q[c, 0::2, Dk - 1] = 1
    k[a, 1::2, 2] = 1
    q[b, 1::2, 9] = q[c, 1::2, 9] = 1
    for i, x in zip(at, value):
        v[a, :, i] = x
    v[b, 0::2, at[2]] = 2.0 ** -16
    for i in at:
        do[c, 0::2, i] = 1
        do[b, 1::2, i] = 1
        do[c, 1::2, i] = 1 if i == at[2] else -1
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    t = {n: x.to(dt) for n, x in t.items()}
    t.update(alpha=torch.ones(1, T, H), beta=torch.ones(1, T, H), state_in=None, dstate_out=None)
    return {n: None if x is None else x.cuda() for n, x in t.items()}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 128), (64, 128), (128, 64)])
@pytest.mark.parametrize("tokens,T", [((0, 1, 2), 3), ((3, 20, 50), 64), ((69, 70, 127), 130)])
@pytest.mark.parametrize("H", [2, 300])
def test_differences_of_large_terms(gdn, dtype, Dk, Dv, tokens, T, H):
    import torch
    t = make(tokens, T, H, Dk, Dv, dtype)
    got = gdn.backward(**t)
    two = {n: x if x is None else x[:, :, :2] for n, x in t.items()}
    ref = adjoint(host(two))
    a, _, c = tokens
    assert abs(float(ref[0][0, c, 0, 7])) == abs(float(ref[1][0, c, 0, 7])) == abs(float(ref[1][0, a, 1, 9])) == 2.0 ** -16
    for name, x, r in zip(("dq", "dk", "dv"), got, ref):
        x = x.cpu()
        for h in range(0, H, 2):
            assert torch.equal(x[:, :, h:h + 2], r.to(x.dtype)), (name, h)
