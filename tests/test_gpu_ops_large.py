"""GPU: the operators where element offsets pass 32 bits, and the refusal of sizes that do not fit
the 32-bit arguments below the binding.  Expected values come from a small call of the
same operator, itself checked against fp64 elsewhere."""
import pytest

import test_gpu_backward as backward
import test_gpu_block_norm as norm

pytestmark = pytest.mark.gpu


def room(gib):
    import torch
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < gib << 30:
        pytest.skip(f"needs {gib} GiB of device memory")


def test_step_in_a_large_pool(gdn):
    """Slot 4096 of 64 heads begins at element 2^32: the states there are updated, and not those that
    an offset of 32 bits would find."""
    import torch
    room(24)
    H, D, P = 64, 128, 4100
    slots = [4096, 4099, 2]
    g = torch.Generator().manual_seed(31)
    q, k = (torch.nn.functional.normalize(torch.randn(3, 2, H, D, generator=g), dim=-1).cuda() for _ in range(2))
    v = torch.randn(3, 2, H, D, generator=g).cuda()
    a, b = (torch.rand(3, 2, H, generator=g).cuda() for _ in range(2))
    states = torch.randn(3, H, D, D, generator=g).cuda()
    ref, after = gdn.step(q, k, v, a, b, states, state_out=torch.empty_like(states))
    pool = torch.empty(P, H, D, D, device="cuda")
    pool[:8] = 7.0
    for s, x in zip(slots, states):
        pool[s] = x
    out, _ = gdn.step(q, k, v, a, b, pool, slots=torch.tensor(slots, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, ref)
    for s, x in zip(slots, after):
        assert torch.equal(pool[s], x), s
    assert all((pool[s] == 7.0).all() for s in (0, 1, 3, 4, 5))


def test_block_norm_of_many_rows(gdn):
    """The last five of 2^19 + 5 rows of 8192 channels; the others are zero, and so are their parts in
    the sums over rows."""
    import torch
    room(48)
    n, R, C = 5, (1 << 19) + 5, 8192
    t = norm.make(1, n, C, n, "bf16", 32)
    big = {name: torch.zeros(1, R, C, dtype=torch.bfloat16, device="cuda") for name in ("x", "y", "du")}
    for name in big:
        big[name][:, -n:] = t[name]
    t["dr"] = None
    w = (t["gate"], t["w_post"], t["w_pre"])
    u = torch.empty_like(big["x"])
    r, u = gdn.block_norm(big["x"], big["y"], *w, gate_tokens=R, res_scale=0.7, u=u, r=torch.empty_like(u))
    norm.check_forward(t, r[:, -n:], u[:, -n:], n, 0.7)
    assert not r[:, :R - n:997].any() and not u[:, :R - n:997].any()
    got = gdn.block_norm_backward(big["x"], big["y"], *w, big["du"], gate_tokens=R, res_scale=0.7, dx=r, dy=u)
    norm.check_grad(t, (got[0][:, -n:], got[1][:, -n:]) + got[2:], n, 0.7)


def test_backward_of_many_chunks(gdn):
    """The last of 64 heads of 131153 tokens lies behind element 2^31 of the kept states and byte 2^32 of
    the workspace; against the call of that head alone (each within the tolerance of the
    gradient, so twice that, and one step of bf16, between them)."""
    import torch
    room(96)
    H, T, D = 64, 131153, 128
    one = backward.make(1, T, 1, D, D, "bf16", 33, mu=-3.0)
    ref = gdn.backward(**one)
    big = {n: (x.expand(-1, H, -1, -1) if n in ("state_in", "dstate_out") else x.expand(-1, -1, H, *x.shape[3:])).contiguous()
           for n, x in one.items()}
    got = gdn.backward(**big)
    for name, x, r in zip(backward.NAMES, got, ref):
        for h in (0, H - 1):
            y = (x[:, h:h + 1] if name == "dstate_in" else x[:, :, h:h + 1]).double()
            r64 = r.double()
            step = 2.0 ** -7 if r.dtype == torch.bfloat16 else 0.0
            over = ((y - r64).abs() - step * r64.abs()).clamp_min(0.0)
            assert y.isfinite().all() and float(over.norm()) <= 2 * backward.TOL["bf16"] * float(r64.norm()), (name, h)


def test_block_norm_rows_past_32_bits_are_refused(gdn):
    import torch
    room(16)
    x = torch.empty(1, (1 << 32) + 4, 1, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(1, device="cuda")
    with pytest.raises(ValueError, match="2\\^31"):
        gdn.block_norm(x, x, None, w, w, r=x, u=x)
    with pytest.raises(ValueError, match="2\\^31"):
        gdn.block_norm_backward(x, x, None, w, w, x, dx=x, dy=x)
