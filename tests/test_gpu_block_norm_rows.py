"""GPU: the block norm on more rows than a launch of one team to four of them has threads for."""
import pytest

from test_gpu_block_norm import check_forward, make
from test_gpu_ops_large import room

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [3, 9])
def test_more_rows_than_a_launch_has_threads(gdn, C):
    """2^28 + 1029 rows, copies of 1024: a row's result does not depend on its place."""
    import torch
    room(40)
    n, R = 1024, (1 << 28) + 1024 + 5
    t = make(1, n, C, 1, "bf16", C, gated=False)
    w = (t["w_post"], t["w_pre"])
    ref = gdn.block_norm(t["x"], t["y"], None, *w, res_scale=0.5)
    check_forward(t, *ref, 1, 0.5)
    big = [t[k].expand(R // n + 1, n, C).reshape(1, -1, C)[:, :R].contiguous() for k in ("x", "y")]
    got = gdn.block_norm(*big, None, *w, res_scale=0.5, r=big[0], u=big[1])
    for x, y in zip(got, ref):
        whole = R // n * n
        assert (x[:, :whole].view(-1, n, C) == y).all() and torch.equal(x[:, whole:], y[:, :R - whole])


def test_gate_tokens_is_a_whole_number(gdn):
    """1.5 is refused, not cut to 1."""
    t = make(1, 6, 16, 1, "f32", 4)
    args = (t["x"], t["y"], t["gate"], t["w_post"], t["w_pre"])
    for bad in (1.5, (1 << 32) + 1, -1, 0):
        with pytest.raises(ValueError):
            gdn.block_norm(*args, gate_tokens=bad)
        with pytest.raises(ValueError):
            gdn.block_norm_backward(*args, t["du"], gate_tokens=bad)
    check_forward(t, *gdn.block_norm(*args, gate_tokens=1.0), 1, 1.0)
