"""GPU: what the operators write in place is known to autograd: a saved tensor that a call has written is
an error in the backward pass, as after torch's own in-place calls, and a tensor that requires a
gradient is not written while gradients are recorded."""
import pytest

import test_gpu_backward as backward
import test_gpu_block_norm as norm
import test_gpu_step as step

pytestmark = pytest.mark.gpu


def calls(gdn):
    """Per operator: a function of the tensors it writes, and those tensors."""
    import torch
    t, slots = step.make(3, 1, 4, 2, 4, 64, 64, "f32", 1)
    pool, out = t.pop("state"), torch.zeros_like(t["v"])
    yield "step in place", lambda pool, out: gdn.step(**t, state=pool, slots=slots, out=out), (pool, out)
    yield "step to a pool", lambda new: gdn.step(**t, state=pool, slots=slots, state_out=new), (torch.zeros_like(pool),)
    b = backward.make(1, 70, 2, 64, 64, "f32", 2)
    outs = [torch.empty_like(x) for x in gdn.backward(**b)]
    yield "backward", lambda *o: gdn.backward(**b, **dict(zip(backward.NAMES, o))), outs
    n = norm.make(1, 8, 64, 4, "f32", 3)
    w = (n["gate"], n["w_post"], n["w_pre"])
    yield "norm in place", lambda x, y: gdn.block_norm(x, y, *w, gate_tokens=4, r=x, u=y), (n["x"].clone(), n["y"].clone())
    grads = [torch.empty_like(n[k]) for k in ("gate", "w_post", "w_pre")]
    yield "norm gradient", lambda du, dr, dg, dp, dq: gdn.block_norm_backward(
        n["x"], n["y"], *w, du, dr, gate_tokens=4, dx=dr, dy=du, dgate=dg, dw_post=dp, dw_pre=dq), (n["du"], n["dr"], *grads)


def test_saved_tensors(gdn):
    import torch
    for name, call, written in calls(gdn):
        for i in range(len(written)):
            w = torch.ones((), device="cuda", requires_grad=True)
            loss = (w * written[i]).sum()                       # saves the tensor
            loss.backward(retain_graph=True)                    # as yet as it was
            call(*written)
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                loss.backward()
            print(f"[autograd] {name} {i}", flush=True)


def test_inputs_that_are_read_stay_as_they_are(gdn):
    import torch
    t, slots = step.make(3, 1, 4, 2, 4, 64, 64, "f32", 4)
    before = {n: x._version for n, x in t.items()}
    gdn.step(**t, slots=slots, state_out=torch.zeros_like(t["state"]))
    assert slots._version == 0 and {n: x._version for n, x in t.items()} == before


def test_written_tensors_that_require_a_gradient(gdn):
    """Refused while gradients are recorded, whole and as results of a graph; written without."""
    import torch
    for name, call, written in calls(gdn):
        for i, x in enumerate(written):
            leaf = torch.full_like(x, 0.5, requires_grad=True)
            for y in (leaf, leaf * 1.0):
                args = list(written)
                args[i] = y
                with pytest.raises(ValueError, match="requires a gradient"):
                    call(*args)
                assert (y == 0.5).all(), (name, i)
                with torch.no_grad():
                    call(*args)
                    assert not (y == 0.5).all(), (name, i)
                    leaf.fill_(0.5)


def test_inference_tensors(gdn):
    """Made in inference mode, they have no history to tell of: written in it and outside."""
    import torch
    with torch.inference_mode():
        for _, call, written in calls(gdn):
            call(*written)
        made = list(calls(gdn))
    for _, call, written in made:
        call(*written)
