"""GPU: the step with slots and an output of its own making, captured."""
import pytest

from test_gpu_step import make

pytestmark = pytest.mark.gpu


def test_captured_with_a_fresh_output(gdn):
    """Each replay clears the rows that are short or padding and advances the pool as an eager call does."""
    import torch
    t, slots = make(5, 2, 7, 2, 4, 64, 128, "bf16", 51)
    slots[3] = -1
    lengths = torch.tensor([2, 1, 0, 2, 2], dtype=torch.int32, device="cuda")
    eager = {n: x.clone() for n, x in t.items()}
    gdn.step(**{n: x.clone() for n, x in t.items()}, slots=slots, lengths=lengths)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, pool = gdn.step(**t, slots=slots, lengths=lengths)
    for i in range(4):
        graph.replay()
        ref, _ = gdn.step(**eager, slots=slots, lengths=lengths)
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(pool, eager["state"]), i
        out.fill_(float("nan"))
        lengths[i] = (int(lengths[i]) + 1) % 3
