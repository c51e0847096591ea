"""What counts as a step of AdamW, and which tensors it steps."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("shape", [(0, 16), (3, 0), (0,)])
def test_steps_of_empty_tensors_count(shape, bits):
    """Wherever the number of steps is kept, eager or replayed."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g = torch.zeros(*shape, device="cuda"), torch.zeros(*shape, device="cuda")
    host, there = AdamW([p], [g], bits=bits, steps=4), AdamW([p], [g], bits=bits, steps=4, on_device=True)
    for t in (5, 6):
        host.step()
        there.step()
        assert host.steps == t == there.steps
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        there.step()
    for t in (7, 8, 9):
        graph.replay()
        assert there.steps == t
