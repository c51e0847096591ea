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


@pytest.mark.parametrize("given", [False, True])
def test_a_step_that_the_host_counts_is_not_captured(given):
    """Its number would be that of the capture in every replay."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g = torch.ones(4, 16, device="cuda"), torch.ones(4, 16, device="cuda")
    opt = AdamW([p], [g])
    opt.step()
    torch.cuda.synchronize()
    before, graph, s = p.clone(), torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=s):
        p.mul_(2)
        with pytest.raises(RuntimeError, match="on_device"):
            opt.step(stream=s if given else None)
    assert opt.steps == 1
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(p, 2 * before)
    opt.step(stream=s if given else None)      # outside the capture it goes on
    torch.cuda.synchronize()
    assert opt.steps == 2 and bool((p < 2 * before).all())


def test_a_rate_on_the_device_goes_with_the_number_of_steps_there():
    import torch
    from paper_2309_03523_amd import binding
    from paper_2309_03523_amd.optimizer import AdamW
    p, g = torch.ones(4, 16, device="cuda"), torch.ones(4, 16, device="cuda")
    opt = AdamW([p], [g])
    kw = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8)
    with pytest.raises(binding.DgcError, match="lr on the device"):
        binding.adamw_step(opt._handle, p.device.index, 1, lr_at=torch.ones(1, device="cuda"), **kw)
    with pytest.raises(ValueError):
        binding.adamw_step(opt._handle, p.device.index, 1, lr_at=torch.ones(2, device="cuda"), **kw)
    assert bool((p == 1).all())
