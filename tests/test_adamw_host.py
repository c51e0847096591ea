"""What AdamW refuses of its arguments before a device is used."""
import types

import pytest


@pytest.mark.parametrize("masters", [(), (None,), (None, None, None)])
def test_masters_from_an_iterator_go_with_the_parameters_one_each(masters):
    """Of two parameters; a shorter one would leave tensors out of every step."""
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g = [torch.zeros(3, 8), torch.zeros(5)], [torch.zeros(3, 8), torch.zeros(5)]
    with pytest.raises(ValueError, match="masters"):
        AdamW(p, g, masters=iter(masters))


def test_a_stream_of_another_device_is_refused():
    import torch
    from paper_2309_03523_amd import binding
    stream = types.SimpleNamespace(device=torch.device("cuda", 1))
    with pytest.raises(ValueError, match="another device"):
        binding.adamw_step(None, 0, 1, lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, stream=stream)
