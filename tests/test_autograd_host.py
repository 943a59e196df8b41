"""The forward calls and autograd: tensors that it follows are refused before anything else is looked at."""
import pytest
import torch

from paper_2009_03106_amd import dpclip as dp


def tensors(leaf):
    x, g = torch.zeros(1, 2, 3, 4), torch.zeros(4)
    return [t.requires_grad_() if i == leaf else t for i, t in enumerate((x, g, torch.zeros(1, 2, 3, 4)))]


@pytest.mark.parametrize("leaf", [0, 1, 2])
def test_headnorm(leaf):
    x, g, out = tensors(leaf)
    with pytest.raises(RuntimeError, match="records no gradients"):
        dp.headnorm([(x, g)], [out])
    with torch.no_grad(), pytest.raises(ValueError):                                      # host tensors
        dp.headnorm([(x, g)], [out])
    with pytest.raises(ValueError):
        dp.headnorm([(x.detach(), g.detach())], [out.detach()])


@pytest.mark.parametrize("leaf", [0, 1, 2])
def test_posbias_add(leaf):
    s, t, out, b = torch.zeros(1, 2, 3, 4), torch.zeros(8, 2), torch.zeros(1, 2, 3, 4), torch.zeros(9, dtype=torch.int32)
    (s, t, out)[leaf].requires_grad_()
    with pytest.raises(RuntimeError, match="records no gradients"):
        dp.posbias_add(s, t, b, out)
    with torch.no_grad(), pytest.raises(ValueError):
        dp.posbias_add(s, t, b, out)
    if leaf == 0:
        with pytest.raises(RuntimeError):
            dp.posbias_add(s * 2, t, b)                                                   # inside a graph, in place
