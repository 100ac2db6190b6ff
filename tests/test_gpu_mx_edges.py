"""Calls of the expert router and the MXFP4 operators at the edges of what their documentation allows, against plain 64-bit forms (mx_reference.py)."""
import pytest
import torch

from test_gpu_mx import check_route

pytestmark = pytest.mark.gpu


# -- router -----------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("a", [10.0, 100.0, 1e3, 1e4])
@pytest.mark.parametrize("spread", [1.0, 0.02])
def test_groups_whose_biases_cancel(kind, a, spread):
    """A group's two choices are rounded at the size of their biases, however small their sum is: groups closer than that, all of them so or every other."""
    E, G = 128, 64
    gen = torch.Generator().manual_seed(int(a))
    l = torch.randn(48, E, generator=gen) * spread
    both = torch.tensor([a, -a]).repeat(G)
    half = both.clone().view(G, 2)
    half[1::2] = 0.0
    for bias in (both, half.view(-1)):
        check_route(l, bias, kind, G, 8, 2, 8, 1, 1.0)
