"""The choice of experts and its gradient, in every form that the kernel is built in, against 64 bits."""
import numpy as np
import pytest

import block_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mad():
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    return m


@pytest.mark.parametrize("T,E,groups", [(3, 8, 2), (5, 60, 4), (40, 64, 8), (9, 256, 8), (2000, 256, 8), (2000, 120, 8), (7, 1024, 64)])
def test_groups_of_experts_with_the_lowest_bias(mad, T, E, groups):
    """A bias of the type's lowest value is a number: the sum of a group's two largest keys is then minus infinity, and the group has experts
    all the same.  Keys and sums are equal, so the lower indices come first."""
    import torch
    print("case lowest bias", T, E, groups, flush=True)
    x = torch.linspace(-1, 1, T * E, device="cuda").view(T, E)
    bias = torch.full((E,), torch.finfo(torch.float32).min, device="cuda")
    size, k = E // groups, 3
    for kept in (1, groups):
        ids, w = mad.maddness_route(x, k, "sigmoid", bias, groups, kept, renormalise=False)
        assert (ids.cpu() == torch.arange(k)).all()
        assert (w.double() - torch.sigmoid(x[:, :k].double())).abs().max() <= 8 * 2.0 ** -24
    x[:, :size] = float("-inf")                            # a group without an expert comes before none of the others
    ids, _ = mad.maddness_route(x, k, "sigmoid", bias, groups, 1)
    assert (ids.cpu() == size + torch.arange(k)).all()
