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


def logits_of(seed, T, E, dtype, masked):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((T, E)) * 2).to(dtype)
    if masked:
        x[torch.from_numpy(rng.random((T, E)) < masked)] = float("-inf")
        x[3 % T] = float("-inf")
        x[5 % T] = torch.finfo(dtype).min
        x[6 % T, 0] = float("nan")
        x[7 % T, E - 1] = float("inf")
    return x


# tokens, experts, choices, groups, kept, and the lanes to a token and experts to a lane that they go by
FORMS = [(1100, 100, 6, 1, 1, 16, 8), (1100, 128, 20, 4, 3, 16, 8), (1100, 256, 8, 8, 4, 16, 16), (1100, 200, 8, 5, 2, 16, 16), (1100, 256, 20, 1, 1, 16, 16),
         (1027, 250, 32, 10, 7, 16, 16), (40, 16, 16, 1, 1, 16, 1), (40, 32, 32, 4, 4, 16, 2), (1100, 64, 30, 16, 9, 16, 4), (1100, 256, 8, 32, 9, 64, 4),
         (1100, 300, 20, 1, 1, 64, 8), (1100, 768, 8, 8, 3, 64, 16), (70, 900, 24, 30, 11, 64, 16)]


@pytest.mark.parametrize("T,E,k,groups,kept,lanes,each", FORMS)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_route_in_every_form(mad, T, E, k, groups, kept, lanes, each, kind, dtype):
    import torch
    print("case route", T, E, k, groups, kept, kind, dtype, flush=True)
    rng = np.random.default_rng(E)
    for masked, bias, renormalise in ((0, None, True), (0.3, rng.standard_normal(E).astype(np.float32) * 0.1, False)):
        x = logits_of(T * E + k, T, E, getattr(torch, dtype), masked)
        with np.errstate(invalid="ignore"):
            want, w, gap = ref.route(x.double().numpy(), k, kind, bias, groups, kept, renormalise, 1.5)
        ids, weights = mad.maddness_route(x.cuda(), k, kind, None if bias is None else torch.from_numpy(bias).cuda(), groups, kept, renormalise, 1.5)
        kernel = mad.maddness_last_kernel()
        assert kernel.startswith("route_kernel") and f"LANES = {lanes}, R = {each}]" in kernel, kernel
        ids, weights = ids.cpu().numpy(), weights.double().cpu().numpy()
        # keys are sums of a score of at most 1 (error of a few 2^-24) and a bias, group values of two keys: choices further apart are the same
        sure = (gap > 32 * 2.0 ** -24) | (gap == np.inf)
        assert sure.sum() > 8
        assert (ids[sure] == want[sure]).all()
        # 2^-24 for the exponential's argument of up to 16 and its value, the sums of up to k, two divisions, the factor
        assert (np.abs(weights - w)[sure] <= 64 * 2.0 ** -24 * np.abs(w[sure]) + 1e-37).all()
        # a choice that was too close to compare: experts that are there, each once, with their own scores in place
        s, seen = ref.scores(x.double().numpy(), kind)
        for t in np.flatnonzero(~sure):
            there = ids[t][ids[t] >= 0]
            assert len(set(there)) == len(there) and seen[t, there].all()
            if not renormalise:
                assert (np.abs(weights[t][ids[t] >= 0] - 1.5 * s[t, there]) <= 64 * 2.0 ** -24 * 1.5 * s[t, there] + 1e-37).all()


@pytest.mark.parametrize("T,E,k,groups,kept,lanes,each", FORMS)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_route_gradient_in_every_form(mad, T, E, k, groups, kept, lanes, each, kind, renormalise, dtype):
    import torch
    if groups > 16 and E <= 256:
        lanes, each = 16, 16                               # (the gradient knows no groups)
    print("case route gradient", T, E, k, kind, renormalise, dtype, flush=True)
    rng = np.random.default_rng(E + k)
    x = logits_of(E + T, T, E, getattr(torch, dtype), 0.2)
    ids = rng.integers(-1, E, (T, k)).astype(np.int32)                    # any: the same twice, none, and beyond
    ids[1, 0], ids[2, k - 1] = E, -7
    dw = rng.standard_normal((T, k)).astype(np.float32)
    x64 = x.double().numpy()
    with np.errstate(invalid="ignore"):
        want = ref.route_gradient(x64, ids, dw.astype(np.float64), kind, renormalise, 2.0)
        s, _ = ref.scores(x64, kind)
    wide = torch.zeros(T, E + 3, dtype=x.dtype, device="cuda")
    wide[:, 1:E + 1] = x.cuda()
    for place in (x.cuda(), wide[:, 1:E + 1]):                            # in whole runs, and one by one
        got = mad.maddness_route_gradient(place, torch.from_numpy(ids).cuda(), torch.from_numpy(dw).cuda(), kind, renormalise, 2.0)
        kernel = mad.maddness_last_kernel()
        assert kernel.startswith("route_gradient_kernel") and f"LANES = {lanes}, R = {each}]" in kernel, kernel
        got = got.double().cpu().numpy()
        # every term is at most factor |dw| s / total (renormalised; total >= the s itself) and carries some 64 roundings of 2^-24, k of them in
        # sums; one rounding to the scores' type
        there = (ids >= 0) & (ids < E)
        mine = np.where(there, np.take_along_axis(s, np.clip(ids, 0, E - 1), 1), 0)
        total = np.maximum(mine.sum(1, keepdims=True), 1e-30) if renormalise else 1.0
        size = (np.abs(dw) * there).max(1, keepdims=True) * 2.0 * 2 * k
        unit, least = {"float32": (0, 1e-36), "bfloat16": (2.0 ** -8, 1e-36), "float16": (2.0 ** -11, 2.0 ** -25)}[dtype]
        tol = (64 + k) * 2.0 ** -24 * size * s / total + 1.01 * unit * np.abs(want) + least
        assert (np.abs(got - want) <= tol).all()
