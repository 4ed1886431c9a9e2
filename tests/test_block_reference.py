"""The 64-bit reference of the block format and of the choice of experts against their own definitions (no GPU)."""
import numpy as np
import pytest

import block_reference as ref


def test_levels_round_trip():
    torch = pytest.importorskip("torch")
    bytes_ = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(bytes_).view(torch.float8_e4m3fn).double().numpy()
    got = ref.value(bytes_[None], np.full((1, 2), 127, np.uint8), 1)[0]
    assert np.array_equal(got, want, equal_nan=True)
    fine = ~np.isnan(want)
    assert (ref.e4m3(want[fine]) == bytes_[fine]).all()


@pytest.mark.parametrize("tile", [1, 128])
def test_quantise_takes_the_least_power_of_two(tile):
    rng = np.random.default_rng(tile)
    x = rng.standard_normal((260, 300)) * np.exp(3 * rng.standard_normal((260, 1)))
    x[:, 128:256] *= 448 / np.abs(x[:, 128:256]).max()                     # the largest value of all
    q, e = ref.quantise(x, tile)
    v = ref.value(q, e, tile)
    scale = 2.0 ** (e.astype(int) - 127)[np.arange(260) // tile][:, np.arange(300) // 128]
    assert (np.abs(x) <= 448 * scale).all()
    assert (np.abs(v - x) <= np.maximum(np.abs(x) / 16, scale * 2.0 ** -10)).all()
    for r in range(e.shape[0]):
        for c in range(e.shape[1]):
            assert np.abs(x[r * tile:(r + 1) * tile, c * 128:(c + 1) * 128]).max() > 448 * 2.0 ** (int(e[r, c]) - 128)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_route_gradient_against_differences(kind, renormalise):
    rng = np.random.default_rng(3)
    T, E, k = 5, 9, 3
    x = rng.standard_normal((T, E))
    x[1, 2:5] = -np.inf
    x[2] = -np.inf
    ids, _, _ = ref.route(x, k, kind)
    dw = rng.standard_normal((T, k))
    got = ref.route_gradient(x, ids, dw, kind, renormalise, 2.5)
    h = 1e-6
    for t in range(T):
        for e in range(E):
            if x[t, e] == -np.inf:
                assert got[t, e] == 0
                continue
            up, down = x.copy(), x.copy()
            up[t, e] += h
            down[t, e] -= h
            d = ((ref.weights_of(up, ids, kind, renormalise, 2.5) - ref.weights_of(down, ids, kind, renormalise, 2.5)) * dw).sum() / (2 * h)
            # central differences of a function with derivatives of order 1: h^2 and rounding 2^-52 / h
            assert abs(d - got[t, e]) < 1e-8
