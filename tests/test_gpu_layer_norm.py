"""The layer norm, its integers and its gradient, within what fp32 sums and roundings may change."""
import numpy as np
import pytest

import layer_reference as ref
from test_gpu_integer_product import DTYPES, activations, check, dev, host, torch_type
from test_gpu_integer_product import mad  # noqa: F401

pytestmark = pytest.mark.gpu

# (rows, cols, elements between rows, before the first)
CASES = [(1, 1, 0, 0), (4, 2, 0, 1), (3, 7, 1, 0), (5, 8, 0, 0), (4, 9, 1, 1), (1, 64, 0, 0), (2, 65, 3, 1), (300, 510, 0, 0), (9, 512, 0, 1), (6, 513, 0, 0), (4099, 37, 0, 0), (5, 1000, 0, 3),
         (9, 1024, 0, 0), (5, 1025, 0, 0), (4, 2048, 0, 0), (3, 2049, 1, 0), (8, 4096, 0, 0), (1030, 4090, 0, 0), (3, 4104, 0, 1), (3, 8192, 0, 0), (2, 8195, 0, 0), (3, 16384, 0, 0),
         (2, 16385, 0, 1), (70, 33000, 0, 0)]


def depth_of(cols):
    """Additions on the way of an element to its row's sum: the 32 of a lane at most, or a 1024th of a long row, and 6 + 15 between lanes and wavefronts."""
    return max(32, -(-cols // 1024)) + 21


def row_depth(mad, rows, cols):
    """And of a row to the sums over rows: what a workgroup takes in turn, its four wavefronts, and the workgroups'."""
    parts = max(1, mad.lib().maddness_layer_norm_gradient_workspace(rows, cols) // (8 * cols))
    return -(-rows // parts) + 4 + -(-parts // 16) + 16


def parameters(rng, cols, dtype):
    import torch
    w = torch.from_numpy(1 + 0.3 * rng.normal(size=cols)).to(torch_type(dtype)).cuda()
    b = torch.from_numpy(0.5 * rng.normal(size=cols)).to(torch_type(dtype)).cuda()
    return w, b


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%dx%d_p%d_o%d" % c)
def test_layer_norm_and_gradient(mad, case, dtype):
    import torch
    rows, cols, pad, before = case
    print("case norm", case, dtype, flush=True)
    rng = np.random.default_rng(rows + 5 * cols)
    x = activations(rng, rows, cols) + 2 * rng.normal(size=(rows, 1))
    if rows > 2:
        x[1] = 3.25                                    # a row of equal numbers
    x_d = dev(x, dtype, pad, before)
    kinds = dict(zip(DTYPES, ("f32", "f16", "bf16")))
    other = DTYPES[(DTYPES.index(dtype) + 1) % 3]
    eps = 1e-3
    xh = host(x_d)
    for parameter_type, out_type in ((None, dtype), ("f32", dtype), (kinds[dtype], other)):
        w, b = parameters(rng, cols, parameter_type) if parameter_type else (None, None)
        wh, bh = (host(w), host(b)) if parameter_type else (None, None)
        y, mean, rstd = mad.maddness_layer_norm(x_d, w, b, eps=eps, training=True, out_dtype=torch_type(out_type))
        want, mean_w, rstd_w, e_y, e_mean, e_r = ref.norm(xh, wh, bh, eps, depth_of(cols))
        assert y.dtype is torch_type(out_type) and (np.abs(host(mean) - mean_w) <= e_mean).all() and (np.abs(host(rstd) - rstd_w) <= e_r).all()
        check(y, want, e_y, out_type, (case, dtype, parameter_type))
        assert torch.equal(mad.maddness_layer_norm(x_d, w, b, eps=eps, out_dtype=torch_type(out_type)), y)
        # the gradient, from a gradient of another type and stride
        g_d = dev(rng.normal(size=(rows, cols)) * 0.1, out_type, 1 - pad % 2, 1 - before % 2)
        dx, dw, db = mad.maddness_layer_norm_gradient(g_d, x_d, mean, rstd, w, parameters=True)
        want_dx, want_dw, want_db, e_dx, e_dw, e_db = ref.norm_gradient(host(g_d), xh, host(mean), host(rstd), wh, depth_of(cols), row_depth(mad, rows, cols))
        assert dx.dtype is x_d.dtype and dw.dtype is torch.float32
        check(dx, want_dx, e_dx, dtype, (case, dtype, "dx"))
        check(dw, want_dw, e_dw, "f32", (case, dtype, "dweight"))
        check(db, want_db, e_db, "f32", (case, dtype, "dbias"))
        alone = mad.maddness_layer_norm_gradient(g_d, x_d, mean, rstd, w, parameters=False)
        assert torch.equal(alone[0], dx) and alone[1] is None and alone[2] is None


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", [(1, 5, 0, 0), (3, 8, 0, 0), (5, 70, 1, 1), (130, 510, 0, 0), (4, 1000, 0, 0), (3, 2000, 0, 1), (8, 4096, 0, 0), (2, 8001, 0, 0), (2, 16000, 0, 0), (2, 17000, 0, 0)],
                         ids=lambda c: "%dx%d_p%d_o%d" % c)
def test_layer_norm_to_integers(mad, case, dtype):
    """Integers of the fp32 result: equal to those of the call that returns it, which differs by roundings of fp32 only."""
    import torch
    rows, cols, pad, before = case
    print("case norm to integers", case, dtype, flush=True)
    rng = np.random.default_rng(rows + cols)
    x_d = dev(activations(rng, rows, cols), dtype, pad, before)
    w, b = parameters(rng, cols, "f32")
    got, mean, rstd = mad.maddness_layer_norm(x_d, w, b, training=True, integer=True)
    y, mean2, rstd2 = mad.maddness_layer_norm(x_d, w, b, training=True, out_dtype=torch.float32)
    assert torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    only = mad.maddness_layer_norm(x_d, w, b, integer=True)
    assert torch.equal(only.q, got.q) and torch.equal(only.scale, got.scale)
    want, _, _, e_y, _, _ = ref.norm(host(x_d), host(w), host(b), 1e-5, depth_of(cols))
    again = mad.maddness_quantise_rows(y)
    assert torch.equal(again.q, got.q) and torch.equal(again.scale, got.scale)
    q, scale = ref.quantise(host(y))
    e_scale = e_y.max(1) / 127 + 2 * ref.U * scale
    assert (np.abs(host(got.scale) - np.abs(want).max(1) / 127) <= e_scale).all()
    # what the integers stand for is half a step from the exact result at most, beside what that and the step are off by
    off = np.abs(host(got.q) * host(got.scale)[:, None] - want)
    assert (off <= 0.5 * host(got.scale)[:, None] * (1 + 1e-6) + e_y).all()
    padded = torch.as_strided(got.q, (rows, got.q.stride(0)), (got.q.stride(0), 1))
    assert not padded[:, cols:].any()


def test_statistics_of_rows_far_from_zero(mad):
    """A mean 4000 times the deviation: the variance is that of the centred values."""
    import torch
    rng = np.random.default_rng(2)
    x = (4000 + rng.normal(size=(40, 700))).astype(np.float32)
    y, mean, rstd = mad.maddness_layer_norm(torch.from_numpy(x).cuda(), eps=0.0, training=True)
    want, mean_w, rstd_w, e_y, e_mean, e_r = ref.norm(x, None, None, 0.0, depth_of(700))
    # the bound says something: half of the mean's (55 U 4000)^2 = 1.72e-4 over the smallest variance of 0.897, and 4e-6 beside it, is 1.02e-4; squares of the
    # values themselves would leave the variance off by 4000^2 U = 0.95
    assert e_r.max() < 1.2e-4 * rstd_w.max()
    check(y, want, e_y, "f32")
    assert (np.abs(host(rstd) - rstd_w) <= e_r).all()


def test_rows_that_are_not_finite_stay_alone(mad):
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(9, 600, generator=g, device="cuda")
    want, mean, rstd = mad.maddness_layer_norm(x, training=True)
    bad = x.clone()
    bad[2, 5], bad[4, 0], bad[7, 599] = float("nan"), float("inf"), -float("inf")
    y, _, _ = mad.maddness_layer_norm(bad, training=True)
    good = [0, 1, 3, 5, 6, 8]
    assert torch.equal(y[good], want[good]) and not y[[2, 4, 7]].isfinite().any()
    q = mad.maddness_layer_norm(bad, integer=True)
    assert bool(q.scale[[2, 4, 7]].isnan().all()) and not q.scale[good].isnan().any()
    grad = torch.randn(9, 600, generator=g, device="cuda")
    dx, _, _ = mad.maddness_layer_norm_gradient(grad, x, mean, rstd)
    grad[3, 3] = float("nan")
    dx2, _, _ = mad.maddness_layer_norm_gradient(grad, x, mean, rstd)
    keep = [0, 1, 2, 4, 5, 6, 7, 8]
    assert torch.equal(dx2[keep], dx[keep]) and bool(dx2[3].isnan().all())


def test_no_rows(mad):
    import torch
    x = torch.zeros((0, 48), device="cuda")
    w = torch.ones(48, device="cuda")
    y, mean, rstd = mad.maddness_layer_norm(x, w, w, training=True)
    assert y.shape == (0, 48) and mean.shape == (0,)
    dx, dw, db = mad.maddness_layer_norm_gradient(y, x, mean, rstd, w)
    assert dx.shape == (0, 48) and not dw.any() and not db.any() and dw.shape == (48,)
    assert mad.maddness_layer_norm(x, integer=True).shape == (0, 48)


def test_rows_are_written_once_and_nothing_else(mad):
    import torch
    x = torch.randn(33, 700, device="cuda")
    wide = torch.full((33, 720), -7.0, device="cuda")
    got = mad.maddness_layer_norm(x, out=wide[:, 5:705])
    assert got.data_ptr() == wide[:, 5:705].data_ptr() and torch.equal(got, mad.maddness_layer_norm(x))
    assert bool((wide[:, :5] == -7).all()) and bool((wide[:, 705:] == -7).all())


def test_refusals(mad):
    import torch
    x, w = torch.ones((3, 32), device="cuda"), torch.ones(32, device="cuda")
    y, mean, rstd = mad.maddness_layer_norm(x, w, training=True)
    for kw in (dict(weight=w[:31]), dict(weight=torch.ones(64, device="cuda")[::2]), dict(bias=w.reshape(1, 32)), dict(integer=True, out=x.clone()), dict(integer=True, out_dtype=torch.float32),
               dict(out=torch.empty((3, 31), device="cuda")), dict(out=x.clone(), out_dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            mad.maddness_layer_norm(x, **kw)
    for kw in (dict(weight=w, bias=w.half()), dict(weight=w.double()), dict(out_dtype=torch.int8)):
        with pytest.raises(TypeError):
            mad.maddness_layer_norm(x, **kw)
    for kw in (dict(eps=-1.0), dict(eps=float("nan"))):
        with pytest.raises(mad.MaddnessError):
            mad.maddness_layer_norm(x, **kw)
    with pytest.raises(mad.MaddnessError, match="mean"):
        mad.maddness_layer_norm(torch.ones((3, 0), device="cuda"))
    with pytest.raises(ValueError):
        mad.maddness_layer_norm_gradient(y[:2], x, mean, rstd)
    with pytest.raises(ValueError):
        mad.maddness_layer_norm_gradient(y, x, mean[:2], rstd)
    with pytest.raises(TypeError):
        mad.maddness_layer_norm_gradient(y, x, mean.double(), rstd)
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_layer_norm(x.clone().requires_grad_())
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_layer_norm(x, torch.nn.Parameter(w))
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_layer_norm_gradient(y, x, mean, rstd, torch.nn.Parameter(w))


@pytest.mark.parametrize("cols", [8, 100, 510, 700, 1000, 1023, 1500, 2049, 4096, 4095, 5000, 8191, 12345, 16384, 20000])
def test_rows_of_one_number(mad, cols):
    """Their sum is exact (4000 = 125 * 2^5, and sums below 2^29), so the mean is the number, the norm the bias, and a gradient of one number centres to nothing."""
    import torch
    x = torch.full((5, cols), 4000.0, device="cuda")
    b = torch.linspace(-1, 1, cols, device="cuda")
    y, mean, rstd = mad.maddness_layer_norm(x, torch.full_like(b, 3.0), b, training=True)
    assert bool((mean == 4000).all()) and torch.equal(y, b.expand(5, cols))
    assert bool((rstd == rstd[0]).all()) and abs(float(rstd[0]) * 1e-5 ** 0.5 - 1) < 4 * ref.U
    dx, dw, db = mad.maddness_layer_norm_gradient(x, x, mean, rstd, parameters=True)
    assert not dx.any() and not dw.any() and bool((db == 20000).all())


@pytest.mark.parametrize("size", [(1 << 21, 7), (20000, 16400), (3000, 540000)], ids=lambda c: "%dx%d" % c)
def test_sums_over_many_rows_of_any_length(mad, size):
    """Lengths whose sums over rows are taken a column to a thread: hundreds or thousands of rows to each, added in fp64, so that only the
    parts' sum is left to fp32."""
    import torch
    rows, cols = size
    print("case many rows", size, flush=True)
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, generator=g, device="cuda", dtype=torch.bfloat16 if cols > 7 else torch.float32)
    grad = torch.full((rows, cols), 1.1, device="cuda")
    x[:, 3] = 2.5                                              # (a column whose h hardly changes: all of its terms have one sign)
    _, mean, rstd = mad.maddness_layer_norm(x, training=True)
    _, dw, db = mad.maddness_layer_norm_gradient(grad, x, mean, rstd, parameters=True)
    parts = mad.lib().maddness_layer_norm_gradient_workspace(rows, cols) // (8 * cols)
    assert rows // parts > 100
    depth = -(-parts // 32) + 18                               # additions of a part, and its own rounding
    keep = torch.arange(0, cols, max(1, cols // 1000), device="cuda").unique()
    keep = torch.cat([keep, torch.tensor([3, cols - 1], device="cuda")])
    h = (x[:, keep].double() - mean.double().unsqueeze(1)) * rstd.double().unsqueeze(1)
    gk = grad[:, keep].double()
    want_w, size_w, want_b = (gk * h).sum(0), (gk * h).abs().sum(0), gk.sum(0)
    # h is rounded twice
    assert bool(((dw[keep].double() - want_w).abs() <= 1.01 * (depth + 2) * ref.U * size_w).all())
    assert bool(((db[keep].double() - want_b).abs() <= 1.01 * depth * ref.U * want_b).all())


def test_sums_of_a_long_row(mad):
    """Four million numbers: 4096 to a thread, added in fp64, so that mean and deviation are off by their last roundings only."""
    import torch
    cols, U = 1 << 22, ref.U
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(2, cols, generator=g, device="cuda") + 3.7
    y, mean, rstd = mad.maddness_layer_norm(x, training=True)
    mean_w = x.double().mean(1)
    assert bool(((mean.double() - mean_w).abs() <= 1.01 * U * mean_w.abs()).all())
    d = x.double() - mean.double().unsqueeze(1)
    r = 1 / torch.sqrt((d * d).mean(1) + 1e-5)
    # centred values are rounded (2 U in their squares), the variance and its sum with eps too: half of 4 U in the root, which is rounded, as the quotient is
    assert bool(((rstd.double() - r).abs() <= 1.01 * 4 * U * r).all())
    grad = 1.1 + 0.1 * torch.randn(2, cols, generator=g, device="cuda")
    dx, _, _ = mad.maddness_layer_norm_gradient(grad, x, mean, rstd, parameters=False)
    h = d * rstd.double().unsqueeze(1)
    u = grad.double()
    su, suh = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    want = rstd.double().unsqueeze(1) * (u - su - h * suh)
    # su to one rounding; h to two, in suh (once more rounded) and beside it; u - su and the sum one each, the factor one
    parts = u.abs() + su.abs() + (h * suh).abs()
    most = 1.01 * rstd.double().unsqueeze(1) * U * (su.abs() + h.abs() * 3 * (u * h).abs().mean(1, keepdim=True) + 2 * (h * suh).abs() + 3 * parts)
    assert bool(((dx.double() - want).abs() <= most + U * want.abs()).all())
