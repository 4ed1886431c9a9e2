"""The norm over many tensors, and their scaling: the norm to its last rounding, the scaled elements to two of fp32 and one of their type."""
import math

import pytest

import layer_reference as ref
from test_gpu_integer_product import DTYPES, torch_type
from test_gpu_integer_product import mad  # noqa: F401

pytestmark = pytest.mark.gpu

# counts of elements of a list of tensors
LISTS = {
    "one element": [1],
    "empty ones": [0, 5, 0, 0, 7, 0],
    "odd sizes": [1, 2, 3, 7, 8, 9, 63, 64, 65, 255, 257, 1000],
    "around a piece": [16383, 16384, 16385, 32768, 32769],
    "large and small": [1 << 22, 3, 100003, 1, 16384 * 40 + 1],
    "as many as a launch takes": [33] * 96,
    "more than a launch takes": [5 + i % 40 for i in range(300)],
    "more pieces than workgroups": [16384 * 2500 + 77, 11],
}


def tensors(counts, types, seed=0, offset=0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    made = []
    for i, n in enumerate(counts):
        dtype = torch_type(types[i % len(types)])
        made.append((torch.randn(n + offset, generator=g, device="cuda") * 10.0 ** (i % 4 - 2)).to(dtype)[offset:])
    return made


def exact_norm(ts):
    return math.sqrt(math.fsum(float((t.double() ** 2).sum()) for t in ts))


def close_to(norm, want):
    # the sum of squares in fp64 is off by 1e-12 of itself, also over 2^26 elements in a row; then one rounding
    assert norm.shape == () and abs(float(norm) - want) <= 1.0001 * ref.U * want + 1e-11 * want, (float(norm), want)


def scaled(got, t, norm, top, dtype):
    factor = min(1.0, top / norm)
    want = t.double() * factor
    most = (0 if factor == 1 else 2.01) * ref.U * want.abs() + ref.HALF[dtype] * want.abs() + ref.TINY[dtype]
    assert bool(((got.double() - want).abs() <= most).all())


@pytest.mark.parametrize("types", [["f32"], ["f16"], ["bf16"], DTYPES], ids=lambda t: "_".join(t))
@pytest.mark.parametrize("name", list(LISTS))
def test_norm_and_clipping(mad, name, types):
    import torch
    counts = LISTS[name]
    print("case clip", name, types, flush=True)
    ts = tensors(counts, types, len(counts), offset=1 if name == "odd sizes" else 0)
    want = exact_norm(ts)
    norm = mad.maddness_gradient_norm(ts)
    close_to(norm, want)
    top = 0.37 * want
    kept = [t.clone() for t in ts]
    # into other tensors, of every type
    outs = [torch.full_like(t, 5.0, dtype=torch_type(DTYPES[i % 3])) for i, t in enumerate(ts)]
    again = mad.maddness_clip_gradients(ts, top, out=outs)
    assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(ts, kept))
    for i, (o, t) in enumerate(zip(outs, ts)):
        scaled(o, t, float(norm), top, DTYPES[i % 3])
    # a norm below the largest: as they are
    mad.maddness_clip_gradients(ts, 1.1 * want, out=outs)
    for i, (o, t) in enumerate(zip(outs, ts)):
        assert torch.equal(o, t.to(o.dtype))
    mad.maddness_clip_gradients(ts, 1.1 * want)
    assert all(torch.equal(a, b) for a, b in zip(ts, kept))
    # in place
    mad.maddness_clip_gradients(ts, top)
    for i, (o, t) in enumerate(zip(ts, kept)):
        scaled(o, t, float(norm), top, types[i % len(types)])


def test_a_norm_that_is_given(mad):
    import torch
    ts = tensors([100, 20000], ["f32", "bf16"])
    kept = [t.clone() for t in ts]
    given = torch.tensor([8.0], device="cuda")
    assert mad.maddness_clip_gradients(ts, 2.0, norm=given) is given and float(given) == 8.0
    assert torch.equal(ts[0], kept[0] * 0.25) and torch.equal(ts[1], kept[1] * 0.25)
    mad.maddness_clip_gradients(ts, 8.0, norm=given)
    assert torch.equal(ts[0], kept[0] * 0.25)
    assert mad.maddness_clip_gradients([], 1.0, norm=given) is given


def test_none_and_empty(mad):
    import torch
    assert float(mad.maddness_gradient_norm([])) == 0
    assert float(mad.maddness_gradient_norm([torch.empty(0, device="cuda")])) == 0
    assert float(mad.maddness_clip_gradients([], 1.0)) == 0
    z = torch.zeros(50, device="cuda")
    assert float(mad.maddness_clip_gradients([z], 0.0)) == 0 and not z.any()
    one = torch.ones(50, device="cuda")
    mad.maddness_clip_gradients([one], 0.0)
    assert not one.any()


def test_numbers_that_are_not_finite(mad):
    """They show in the norm and scale nothing; squares beyond fp32's range, above and below, are no problem."""
    import torch
    for bad in (float("nan"), float("inf"), -float("inf")):
        t = torch.ones(70000, device="cuda")
        t[69999] = bad
        kept = t.clone()
        norm = mad.maddness_clip_gradients([torch.ones(3, device="cuda"), t], 1e-3)
        assert math.isnan(float(norm)) if math.isnan(bad) else float(norm) == math.inf
        assert torch.equal(t.nan_to_num(1.5), kept.nan_to_num(1.5))
    big = torch.full((10000,), 1e30, device="cuda")
    close_to(mad.maddness_gradient_norm([big]), math.sqrt(10000.0) * float(big[0]))
    small = torch.full((10000,), 1e-30, device="cuda")
    close_to(mad.maddness_gradient_norm([small]), math.sqrt(10000.0) * float(small[0]))
    top = torch.full((4,), 3e38, device="cuda")                      # the norm itself is beyond fp32
    assert float(mad.maddness_clip_gradients([top], 1.0)) == math.inf and float(top[0]) == float(torch.tensor(3e38))
    mad.maddness_clip_gradients([big], math.inf)
    assert float(big[0]) == float(torch.tensor(1e30))


def test_orders_of_memory(mad):
    """Tensors that fill their memory in another order are scaled as any; views with gaps are refused."""
    import torch
    t = torch.randn(6, 5, 4, device="cuda").permute(2, 0, 1)
    kept = t.clone()
    norm = mad.maddness_clip_gradients([t], 1.0)
    scaled(t, kept, float(norm), 1.0, "f32")
    out = torch.empty_like(t, dtype=torch.bfloat16)
    assert out.stride() == t.stride()
    mad.maddness_clip_gradients([kept], 1e9, out=[torch.empty_like(kept)])
    mad.maddness_clip_gradients([t], 1e9, out=[out])
    assert torch.equal(out, t.bfloat16())
    for bad in (torch.zeros(4, 6, device="cuda")[:, :5], torch.zeros(10, device="cuda")[::2], torch.zeros(1, device="cuda").expand(5)):
        with pytest.raises(ValueError, match="gaps"):
            mad.maddness_gradient_norm([torch.zeros(3, device="cuda"), bad])


def test_the_same_bits_again(mad):
    import torch
    ts = tensors([500001, 70, 90000], DTYPES)
    first = mad.maddness_gradient_norm(ts)
    assert all(torch.equal(mad.maddness_gradient_norm(ts), first) for _ in range(5))
    # a tensor given twice counts twice
    close_to(mad.maddness_gradient_norm([ts[0], ts[0]]), math.sqrt(2) * exact_norm(ts[:1]))


def test_refusals(mad):
    import torch
    t = torch.ones(8, device="cuda")
    for call in (lambda: mad.maddness_gradient_norm(t), lambda: mad.maddness_gradient_norm([t.cpu()]), lambda: mad.maddness_gradient_norm([t.long()]),
                 lambda: mad.maddness_gradient_norm([t, None])):
        with pytest.raises((TypeError, AttributeError)):
            call()
    with pytest.raises(mad.MaddnessError, match="overlap"):
        mad.maddness_clip_gradients([t, t], 1.0)
    with pytest.raises(mad.MaddnessError, match="overlap"):
        mad.maddness_clip_gradients([t[:5], t[4:]], 1.0)
    with pytest.raises(mad.MaddnessError, match="max_norm"):
        mad.maddness_clip_gradients([t], -1.0)
    with pytest.raises(mad.MaddnessError, match="max_norm"):
        mad.maddness_clip_gradients([t], float("nan"))
    with pytest.raises(ValueError):
        mad.maddness_clip_gradients([t], 1.0, out=[])
    with pytest.raises(ValueError):
        mad.maddness_clip_gradients([t], 1.0, out=[torch.empty(7, device="cuda")])
    with pytest.raises(TypeError):
        mad.maddness_clip_gradients([t], 1.0, norm=torch.ones(1, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        mad.maddness_clip_gradients([t], 1.0, norm=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_clip_gradients([torch.nn.Parameter(t)], 1.0)
    assert float(t.sum()) == 8


def test_the_factor_is_that_of_the_whole_norm(mad):
    """The quotient is formed before the norm is rounded to fp32: an element is off by the factor's rounding and its own."""
    import torch
    for seed in range(24):
        for counts in ([5000, 77], [300000, 12, 4000] + [9] * 10):
            ts = tensors(counts, ["f32"], seed)
            norm = exact_norm(ts)
            outs = [torch.empty_like(t) for t in ts]
            mad.maddness_clip_gradients(ts, 1.0, out=outs)
            for o, t in zip(outs, ts):
                want = t.double() * min(1.0, 1.0 / norm)
                assert bool(((o.double() - want).abs() <= 2.001 * ref.U * want.abs() + 2.0 ** -149).all()), (seed, counts)
    # a norm that is given is taken as it is
    t = torch.full((4,), 3.0, device="cuda")
    mad.maddness_clip_gradients([t], 1.0, norm=torch.tensor(7.0, device="cuda"))
    assert bool((t == 3 * (torch.tensor(1.0, device="cuda") / torch.tensor(7.0, device="cuda"))).all())
