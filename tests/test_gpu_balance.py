"""The balance of experts: counts, loss and gradient, within what fp32 scores and sums may change."""
import math

import numpy as np
import pytest

import layer_reference as ref
from test_gpu_integer_product import DTYPES, check, dev, host, torch_type
from test_gpu_integer_product import mad  # noqa: F401

pytestmark = pytest.mark.gpu

U = ref.U
# (tokens, experts, k, elements between rows, before the first)
CASES = [(0, 4, 1, 0, 0), (1, 1, 1, 0, 0), (1, 8, 2, 0, 0), (3, 5, 2, 1, 1), (64, 16, 2, 0, 0), (33, 64, 8, 4, 4), (130, 60, 4, 0, 1), (511, 65, 3, 0, 0), (1000, 100, 6, 0, 0), (77, 256, 8, 0, 0), (5000, 8, 2, 0, 0),
         (40, 257, 8, 0, 0), (300, 1000, 5, 3, 1), (65, 1024, 32, 0, 0), (20000, 31, 4, 0, 0), (9000, 256, 8, 0, 0)]


def problem(case, dtype, masked):
    T, E, k, pad, before = case
    rng = np.random.default_rng(T + 3 * E + k)
    x = rng.normal(size=(T, E)) * 2 + rng.normal(size=E)
    if masked:
        x[rng.random((T, E)) < 0.2] = -np.inf
        x[rng.random(T) < 0.1] = -np.inf
        x[rng.random((T, E)) < 0.002] = np.nan
    logits = dev(x, dtype, pad, before)
    best, ids = logits.float().nan_to_num(nan=-np.inf).topk(k, -1)
    import torch
    ids = torch.where(best > -np.inf, ids, -1).to(torch.int32).contiguous()
    if T > 3:
        ids[2, 0] = E + 5                                 # nobody's
    return logits, ids


def depth_of(T, E):
    """Additions on the way of a token to the fp32 sums: what a lane takes in turn (a chip has 256 compute units or fewer), 2 between groups of lanes, 8
    wavefronts."""
    return -(-T // (8 * (4 if E <= 64 else 1) * 64)) + 10


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "T%d_E%d_k%d_p%d_o%d" % c)
def test_balance_and_gradient(mad, case, masked, kind):
    import torch
    T, E, k, pad, before = case
    print("case balance", case, masked, kind, flush=True)
    for dtype in DTYPES:
        logits, ids = problem(case, dtype, masked)
        factor = 0.25
        loss, counts, push = mad.maddness_balance(logits, ids, scores=kind, factor=factor)
        x, i = host(logits), ids.cpu().numpy()
        want, counts_w, push_w, p, s, seen, rel = ref.balance(x, i, kind, factor)
        assert loss.shape == () and counts.dtype is torch.int32
        assert np.array_equal(counts.cpu().numpy(), counts_w)
        assert (np.abs(host(push) - push_w) <= 1.01 * U * push_w).all()
        # a share is off by its score's part, the sum's (16 to a lane, 6 between lanes, and its terms' own), a division and a product
        rel_p = rel + rel.max(1, keepdims=True, initial=0.0) + 24 * U
        e_loss = ((rel_p * p).sum(0) * push_w).sum() + (depth_of(T, E) + 4) * U * want + 2.0 ** -149
        assert abs(float(loss) - want) <= 1.01 * e_loss, (float(loss), want)
        times = torch.tensor([3.0], device="cuda")
        got = mad.maddness_balance_gradient(logits, push, scores=kind)
        d = ref.balance_gradient(p, s, seen, host(push), kind)
        dot = (p * host(push)).sum(1, keepdims=True)
        e_dot = (p * host(push) * (rel_p + 26 * U)).sum(1, keepdims=True)
        slope = (1 - s) if kind == "sigmoid" else np.ones_like(s)
        apart = np.abs(host(push) - dot)
        bound = 1.01 * (p * (slope * (rel_p * apart + e_dot + 6 * U * (apart + host(push) + dot)) + apart * (rel * s + U if kind == "sigmoid" else 0))) + 2.0 ** -148
        check(got, d, bound, dtype, (case, dtype, kind))
        assert got.dtype is logits.dtype and not got[torch.from_numpy(~seen).cuda()].any()
        # times a gradient of the loss, plus what is there already, into its place
        add = dev(np.random.default_rng(1).normal(size=(T, E)) * 1e-3, dtype, pad, 0)
        add_h = host(add)
        thrice = mad.maddness_balance_gradient(logits, push, scores=kind, loss_gradient=times, add=add, out=add)
        assert thrice.data_ptr() == add.data_ptr()
        total = 3 * d + add_h
        check(thrice, total, 3 * bound + U * (3 * np.abs(d) + 3 * bound) + U * np.abs(total), dtype, (case, dtype, kind, "add"))
        again = mad.maddness_balance(logits, ids, scores=kind, factor=factor)
        assert torch.equal(again[0], loss) and torch.equal(again[2], push)


def test_even_and_uneven(mad):
    import torch
    logits = torch.zeros((64, 8), device="cuda")
    even = (torch.arange(64, device="cuda") % 8).to(torch.int32).reshape(-1, 1)
    assert float(mad.maddness_balance(logits, even, factor=0.5)[0]) == 0.5
    assert float(mad.maddness_balance(logits, torch.zeros_like(even), factor=0.5)[0]) == 0.5
    logits[:, 0] = 100.0
    assert abs(float(mad.maddness_balance(logits, torch.zeros_like(even), factor=0.5)[0]) - 4.0) < 1e-6


def test_no_token_counts(mad):
    """Only padding: no loss, no gradient, nothing that is not a number."""
    import torch
    logits = torch.full((40, 16), -float("inf"), device="cuda")
    ids = torch.full((40, 2), -1, dtype=torch.int32, device="cuda")
    for kind in ("softmax", "sigmoid"):
        loss, counts, push = mad.maddness_balance(logits, ids, scores=kind)
        assert float(loss) == 0 and not counts.any() and not push.any()
        assert not mad.maddness_balance_gradient(logits, push, scores=kind).any()
    # tokens without a choice, and choices of tokens that do not count
    loss, counts, push = mad.maddness_balance(torch.zeros((40, 16), device="cuda"), ids)
    assert float(loss) == 0
    loss, counts, push = mad.maddness_balance(logits, torch.zeros_like(ids))
    assert float(loss) == 0 and int(counts[0]) == 80 and not push.any()


def test_large_logits(mad):
    """Plus infinity counts as the largest number; scores that are 0 to fp32 leave a token out."""
    import torch
    logits = torch.zeros((3, 4), device="cuda")
    logits[0, 1] = float("inf")
    logits[1, 2] = 1e30
    ids = torch.tensor([[1], [2], [0]], dtype=torch.int32, device="cuda")
    loss, counts, push = mad.maddness_balance(logits, ids)
    want = 4 / 9 * (0.25 + 1.25 + 1.25)
    assert abs(float(loss) - want) < 1e-6 and mad.maddness_balance_gradient(logits, push).isfinite().all()
    dead = torch.full((5, 4), -200.0, device="cuda")
    assert float(mad.maddness_balance(dead, ids.new_zeros((5, 1)), scores="sigmoid")[0]) == 0


def test_the_routes_choices(mad):
    """Beside the choice of experts, with whose counts it agrees."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    logits = torch.randn(700, 48, generator=g, device="cuda")
    logits[5] = -float("inf")
    ids, _ = mad.maddness_route(logits, 4)
    _, counts, _ = mad.maddness_balance(logits, ids)
    assert torch.equal(counts, mad.maddness_order(ids, 48)[1])


def test_refusals(mad):
    import torch
    logits = torch.zeros((6, 8), device="cuda")
    ids = torch.zeros((6, 2), dtype=torch.int32, device="cuda")
    _, _, push = mad.maddness_balance(logits, ids)
    for bad in ((logits, ids[:5]), (logits, ids[:, 0]), (logits.t(), ids), (logits, ids.t().contiguous().t()), (logits, ids[:, :0])):
        with pytest.raises(ValueError):
            mad.maddness_balance(*bad)
    with pytest.raises(TypeError):
        mad.maddness_balance(logits, ids.long())
    with pytest.raises(TypeError):
        mad.maddness_balance(logits.double(), ids)
    with pytest.raises(ValueError):
        mad.maddness_balance(logits, ids, scores="tanh")
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_balance(logits.clone().requires_grad_(), ids)
    with pytest.raises(mad.MaddnessError):
        mad.maddness_balance(torch.zeros((2, 1025), device="cuda"), ids[:2])
    with pytest.raises(ValueError):
        mad.maddness_balance_gradient(logits, push[:7])
    with pytest.raises(ValueError):
        mad.maddness_balance_gradient(logits, push, add=logits.half())
    with pytest.raises(ValueError):
        mad.maddness_balance_gradient(logits, push, out=logits[:5].clone())
    with pytest.raises(ValueError):
        mad.maddness_balance_gradient(logits, push, loss_gradient=torch.ones(2, device="cuda"))
    with pytest.raises(ValueError, match="gradient"):
        mad.maddness_balance_gradient(logits, push.clone().requires_grad_())


LEAST = -126 * math.log(2.0)                              # a sigmoid of 2^-126, below which it is 0


def far_logits(dtype):
    """Every 16-bit number between -140 and -80, or a sweep of fp32 ones; none as near to LEAST as fp32 scores are off."""
    import torch
    if dtype == "f32":
        x = np.linspace(-140, -80, 6001).astype(np.float32).astype(np.float64)
    else:
        x = host(torch.arange(-32768, 32768).to(torch.int16).cuda().view(torch_type(dtype)))
    return x[(x >= -140) & (x <= -80) & (np.abs(x - LEAST) > 1e-4)]


def check_sigmoid(mad, logits, ids, what):
    """Loss, counts, push and gradient against 64 bits, in which a score below 2^-126 is 0 too; returns the scores' shares, the loss and its bound."""
    factor, (T, E) = 0.25, logits.shape
    x, i = host(logits), ids.cpu().numpy()
    s, seen, rel = ref.scores(x, "sigmoid")
    s = np.where(s < 2.0 ** -126, 0.0, s)
    total = s.sum(1, keepdims=True)
    p = np.divide(s, total, out=np.zeros_like(s), where=total > 0)
    counts_w = np.bincount(i[(i >= 0) & (i < E)].ravel(), minlength=E)
    push_w = factor * E * counts_w / (counts_w.sum() * int((total > 0).sum()))
    want = float((push_w * p.sum(0)).sum())
    loss, counts, push = mad.maddness_balance(logits, ids, scores="sigmoid", factor=factor)
    assert np.array_equal(counts.cpu().numpy(), counts_w)
    push_h = host(push)
    assert (np.abs(push_h - push_w) <= 1.01 * U * push_w).all(), what
    # bounds as above; shares may be so small that they lose half a step of fp32's subnormal numbers
    rel_p = rel + rel.max(1, keepdims=True) + 24 * U
    e_loss = 1.01 * (((rel_p * p).sum(0) * push_w).sum() + (depth_of(T, E) + 4) * U * want + 2.0 ** -149 * T * push_w.sum()) + 2.0 ** -149
    assert abs(float(loss) - want) <= e_loss, (what, float(loss), want)
    d = ref.balance_gradient(p, s, seen, push_h, "sigmoid")
    dot = (p * push_h).sum(1, keepdims=True)
    e_dot = (p * push_h * (rel_p + 26 * U)).sum(1, keepdims=True)
    apart = np.abs(push_h - dot)
    bound = 1.01 * p * ((1 - s) * (rel_p * apart + e_dot + 6 * U * (apart + push_h + dot)) + apart * (rel * s + U)) + 2.0 ** -148
    for dtype in DTYPES:
        if logits.dtype is torch_type(dtype):
            check(mad.maddness_balance_gradient(logits, push, scores="sigmoid"), d, bound, dtype, what)
    return s, push_w, want, e_loss


# (tokens, experts): every split of a token's experts over lanes, by one workgroup and by many
@pytest.mark.parametrize("size", [(2048, 8), (512, 60), (128, 200), (32, 600), (4099, 8), (4099, 60), (4099, 200), (2051, 600)], ids=lambda c: "T%d_E%d" % c)
def test_sigmoids_that_vanish(mad, size):
    """Finite logits whose exponential has no number in fp32: alone among ordinary ones, half of a token's, all of them (such a token counts nowhere);
    and tokens that have only scores next to the smallest."""
    import torch
    T, E = size
    print("case far sigmoids", size, flush=True)
    for dtype in DTYPES:
        rng = np.random.default_rng(T + E)
        far = far_logits(dtype)
        x = rng.normal(size=(T, E)) * 2
        x[np.arange(0, T, 4), rng.integers(0, E, size=-(-T // 4))] = far[np.arange(-(-T // 4)) % len(far)]
        half = x[1::4]
        half[:] = np.where(rng.random(half.shape) < 0.5, rng.choice(far, half.shape), half)
        x[2::4] = rng.choice(far[far < LEAST], x[2::4].shape)
        x[3::4] = rng.choice(far[far > LEAST], x[3::4].shape)
        logits = dev(x, dtype)
        ids = logits.float().topk(2, -1)[1].to(torch.int32).contiguous()
        check_sigmoid(mad, logits, ids, (size, dtype))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_sigmoids_of_every_logit(mad, dtype):
    """All 65536 numbers of a type, each beside ordinary logits; the scores are those of the choice of experts."""
    import torch
    E = 8
    print("case every sigmoid", dtype, flush=True)
    every = torch.arange(-32768, 32768).to(torch.int16).cuda().view(torch_type(dtype))
    logits = dev(np.random.default_rng(8).normal(size=(65536, E)), dtype)
    logits[torch.arange(65536, device="cuda"), torch.arange(65536, device="cuda") % E] = every
    ids, scores = mad.maddness_route(logits, E, scores="sigmoid", renormalise=False)
    s, push, want, e_loss = check_sigmoid(mad, logits, ids[:, :2].contiguous(), dtype)
    route = np.zeros(s.shape)
    rows, slots = np.nonzero(ids.cpu().numpy() >= 0)
    route[rows, ids.cpu().numpy()[rows, slots]] = host(scores)[rows, slots]
    assert (np.abs(route - s) <= 8 * U * s + 2.0 ** -126).all()
    loss = ((route / route.sum(1, keepdims=True)).sum(0) * push).sum()
    assert abs(loss - want) <= e_loss


def test_slopes_of_large_logits(mad):
    """A sigmoid's slope keeps its digits where the score is next to 1: 1 - s is made of the exponential, not of s."""
    import torch
    T, E = 2400, 8
    rng = np.random.default_rng(12)
    x = rng.normal(size=(T, E))
    x[np.arange(T), np.arange(T) % E] = np.linspace(-20, 100, T)
    x[5::50] = rng.random((T // 50, E)) * 40
    logits = dev(x)
    ids = logits.topk(2, -1)[1].to(torch.int32).contiguous()
    push = host(mad.maddness_balance(logits, ids, scores="sigmoid")[2])
    got = host(mad.maddness_balance_gradient(logits, mad.maddness_balance(logits, ids, scores="sigmoid")[2], scores="sigmoid"))
    x = host(logits)
    _, _, _, p, s, seen, rel = ref.balance(x, ids.cpu().numpy(), "sigmoid", 1.0)
    slope = 1 / (1 + np.exp(x))
    dot = (p * push).sum(1, keepdims=True)
    rel_p = rel + rel.max(1, keepdims=True) + 24 * U
    e_dot = (p * push * (rel_p + 26 * U)).sum(1, keepdims=True)
    apart = np.abs(push - dot)
    # the slope: an exponential of 4 U, a score of 8 and a product; one below 2^-126 may be 0
    bound = 1.01 * p * slope * (rel_p * apart + e_dot + 6 * U * (apart + push + dot) + 14 * U * apart) + p * apart * 2.0 ** -126 + 2.0 ** -148
    off = np.abs(got - p * slope * (push - dot))
    assert (off <= bound + ref.rounding(got, "f32")).all(), float((off / bound).max())
