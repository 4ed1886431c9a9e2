"""The layer of experts in each type, forward and backward, against the same steps in 64 bits on the values that were rounded."""
import numpy as np
import pytest

import block_reference as ref

pytestmark = pytest.mark.gpu

UNIT = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
LEAST = {"float32": 2.0 ** -150, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}


@pytest.fixture(scope="module")
def mad():
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def back(v):
    """Rows as they are after their rounding, and their magnitudes where those below 2^-6 of their power of two count as that much."""
    q, e = ref.quantise(v, 1)
    r = ref.value(q, e, 1)
    return r, np.maximum(np.abs(r), 2.0 ** (e.astype(int)[:, np.arange(v.shape[1]) // 128] - 127 - 6))


@pytest.mark.parametrize("T,E,k,K,N", [(1, 4, 2, 130, 70), (5, 64, 6, 256, 96), (300, 7, 2, 200, 129), (700, 16, 3, 512, 260), (2500, 6, 2, 300, 200)])
@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_layer_rounds_once(mad, T, E, k, K, N, dtype):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    print("case layer", T, E, k, K, N, dtype, flush=True)
    rng = np.random.default_rng(T + E)
    dt = getattr(torch, dtype)
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dt).cuda()      # noqa: E731
    x, weight, grad, logits = make(T, K), make(E, N, K), make(T, N), make(T, E)
    if T > 8:
        logits[torch.from_numpy(rng.random((T, E)) < 0.1).cuda()] = float("-inf")
        logits[3] = float("-inf")
    layer = ExpertLayer.from_weights(weight, k)
    out, saved = layer.forward(x, logits, training=True)
    serving, chosen = ExpertLayer(layer.W, None, k).forward(x, logits)
    assert torch.equal(chosen.ids, saved.ids) and torch.equal(chosen.weights, saved.weights)
    dx, dW, dlogits = layer.backward(saved, grad)
    assert {t.dtype for t in (out, serving, dx, dW, dlogits)} == {dt}
    h = lambda t: t.double().cpu().numpy()      # noqa: E731
    W, X, G, L, ids, w = h(layer.W.values()), h(x), h(grad), h(logits), saved.ids.cpu().numpy(), h(saved.weights)
    want, wdx, wdW, wdw = np.zeros((T, N)), np.zeros((T, K)), np.zeros((E, N, K)), np.zeros((T, k))
    size, sdx, sdW, sdw, cut = (np.zeros_like(a) for a in (want, wdx, wdW, wdw, wdW))
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if not len(t):
            continue
        Xq, wt = back(X[t])[0], w[t, j][:, None]
        y, sy = Xq @ W[e].T, np.abs(Xq) @ np.abs(W[e]).T
        want[t] += wt * y
        size[t] += wt * sy
        wdw[t, j], sdw[t, j] = (G[t] * y).sum(1), (np.abs(G[t]) * sy).sum(1)
        dy = (wt.astype(np.float32) * G[t].astype(np.float32)).astype(np.float64)
        q = back(dy)[0]
        wdx[t] += q @ W[e]
        sdx[t] += np.abs(q) @ np.abs(W[e])
        (a, a_cut), (b, b_cut) = back(np.ascontiguousarray(dy.T)), back(np.ascontiguousarray(X[t].T))
        wdW[e], sdW[e], cut[e] = a @ b.T, np.abs(a) @ np.abs(b).T, a_cut @ b_cut.T
    # sums of K, N or the tokens' number of products and of k in fp32, and one rounding to the type; the matrices' gradient to
    # bfloat16 may come from products of which seven of every eight are cut off at 2^-13 of the largest
    unit, least = UNIT[dtype], LEAST[dtype]
    for got, m, s, n, what in ((out, want, size, K, "out"), (serving, want, size, K, "serving"), (dx, wdx, sdx, N, "dx"), (dW, wdW, sdW, T + 128, "dW")):
        tol = (n + k + 16) * 2.0 ** -23 * s + 1.01 * unit * np.abs(m) + least
        if what == "dW" and dtype == "bfloat16":
            tol += 7 * 2.0 ** -13 * cut
        assert (np.abs(h(got) - m) <= tol).all(), (what, np.max(np.abs(h(got) - m) / tol))
    sw, _ = ref.scores(L, "softmax")
    wdl = ref.route_gradient(L, ids, wdw, "softmax", True, 1.0)
    mine = np.where(ids >= 0, np.take_along_axis(sw, np.clip(ids, 0, E - 1), 1), 0)
    tol = (K + N + 64 + k) * 2.0 ** -23 * sdw.max(1, keepdims=True) * 2 * k * sw / np.maximum(mine.sum(1, keepdims=True), 1e-30)
    assert (np.abs(h(dlogits) - wdl) <= tol + 1.01 * unit * np.abs(wdl) + least).all()


@pytest.mark.parametrize("T", [1, 40, 600])
def test_one_expert_may_pass_the_range_of_float16(mad, T):
    """Results of some 50000 and twice that, negative, whose weighted sum is in range, also where the weight of the second is 0."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    weight = torch.stack([torch.full((40, 256), 0.5), torch.full((40, 256), -1.0)]).cuda()
    layer = ExpertLayer.from_weights(weight, 2)
    x = torch.full((T, 256), 400.0, dtype=torch.float16, device="cuda")
    grad = torch.full((T, 40), 2.0 ** -10, dtype=torch.float16, device="cuda")
    value = float(back(np.full((1, 256), 400.0))[0][0, 0]) * 256            # (400 is no 8-bit number: the layer's is what it is rounded to)
    assert value > 65504
    for low, w in ((-200.0, (1.0, 0.0)), (-1.0, (1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))))):
        logits = torch.tensor([[0.0, low]], device="cuda").repeat(T, 1)
        want = (w[0] / 2 - w[1]) * value
        for training in (False, True):
            out, saved = layer.forward(x, logits, training=training)
            assert ((out.double() - want).abs() <= 2.0 ** -11 * abs(want) + 300 * 2.0 ** -23 * 1.5 * value).all()
        dx, dW, dlogits = layer.backward(saved, grad)
        # d weights = sum over the 40 of 2^-10 y, and d logits = +- w0 w1 (their difference), rounded in fp32
        d = w[0] * w[1] * 40 * 2.0 ** -10 * 1.5 * value
        assert (dlogits.double() - torch.tensor([d, -d], device="cuda")).abs().max() <= 1e-5 * (d + 1e-30)
        assert dx.isfinite().all() and dW.isfinite().all()


def test_layer_in_a_narrower_type_between(mad):
    """slot_dtype: what the products give is rounded to it, no more."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    g = torch.Generator(device="cuda").manual_seed(5)
    W = mad.maddness_quantise_blocks(torch.randn(6, 96, 200, generator=g, device="cuda"), 128)
    for T in (3, 900):
        x, logits = torch.randn(T, 200, generator=g, device="cuda").bfloat16(), torch.randn(T, 6, generator=g, device="cuda")
        ids, w = mad.maddness_route(logits, 2)
        for slot in (None, torch.bfloat16):
            offsets, _, source, place = mad.maddness_order(ids, 6)
            y = mad.maddness_block_product(x, W, offsets, source=source, repeat=2, out_dtype=slot or torch.float32)
            want = mad.maddness_combine(y, place, w, out_dtype=torch.bfloat16)
            assert torch.equal(ExpertLayer(W, None, 2, slot_dtype=slot).forward(x, logits)[0], want)
    with pytest.raises(TypeError, match="slot_dtype"):
        ExpertLayer(W, None, 2, slot_dtype=torch.float64)


def test_the_callers_tensors_may_change_before_the_backward_pass(mad):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    g = torch.Generator(device="cuda").manual_seed(6)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    layer, x, logits, grad = ExpertLayer.from_weights(make(6, 96, 200), 2), make(50, 200), make(50, 6), make(50, 96)
    _, saved = layer.forward(x, logits, training=True)
    want = layer.backward(saved, grad)
    _, saved = layer.forward(x, logits, training=True)
    x.zero_()
    logits.neg_()
    for a, b in zip(layer.backward(saved, grad), want):
        assert torch.equal(a, b)
