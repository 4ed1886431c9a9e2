"""The choice of experts, their order, the weighted sum and the layer made of them, against 64 bits."""
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


def logits_of(seed, T, E, dtype, masked):
    import torch
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((T, E)) * 2).to(dtype)
    if masked:
        x[torch.from_numpy(rng.random((T, E)) < masked)] = float("-inf")
        x[3 % T] = float("-inf")
        x[5 % T] = torch.finfo(dtype).min                  # the type's lowest value is a number like others
        x[6 % T, 0] = float("nan")
        x[7 % T, E - 1] = float("inf")
    return x


CHOICES = [(1, 1, 1, 1, 1), (7, 5, 5, 1, 1), (40, 64, 8, 8, 4), (33, 60, 4, 1, 1), (50, 96, 6, 4, 2), (64, 256, 8, 8, 4), (9, 256, 32, 1, 1),
           (130, 257, 3, 1, 1), (21, 510, 8, 6, 2), (17, 1024, 8, 64, 7), (1000, 128, 2, 1, 1)]


@pytest.mark.parametrize("T,E,k,groups,kept", CHOICES)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_route(mad, T, E, k, groups, kept, kind, dtype):
    import torch
    print("case route", T, E, k, groups, kept, kind, dtype, flush=True)
    rng = np.random.default_rng(E)
    for masked, bias, renormalise in ((0, None, True), (0.4, rng.standard_normal(E).astype(np.float32) * 0.1, False)):
        x = logits_of(T * E + k, T, E, getattr(torch, dtype), masked)
        if bias is not None and E > 8:
            bias[2], bias[4] = -np.inf, np.nan
        with np.errstate(invalid="ignore"):
            want, w, gap = ref.route(x.double().numpy(), k, kind, bias, groups, kept, renormalise, 1.5)
        wide = torch.zeros(T, E + 3, dtype=x.dtype, device="cuda")
        wide[:, 1:E + 1] = x.cuda()
        ids, weights = mad.maddness_route(wide[:, 1:E + 1], k, kind, None if bias is None else torch.from_numpy(bias).cuda(), groups, kept,
                                          renormalise, 1.5)
        ids, weights = ids.cpu().numpy(), weights.double().cpu().numpy()
        # keys are sums of a score of at most 1 (error of a few 2^-24) and a bias, group values of two keys: choices further apart are the same
        sure = (gap > 32 * 2.0 ** -24) | (gap == np.inf)
        assert sure.mean() > 0.5 or T < 4 or masked
        assert (ids[sure] == want[sure]).all()
        # 2^-24 for the exponential's argument of up to 16 and its value, the sum, two divisions, the factor
        assert (np.abs(weights - w)[sure] <= 64 * 2.0 ** -24 * np.abs(w[sure]) + 1e-37).all()
        assert (ids[np.isneginf(x.float().numpy()).all(1)] == -1).all()


def test_route_ties_go_to_the_lowest_index(mad):
    import torch
    for E in (8, 64, 200, 1024):
        ids, w = mad.maddness_route(torch.zeros(5, E, device="cuda"), 4)
        assert (ids.cpu() == torch.arange(4)).all() and (w == 0.25).all()
        x = torch.zeros(5, E, device="cuda")
        x[:, E // 2:] = 1
        assert (mad.maddness_route(x, 3, "sigmoid")[0].cpu() == E // 2 + torch.arange(3)).all()
        ids, _ = mad.maddness_route(torch.zeros(3, E, device="cuda"), 4, groups=4, kept_groups=2)
        assert (ids.cpu() == torch.tensor([[i for i in range(E // 2)][:4]])).all()


def test_route_with_scores_of_zero(mad):
    """Sigmoids that underflow to 0: still a choice, weights 0 where all are."""
    import torch
    x = torch.full((2, 6), -200.0, device="cuda")
    x[1, 4] = 0
    ids, w = mad.maddness_route(x, 2, "sigmoid")
    assert ids.cpu().tolist() == [[0, 1], [4, 0]]
    assert w.cpu().tolist() == [[0, 0], [1, 0]]


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (6, 5, 2), (40, 64, 8), (33, 60, 4), (64, 256, 8), (20, 300, 32), (9, 1024, 6)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_route_gradient(mad, T, E, k, kind, renormalise):
    import torch
    print("case route gradient", T, E, k, kind, renormalise, flush=True)
    rng = np.random.default_rng(E + k)
    x = logits_of(E + T, T, E, torch.float32, 0.2 if T > 8 else 0)
    ids = rng.integers(-1, E, (T, k)).astype(np.int32)                    # any: the same twice, none, and beyond
    if T > 8:
        ids[0] = ref.route(x.double().numpy()[:1], k, kind)[0][0]
        ids[1, 0], ids[2, k - 1] = E, -7
    dw = rng.standard_normal((T, k)).astype(np.float32)
    with np.errstate(invalid="ignore"):
        want = ref.route_gradient(x.double().numpy(), ids, dw.astype(np.float64), kind, renormalise, 2.0)
        s, _ = ref.scores(x.double().numpy(), kind)
    got = mad.maddness_route_gradient(x.cuda(), torch.from_numpy(ids).cuda(), torch.from_numpy(dw).cuda(), kind, renormalise, 2.0)
    got = got.double().cpu().numpy()
    # every term is at most factor |dw| s / total (renormalised; total >= the s itself) and carries some 64 roundings of 2^-24, k of them in sums
    there = (ids >= 0) & (ids < E)
    mine = np.where(there, np.take_along_axis(s, np.clip(ids, 0, E - 1), 1), 0)
    total = np.maximum(mine.sum(1, keepdims=True), 1e-30) if renormalise else 1.0
    size = (np.abs(dw) * there).max(1, keepdims=True) * 2.0 * 2 * k
    tol = (64 + k) * 2.0 ** -24 * size * s / total + 1e-36
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("slots,E", [(0, 3), (1, 1), (63, 5), (64, 64), (1000, 7), (1024, 1024), (5000, 60), (100003, 256), (1200000, 9)])
@pytest.mark.parametrize("align", [1, 16, 128])
def test_order(mad, slots, E, align):
    import torch
    print("case order", slots, E, align, flush=True)
    rng = np.random.default_rng(slots + E)
    ids = np.minimum(rng.integers(-2, E + 2, slots), rng.integers(0, E + 1, slots)).astype(np.int32)
    offsets, counts, source, place = (t.cpu().numpy() for t in mad.maddness_order(torch.from_numpy(ids).cuda(), E, align))
    ok = (ids >= 0) & (ids < E)
    n = np.bincount(ids[ok], minlength=E)
    assert (counts == n).all()
    assert (offsets == np.concatenate([[0], np.cumsum(-(-n // align) * align)])).all()
    want = np.full(source.shape, -1)
    for e in range(E):
        want[offsets[e]:offsets[e] + n[e]] = np.flatnonzero(ids == e)
    assert (source == want).all()
    want_place = np.full(slots, -1)
    want_place[want[want >= 0]] = np.flatnonzero(want >= 0)
    assert (place == want_place).all()


@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (5, 2, 7), (37, 6, 512), (64, 3, 510), (9, 8, 1030)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_combine(mad, T, k, N, dtype):
    import torch
    print("case combine", T, k, N, dtype, flush=True)
    rng = np.random.default_rng(T * N)
    dt = getattr(torch, dtype)
    rows = T * k + 3
    y = torch.from_numpy(rng.standard_normal((rows, N + 3))).to(dt).cuda()[:, 2:N + 2]
    grad = torch.from_numpy(rng.standard_normal((T, N + 1))).to(dt).cuda()[:, 1:]
    place = rng.integers(-2, rows + 2, (T, k)).astype(np.int32)
    w = rng.standard_normal((T, k)).astype(np.float32)
    ok = (place >= 0) & (place < rows)
    yy = np.where(ok[..., None], y.double().cpu().numpy()[np.where(ok, place, 0)], 0)
    place_d, w_d = torch.from_numpy(place).cuda(), torch.from_numpy(w).cuda()
    for weights, ww in ((None, np.ones((T, k))), (w_d, w.astype(np.float64))):
        for out_dt, unit in ((torch.float32, 0.0), (dt, {"float32": 0, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype])):
            got = mad.maddness_combine(y, place_d, weights, out_dtype=out_dt).double().cpu().numpy()
            want = (ww[..., None] * yy).sum(1)
            assert (np.abs(got - want) <= 2 * k * 2.0 ** -24 * np.abs(ww[..., None] * yy).sum(1) + 1.01 * unit * np.abs(want) + 1e-7 * (unit > 0)).all()
    got = mad.maddness_combine_gradient(grad, y, place_d).double().cpu().numpy()
    terms = grad.double().cpu().numpy()[:, None] * yy
    assert (np.abs(got - terms.sum(2)) <= 2 * N * 2.0 ** -24 * np.abs(terms).sum(2) + 1e-30).all()


@pytest.mark.parametrize("T,E,k,K,N", [(1, 4, 2, 130, 70), (5, 64, 6, 256, 96), (300, 7, 2, 200, 129), (700, 16, 3, 512, 260)])
def test_layer(mad, T, E, k, K, N):
    """Forward and backward of the whole layer against the same steps in 64 bits on the values that were rounded."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    print("case layer", T, E, k, K, N, flush=True)
    rng = np.random.default_rng(T + E)
    f32 = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda()      # noqa: E731
    x, weight, grad = f32(T, K), f32(E, N, K), f32(T, N)
    logits = logits_of(T, T, E, torch.float32, 0.1 if T > 8 else 0).cuda()
    logits.nan_to_num_(0.0, 0.0, float("-inf"))
    layer = ExpertLayer.from_weights(weight, k)
    out, saved = layer.forward(x, logits, training=True)
    serving, _ = ExpertLayer(layer.W, None, k).forward(x, logits)
    dx, dW, dlogits = layer.backward(saved, grad)
    h = lambda t: t.double().cpu().numpy()      # noqa: E731
    W, X, G, ids, w = h(layer.W.values()), h(x), h(grad), saved.ids.cpu().numpy(), h(saved.weights)
    back = lambda m, tile=1: ref.value(*ref.quantise(m, tile), tile)      # noqa: E731
    want, wdx, wdW, wdw = np.zeros((T, N)), np.zeros((T, K)), np.zeros((E, N, K)), np.zeros((T, k))
    size, sdx, sdW, sdw = np.zeros((T, N)), np.zeros((T, K)), np.zeros((E, N, K)), np.zeros((T, k))
    for e in range(E):
        t, j = np.nonzero(ids == e)
        if not len(t):
            continue
        Xq, y_of = back(X[t]), lambda a, b: a @ b.T      # noqa: E731
        y, sy = y_of(Xq, W[e]), y_of(np.abs(Xq), np.abs(W[e]))
        wt = w[t, j][:, None]
        want[t] += wt * y
        size[t] += wt * sy
        wdw[t, j], sdw[t, j] = (G[t] * y).sum(1), (np.abs(G[t]) * sy).sum(1)
        dy = (wt.astype(np.float32) * G[t].astype(np.float32)).astype(np.float64)
        q = back(dy)
        wdx[t] += q @ W[e]
        sdx[t] += np.abs(q) @ np.abs(W[e])
        a, b = back(np.ascontiguousarray(dy.T)), back(np.ascontiguousarray(X[t].T))
        wdW[e], sdW[e] = a @ b.T, np.abs(a) @ np.abs(b).T
    # sums of K, N or the tokens' number of products, and of k, in fp32; y comes rounded to fp32 once more
    unit = 2.0 ** -23
    for got, m, s, n, what in ((out, want, size, K, "out"), (serving, want, size, K, "serving"), (dx, wdx, sdx, N, "dx"), (dW, wdW, sdW, T + 128, "dW")):
        assert (np.abs(h(got) - m) <= (n + k + 16) * unit * s + 1e-30).all(), what
    sw, _ = ref.scores(h(logits), "softmax")
    wdl = ref.route_gradient(h(logits), ids, wdw, "softmax", True, 1.0)
    mine = np.where(ids >= 0, np.take_along_axis(sw, np.clip(ids, 0, E - 1), 1), 0)
    off = (K + N + 64 + k) * unit * sdw.max(1, keepdims=True) * 2 * k
    assert (np.abs(h(dlogits) - wdl) <= off * sw / np.maximum(mine.sum(1, keepdims=True), 1e-30) + 1e-30).all()


def test_layer_under_a_graph_and_on_another_stream(mad):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    g = torch.Generator(device="cuda").manual_seed(1)
    x, logits = torch.randn(6, 256, generator=g, device="cuda").bfloat16(), torch.randn(6, 16, generator=g, device="cuda")
    layer = ExpertLayer.from_weights(torch.randn(16, 96, 256, generator=g, device="cuda"), 3)
    want = layer.forward(x, logits)[0].clone()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        assert torch.equal(layer.forward(x, logits)[0], want)
        with torch.cuda.graph(graph, stream=side):
            out = layer.forward(x, logits)[0]
    for replay in range(3):
        out.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), replay
        layer.forward(x, logits)
        torch.cuda.synchronize()


def test_layer_of_no_tokens(mad):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    layer = ExpertLayer.from_weights(torch.ones(4, 32, 64, device="cuda"), 2)
    out, saved = layer.forward(torch.zeros(0, 64, device="cuda"), torch.zeros(0, 4, device="cuda"), training=True)
    dx, dW, dlogits = layer.backward(saved, torch.zeros(0, 32, device="cuda"))
    assert out.shape == (0, 32) and dx.shape == (0, 64) and dlogits.shape == (0, 4) and (dW == 0).all() and dW.shape == (4, 32, 64)


def test_example_learns(mad):
    from paper_2106_10860_amd.expert_layer import train_example
    losses = train_example()
    print("losses", losses[::10], flush=True)
    assert losses[-1] < 0.5 * losses[0]


def test_calls_without_the_native_marshalling_give_the_same(mad, monkeypatch):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    x, logits, bias, weight, grad = r(50, 200).bfloat16(), r(50, 24), 0.1 * r(24), r(24, 70, 200), r(50, 70).bfloat16()
    side = torch.cuda.Stream()

    def all_calls():
        seen = []
        W, Wt = mad.maddness_quantise_blocks(weight, 128, both=True)
        for stream in (None, side):
            torch.cuda.synchronize()
            ids, w = mad.maddness_route(logits, 3, "sigmoid", bias, 4, 2, True, 2.0, stream=stream)
            offsets, counts, source, place = mad.maddness_order(ids, 24, 128, stream=stream)
            a, at = mad.maddness_quantise_blocks(x, both=True, source=source, repeat=3, factors=w, stream=stream)
            one = mad.maddness_quantise_blocks(x, transposed=True, stream=stream)
            y = mad.maddness_block_product(a, W, offsets, out_dtype=torch.float32, stream=stream)
            torch.cuda.synchronize()
            y = torch.where((source >= 0)[:, None], y, 0)      # (rows that no expert has are not written)
            torch.cuda.synchronize()
            d = mad.maddness_block_product(at, at, offsets, by="depth", stream=stream)
            few = mad.maddness_block_product(x[:3], mad.BlockMatrix(W.q[0], W.scale[0], 128), stream=stream)
            many = mad.maddness_block_product(x, mad.BlockMatrix(W.q[0], W.scale[0], 128), out=torch.zeros(50, 70, device="cuda"), stream=stream)
            out = mad.maddness_combine(y, place, w, out_dtype=torch.bfloat16, stream=stream)
            dw = mad.maddness_combine_gradient(grad, y, place, stream=stream)
            dl = mad.maddness_route_gradient(logits, ids, dw, "sigmoid", True, 2.0, stream=stream)
            torch.cuda.synchronize()
            seen += [ids, w, offsets, counts, source, place, a.values(), at.values(), one.values(), y, d, few, many, out, dw, dl]
        return seen

    native = all_calls()
    assert mad._native.__name__ == "maddness_binding"
    monkeypatch.setattr(mad, "_native", mad._NotBuilt)
    plain = all_calls()
    for i, (a, b) in enumerate(zip(native, plain)):
        assert a.dtype is b.dtype and torch.equal(a, b), i


def test_sums_over_no_columns(mad):
    import torch
    place = torch.zeros(5, 2, dtype=torch.int32, device="cuda")
    y, gradient = torch.zeros(7, 0, device="cuda"), torch.zeros(5, 0, device="cuda")
    assert mad.maddness_combine(y, place).shape == (5, 0)
    assert torch.equal(mad.maddness_combine_gradient(gradient, y, place), torch.zeros(5, 2, device="cuda"))


def test_more_tokens_than_a_launch_takes(mad):
    import torch
    T = (1 << 25) + 77
    logits = torch.randn(T, 4, dtype=torch.float16, device="cuda")
    ids, weights = mad.maddness_route(logits, 1, "sigmoid", renormalise=False)
    last, last_weights = mad.maddness_route(logits[-500:], 1, "sigmoid", renormalise=False)
    assert torch.equal(ids[-500:], last) and torch.equal(weights[-500:], last_weights)
    gradient = mad.maddness_route_gradient(logits, ids, weights, "sigmoid", renormalise=False)
    assert torch.equal(gradient[-500:], mad.maddness_route_gradient(logits[-500:], last, last_weights, "sigmoid", renormalise=False))
    del logits, gradient, weights
    y = torch.randn(4, 8, device="cuda").to(torch.bfloat16)
    out = mad.maddness_combine(y, ids)
    assert torch.equal(out, y[ids[:, 0].long()])
    dw = mad.maddness_combine_gradient(out, y, ids)
    assert torch.equal(dw[-500:], mad.maddness_combine_gradient(out[-500:], y, ids[-500:]))


def test_layer_takes_the_gradient_of_a_sum(mad):
    """One number in every place, which the caller has as a tensor without strides."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    g = torch.Generator(device="cuda").manual_seed(2)
    layer = ExpertLayer.from_weights(torch.randn(4, 96, 64, generator=g, device="cuda"), 2)
    x, logits = torch.randn(50, 64, generator=g, device="cuda"), torch.randn(50, 4, generator=g, device="cuda")
    _, saved = layer.forward(x, logits, training=True)
    ones = torch.ones((), device="cuda").expand(50, 96)
    for got, want in zip(layer.backward(saved, ones), layer.backward(saved, ones.contiguous())):
        assert torch.equal(got, want)


@pytest.mark.parametrize("T,E,k,K,N", [(1, 1, 1, 8, 1), (1, 8, 2, 512, 96), (4, 64, 6, 1024, 512), (37, 5, 3, 330, 70), (50, 3, 2, 2000, 33), (256, 40, 2, 200, 129)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("skew", [False, True])
def test_product_by_choice_is_that_by_rows(mad, T, E, k, K, N, dtype, skew):
    """Every slot's row by its expert's matrix: within the bound of its terms, and what an order of the slots gives."""
    import torch
    from test_gpu_block_product import check
    print("case by choice", T, E, k, K, N, dtype, skew, flush=True)
    rng = np.random.default_rng(T + E)
    ids = rng.integers(-2, E + 2, (T, k)).astype(np.int32)                # some of no expert
    if skew:
        ids[rng.random((T, k)) < 0.8] = E // 2
    x = torch.from_numpy(rng.standard_normal((T, K))).to(getattr(torch, dtype)).cuda()
    W = mad.maddness_quantise_blocks(torch.from_numpy(rng.standard_normal((E, N, K)).astype(np.float32)).cuda(), 128)
    ids_d = torch.from_numpy(ids).cuda()
    A = mad.maddness_quantise_blocks(x)
    flat = ids.reshape(-1)
    for a in (x, A):
        out = torch.full((T * k, N + 2), 7.0, dtype=torch.float32, device="cuda")
        mad.maddness_block_product(a, W, by="choice", source=ids_d, out=out[:, 1:N + 1])
        assert (out[:, 0] == 7).all() and (out[:, N + 1:] == 7).all()
        out = out[:, 1:N + 1]
        assert (out.cpu()[torch.from_numpy((flat < 0) | (flat >= E))] == 0).all()
        for e in range(E):
            slots = np.nonzero(flat == e)[0]
            if len(slots):
                check(out[torch.from_numpy(slots).cuda()], A.values()[torch.from_numpy(slots // k).cuda()].double().cpu().numpy(),
                      W.values()[e].double().cpu().numpy(), f"expert {e}")
    weights = torch.rand(T, k, device="cuda")
    y = mad.maddness_block_product(x, W, by="choice", source=ids_d, out_dtype=x.dtype)
    got = mad.maddness_combine(y, None, weights)
    want = sum(weights[:, j:j + 1].double() * y.view(T, k, N)[:, j].double() for j in range(k))
    size = sum(weights[:, j:j + 1].double() * y.view(T, k, N)[:, j].double().abs() for j in range(k))
    # k roundings of fp32 and one of the result
    unit = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}[dtype]
    assert ((got.double() - want).abs() <= (k + 1) * 2.0 ** -23 * size + 1.01 * unit * want.abs() + 2.0 ** -24).all()
    # one slot at a time: source as it is, of any rows
    assert torch.equal(mad.maddness_block_product(x, W, by="choice", source=ids_d.view(-1), repeat=k, out_dtype=x.dtype), y)


def test_product_by_choice_of_nothing(mad):
    import torch
    W = mad.maddness_quantise_blocks(torch.ones(3, 20, 32, device="cuda"), 128)
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    assert mad.maddness_block_product(torch.zeros(0, 32, device="cuda"), W, by="choice", source=none).shape == (0, 20)
    assert mad.maddness_block_product(torch.ones(4, 32, device="cuda"), W, by="choice", source=none).shape == (0, 20)
    W0 = mad.BlockMatrix.empty((3, 20, 0), 128)
    got = mad.maddness_block_product(torch.ones(2, 0, device="cuda"), W0, by="choice", source=torch.tensor([[0], [2]], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, torch.zeros(2, 20, dtype=torch.bfloat16, device="cuda"))


def test_layer_by_choice_is_the_layer_by_order(mad, monkeypatch):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    g = torch.Generator(device="cuda").manual_seed(4)
    layer = ExpertLayer.from_weights(torch.randn(24, 200, 300, generator=g, device="cuda"), 4)
    for T in (1, 5, 60):
        x, logits = torch.randn(T, 300, generator=g, device="cuda").half(), torch.randn(T, 24, generator=g, device="cuda")
        logits[T // 2] = float("-inf")                                     # a token without an expert
        assert layer.by_choice(T)
        out, saved = layer.forward(x, logits)
        assert (out[T // 2] == 0).all() and out.isfinite().all()
        with monkeypatch.context() as way:
            way.setattr(ExpertLayer, "by_choice", lambda self, tokens: False)
            other, _ = layer.forward(x, logits)
        assert torch.equal(out, other)
    assert not layer.by_choice(97)


def test_choice_refuses(mad):
    import torch
    W = mad.maddness_quantise_blocks(torch.ones(3, 20, 32, device="cuda"), 128)
    x, ids = torch.ones(4, 32, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    for kw, error in ((dict(by="choice"), "source"), (dict(by="choice", source=ids, offsets=torch.zeros(4, dtype=torch.int32, device="cuda")), "offsets"),
                      (dict(by="choice", source=ids[:, :1]), "contiguous|view"), (dict(by="choices", source=ids), "by must"),
                      (dict(by="choice", source=ids.view(-1)), "rows"), (dict(by="choice", source=ids.view(-1), repeat=0), "repeat")):
        with pytest.raises((ValueError, RuntimeError), match=error):
            mad.maddness_block_product(x, W, **kw)
    with pytest.raises((ValueError, RuntimeError), match="slots"):
        mad.maddness_block_product(torch.ones(600, 32, device="cuda"), W, by="choice", source=torch.zeros(600, dtype=torch.int32, device="cuda"))
    with pytest.raises((TypeError, ValueError), match="int32"):
        mad.maddness_block_product(x, W, by="choice", source=ids.long())
    with pytest.raises((ValueError, RuntimeError), match="place"):
        mad.maddness_combine(torch.ones(7, 20, device="cuda"), None, torch.ones(4, 2, device="cuda"))
    with pytest.raises(ValueError, match="place"):
        mad.maddness_combine(torch.ones(8, 20, device="cuda"))


def test_choice_without_the_native_marshalling_gives_the_same(mad, monkeypatch):
    import torch
    W = mad.maddness_quantise_blocks(torch.randn(3, 20, 32, device="cuda"), 128)
    x, ids = torch.randn(4, 32, device="cuda"), torch.tensor([[0, 2], [1, -1], [2, 2], [5, 0]], dtype=torch.int32, device="cuda")
    weights = torch.rand(4, 2, device="cuda")

    def all_of():
        y = mad.maddness_block_product(x, W, by="choice", source=ids)
        return y, mad.maddness_combine(y, None, weights), mad.maddness_combine(y, weights=weights)
    want = all_of()
    monkeypatch.setattr(mad, "_native", mad._NotBuilt)
    for a, b in zip(want, all_of()):
        assert torch.equal(a, b)
