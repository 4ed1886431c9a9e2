"""The calls around exact layers as a program makes them: one after the other, captured and replayed, on other streams, by several threads, beside the layer of experts."""
import threading

import numpy as np
import pytest

import layer_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mad():
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    return m


def normal(seed, *shape, dtype=None, scale=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device="cuda")).to(dtype or torch.float32)


def host(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows", [1, 5, 64, 333])
def test_serving(mad, rows):
    """Norm, integers, product, bias, as a served layer runs: against the same steps in 64 bits from the integers on, and the norm's own bounds before them."""
    import torch
    print("case serving", rows, flush=True)
    x, weight, w, b, bias = normal(1, rows, 700, dtype=torch.bfloat16), normal(2, 300, 700), 1 + 0.1 * normal(3, 700), 0.1 * normal(4, 700), normal(5, 300)
    W = mad.maddness_quantise_rows(weight)
    h = mad.maddness_layer_norm(x, w, b, integer=True)
    y = mad.maddness_integer_product(h, W, bias=bias, out_dtype=torch.float32)
    want, bound = ref.product(h.q.cpu().numpy().astype(np.int64), host(h.scale), W.q.cpu().numpy().astype(np.int64), host(W.scale), host(bias))
    assert (np.abs(host(y) - want) <= bound + ref.rounding(want, "f32")).all()
    # against the layer without any rounding: half a step for every one of the 700 products, on both sides
    exact = ref.norm(host(x), host(w), host(b), 1e-5, 0)[0]
    e_h, e_w = 0.5 * host(h.scale)[:, None] * 1.0001 + 1e-5, 0.5 * host(W.scale)[None, :] * 1.0001
    most = e_h * np.abs(host(weight)).sum(1)[None, :] + e_w * np.abs(exact).sum(1)[:, None] + 700 * e_h * e_w
    assert (np.abs(host(y) - (exact @ host(weight).T + host(bias))) <= most + bound).all()


def step(mad, layer, x, gate, w, b, grad, clip, gradients=None):
    """A training step's calls up to the clipped gradients."""
    h, mean, rstd = mad.maddness_layer_norm(x, w, b, training=True)
    logits = h @ gate.T
    out, saved = layer.forward(h, logits, training=True)
    dh, dW, dlogits = layer.backward(saved, grad)
    dx, dw, db = mad.maddness_layer_norm_gradient(dh + dlogits @ gate, x, mean, rstd, w)
    made = [dW, dlogits.T @ h, dw, db]
    norm = mad.maddness_clip_gradients(made, clip)
    return [out, saved.balance_loss, saved.counts, dx, norm, *made]


def problem(mad, T=300, E=8, K=256, N=192, seed=0):
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    layer = ExpertLayer.from_weights(normal(seed, E, N, K, scale=K ** -0.5), 2, balance=0.02)
    return layer, normal(seed + 1, T, K), normal(seed + 2, E, K, scale=0.1), 1 + 0.1 * normal(seed + 3, K), 0.1 * normal(seed + 4, K), normal(seed + 5, T, N, scale=1e-2)


def test_the_layers_balance(mad):
    """With `balance` the layer's results are as without, and the logits' gradient has the loss's beside the choice's."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    for scores in ("softmax", "sigmoid"):
        layer, x, gate, _, _, grad = problem(mad)
        logits = x @ gate.T
        plain = ExpertLayer(layer.W, layer.Wt, 2, scores=scores)
        with_balance = ExpertLayer(layer.W, layer.Wt, 2, scores=scores, balance=0.5)
        out, saved = plain.forward(x, logits, training=True)
        out2, saved2 = with_balance.forward(x, logits, training=True)
        assert torch.equal(out, out2) and saved.balance_loss is None and saved.push is None
        loss, counts, push = mad.maddness_balance(logits, saved.ids, scores=scores, factor=0.5)
        assert torch.equal(saved2.balance_loss, loss) and torch.equal(saved2.counts, counts) and int(counts.sum()) == saved.ids.numel()
        dx, dW, dlogits = plain.backward(saved, grad)
        dx2, dW2, dlogits2 = with_balance.backward(saved2, grad)
        assert torch.equal(dx, dx2) and torch.equal(dW, dW2)
        assert torch.equal(dlogits2, mad.maddness_balance_gradient(logits, push, scores=scores, add=dlogits))
        ten = with_balance.backward(saved2, grad, balance_gradient=torch.tensor([10.0], device="cuda"))[2]
        assert torch.equal(ten, mad.maddness_balance_gradient(logits, push, scores=scores, add=dlogits, loss_gradient=torch.tensor(10.0, device="cuda")))
        serving, chosen = with_balance.forward(x, logits)
        assert chosen.balance_loss is None


def test_the_balances_gradient_against_differences(mad):
    """The loss itself, moved along a direction: fp32 losses of 300 tokens differ by 2e-6 of themselves at most, a second difference by the step."""
    import torch
    layer, x, gate, _, _, _ = problem(mad)
    logits = x @ gate.T
    ids, _ = mad.maddness_route(logits, 2)
    loss, _, push = mad.maddness_balance(logits, ids)
    d = mad.maddness_balance_gradient(logits, push)
    direction = normal(9, *logits.shape)
    # the counts have no gradient: the same ids on both sides
    eps = 1e-2
    up, down = (float(mad.maddness_balance(logits + s * eps * direction, ids)[0]) for s in (1, -1))
    slope, want = (up - down) / (2 * eps), float((d.double() * direction.double()).sum())
    # third derivatives of a softmax are below 6, push sums to 8 at most over 300 tokens' shares: eps^2 of that, and the losses' own rounding
    size = float((direction.double().abs().amax(1) ** 3).mean()) * float(push.sum()) * 300
    assert abs(slope - want) <= 2e-6 * abs(up) / eps + eps ** 2 * size


def test_a_training_step(mad):
    """Each gradient within the norm's bound, and the norm that of the unclipped ones."""
    import torch
    layer, x, gate, w, b, grad = problem(mad)
    wide = step(mad, layer, x, gate, w, b, grad, 1e9)
    total = float(torch.sqrt(sum((t.double() ** 2).sum() for t in wide[5:])))
    assert abs(float(wide[4]) - total) <= 1e-7 * total
    tight = step(mad, layer, x, gate, w, b, grad, 0.25 * total)
    for a, c in zip(tight[:5], wide[:5]):
        assert torch.equal(a, c)
    for a, c in zip(tight[5:], wide[5:]):
        most = 3.01 * ref.U * c.abs().double() * 0.25 + 2.0 ** -149
        assert bool(((a.double() - c.double() * (0.25 * total / float(wide[4]))).abs() <= most).all())


def test_the_example_runs(mad):
    """Everything in one loop: finite losses, the same again, and without the new parts those of before."""
    from paper_2106_10860_amd.expert_layer import train_example
    small = dict(steps=4, tokens=300, inputs=128, outputs=96, experts=4)
    first = train_example(norm=True, balance=0.05, clip=0.01, **small)
    assert len(first) == 4 and np.isfinite(first).all()
    assert train_example(norm=True, balance=0.05, clip=0.01, **small) == first
    assert train_example(**small) == train_example(norm=False, balance=0.0, clip=None, **small)
    assert train_example(clip=1e9, **small) == train_example(**small)


def test_a_training_step_captured(mad):
    """Every replay, with eager work and other inputs between, gives the eager results of those inputs to the bit."""
    import torch
    layer, x, gate, w, b, grad = problem(mad)
    inputs = [x, normal(50, *x.shape), normal(51, *x.shape), x.clone()]
    want = [[t.clone() for t in step(mad, layer, v, gate, w, b, grad, 0.01)] for v in inputs]
    held = x.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(mad, layer, held, gate, w, b, grad, 0.01)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step(mad, layer, held, gate, w, b, grad, 0.01)
    for i in (1, 2, 0, 3, 1):
        held.copy_(inputs[i])
        graph.replay()
        eager = step(mad, layer, inputs[2], gate, w, b, grad, 0.01)
        torch.cuda.synchronize()
        for a, c in zip(results, want[i]):
            assert torch.equal(a, c)
        for a, c in zip(eager, want[2]):
            assert torch.equal(a, c)


def test_serving_captured_with_a_workspace_of_its_own(mad):
    """Two graphs with workspaces of their own run beside each other; out and workspace are the caller's."""
    import torch
    x = [normal(1, 200, 512, dtype=torch.bfloat16), normal(2, 200, 512, dtype=torch.bfloat16)]
    W = mad.maddness_quantise_rows(normal(3, 96, 512))
    want = [mad.maddness_integer_product(v, W) for v in x]
    need = mad.lib().maddness_integer_product_workspace(200, 512, mad.MADDNESS_BF16)
    graphs, outs = [], []
    for v in x:
        out, work = torch.empty(200, 96, dtype=torch.bfloat16, device="cuda"), torch.empty(need, dtype=torch.uint8, device="cuda")
        mad.maddness_integer_product(v, W, out=out, workspace=work)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mad.maddness_integer_product(v, W, out=out, workspace=work)
        graphs.append((graph, work))
        outs.append(out)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for s, (graph, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, c) for o, c in zip(outs, want))


def test_other_streams(mad):
    """`stream`: work and memory are that stream's, as with the package's other calls."""
    import torch
    layer, x, gate, w, b, grad = problem(mad, T=2000)
    big = normal(7, 4000, 1024)
    W = mad.maddness_quantise_rows(normal(8, 256, 1024))
    logits = x @ gate.T
    ids, _ = mad.maddness_route(logits, 2)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()

    def run(stream):
        y, mean, rstd = mad.maddness_layer_norm(big, training=True, stream=stream)
        loss, counts, push = mad.maddness_balance(logits, ids, stream=stream)
        copies = [big.clone()] if stream is None else None
        if copies is None:
            with torch.cuda.stream(stream):
                copies = [big.clone()]
        norm = mad.maddness_clip_gradients(copies, 1.0, stream=stream)
        q = mad.maddness_quantise_rows(big, stream=stream)
        return [y, mean, rstd, loss, counts, push, norm, copies[0], q.q, q.scale, mad.maddness_integer_product(big, W, stream=stream),
                *mad.maddness_layer_norm_gradient(y, big, mean, rstd, parameters=True, stream=stream), mad.maddness_balance_gradient(logits, push, stream=stream),
                mad.maddness_gradient_norm([big], stream=stream)]

    want = run(None)
    torch.cuda.synchronize()
    for _ in range(3):
        got = run(s)
        s.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, want))


def test_several_threads(mad):
    """Calls of several threads, each on a stream of its own, at the same time."""
    import torch
    layer, x, gate, w, b, grad = problem(mad)
    want = step(mad, layer, x, gate, w, b, grad, 0.01)
    torch.cuda.synchronize()
    errors = []

    def work():
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(5):
                    got = step(mad, layer, x, gate, w, b, grad, 0.01)
                    s.synchronize()
                    assert all(torch.equal(a, c) for a, c in zip(got, want))
        except Exception as e:        # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors


def test_a_function_of_torchs_own(mad):
    """The norm and its gradient in a torch.autograd.Function, against the 64-bit norm's gradients."""
    import torch

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, mean, rstd = mad.maddness_layer_norm(x, w, b, training=True)
            ctx.save_for_backward(x, mean, rstd, w)
            return y

        @staticmethod
        def backward(ctx, grad):
            x, mean, rstd, w = ctx.saved_tensors
            return mad.maddness_layer_norm_gradient(grad.contiguous(), x, mean, rstd, w)

    x, w, b, grad = (normal(1, 20, 300).requires_grad_(), torch.nn.Parameter(1 + 0.1 * normal(2, 300)), torch.nn.Parameter(normal(3, 300)), normal(4, 20, 300))
    Norm.apply(x, w, b).backward(grad)
    _, mean, r, _, _, _ = ref.norm(host(x.detach()), host(w.detach()), host(b.detach()), 1e-5, 0)
    dx, dw, db, e_dx, e_dw, e_db = ref.norm_gradient(host(grad), host(x.detach()), mean, r, host(w.detach()), 53, 60)
    # (the statistics are fp32 here: a few parts in 10^6 of each term)
    assert (np.abs(host(x.grad) - dx) <= e_dx + 2e-5).all() and (np.abs(host(w.grad) - dw) <= e_dw + 2e-4).all() and (np.abs(host(b.grad) - db) <= e_db + 1e-6).all()


@pytest.mark.parametrize("how", ["native", "python"])
def test_results_are_tensors_as_any(mad, monkeypatch, how):
    """Small results of one call may share an allocation: writing to one leaves the others, each can be saved, used further, and made in inference mode."""
    import torch
    if how == "python":
        monkeypatch.setattr(mad, "_native", mad._NotBuilt)
    x, w, logits = normal(1, 6, 40), 1 + 0.1 * normal(2, 40), normal(3, 9, 5)
    ids, _ = mad.maddness_route(logits, 2)

    def calls():
        y, mean, rstd = mad.maddness_layer_norm(x, w, training=True)
        return [mean, rstd, *mad.maddness_layer_norm_gradient(y, x, mean, rstd, w)[1:], *mad.maddness_balance(logits, ids)]

    want = [t.clone() for t in calls()]
    assert [(t.dtype, tuple(t.shape)) for t in want] == [(torch.float32, (6,))] * 2 + [(torch.float32, (40,))] * 2 + [(torch.float32, ()), (torch.int32, (5,)), (torch.float32, (5,))]
    got = calls()
    for i, t in enumerate(got):
        assert t.is_contiguous() and not t.requires_grad and t._version == 0
        t.add_(1)
        assert all(torch.equal(a, b) for a, b in zip(got[i + 1:], want[i + 1:]))
    for t, c in zip(got, want):
        assert torch.equal(t, c + 1)
    with torch.inference_mode():
        assert all(torch.equal(a, b) for a, b in zip(calls(), want))
    loss = calls()[4].requires_grad_()
    (2 * loss).backward()
    assert float(loss.grad) == 2
    import io
    file = io.BytesIO()
    torch.save(calls(), file)
    file.seek(0)
    assert all(torch.equal(a, b) for a, b in zip(torch.load(file, weights_only=True), want))


def test_the_layers_balance_of_logits_that_vanish(mad):
    """Sigmoid logits of -80 to -140 among a token's: loss and gradient are numbers, the gradient that of the choice with the balance's on top."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    layer, x, gate, _, _, grad = problem(mad)
    logits = x @ gate.T
    logits[::3, 1] = torch.linspace(-140, -80, 100, device="cuda")
    with_balance = ExpertLayer(layer.W, layer.Wt, 2, scores="sigmoid", balance=0.5)
    _, saved = with_balance.forward(x, logits, training=True)
    dlogits = with_balance.backward(saved, grad)[2]
    assert bool(saved.balance_loss.isfinite()) and bool(dlogits.isfinite().all())
    without = ExpertLayer(layer.W, layer.Wt, 2, scores="sigmoid")
    choice = without.backward(without.forward(x, logits, training=True)[1], grad)[2]
    want, counts, push, p, s, seen, _ = ref.balance(host(logits), saved.ids.cpu().numpy(), "sigmoid", 0.5)
    d = ref.balance_gradient(p, s, seen, host(saved.push), "sigmoid")
    # (shares and their products within 100 roundings, as every one of 8 experts' parts has less)
    most = 100 * ref.U * (p * (np.abs(host(saved.push)) + (p * host(saved.push)).sum(1, keepdims=True)) + np.abs(host(choice))) + 2.0 ** -126
    assert abs(float(saved.balance_loss) - want) <= 100 * ref.U * want and (np.abs(host(dlogits) - (host(choice) + d)) <= most).all()


def test_the_example_without_its_options_is_the_plain_loop(mad):
    """The steps of a loop of choice, layer and updates alone, written out: the same losses to the bit."""
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer, train_example
    steps, T, K, N, E, k = 4, 300, 128, 96, 4, 2
    g = torch.Generator(device="cuda").manual_seed(0)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kinds, truth = randn(E, K), randn(E, N, K) / K ** 0.5
    weight, gate = randn(E, N, K) * (0.3 / K ** 0.5), 0.3 * randn(E, K)
    losses = []
    for _ in range(steps):
        kind = torch.randint(E, (T,), generator=g, device="cuda")
        x = kinds[kind] + 0.5 * randn(T, K)
        off = ExpertLayer.from_weights(weight, k)
        out, saved = off.forward(x, x @ gate.T, training=True)
        error = out - torch.bmm(truth[kind], x.unsqueeze(2)).squeeze(2)
        losses.append(float((error ** 2).mean()))
        assert saved.balance_loss is None and saved.counts is None and saved.push is None
        _, dW, dlogits = off.backward(saved, 2 * error / error.numel())
        weight -= 4.0 * dW
        gate -= 0.05 * (dlogits.T @ x)
    assert train_example(steps=steps, tokens=T, inputs=K, outputs=N, experts=E) == losses
