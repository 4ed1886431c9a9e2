"""Operands that require a gradient: the calls on 8-bit block matrices and experts record none, and say so."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def mad(request, monkeypatch):
    import torch
    import paper_2106_10860_amd as m
    assert torch.cuda.is_available()
    m.lib()
    if request.param == "python":
        monkeypatch.setattr(m, "_native", m._NotBuilt)
    return m


def test_operands_that_require_a_gradient_are_refused(mad):
    import torch
    from paper_2106_10860_amd.expert_layer import ExpertLayer
    T, E, k, K, N = 6, 4, 2, 64, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    x, logits, bias, y, out, grad, dw, weight = make(T, K), make(T, E), make(E), make(T * k, N), make(T, N), make(T, N), make(T, k), make(E, N, K)
    W, Wt = mad.maddness_quantise_blocks(weight, 128, both=True)
    B = mad.BlockMatrix(W.q[0], W.scale[0], 128)
    ids, w = mad.maddness_route(logits, k)
    offsets, _, source, place = mad.maddness_order(ids, E)
    calls = {
        "x": (x, lambda t: mad.maddness_quantise_blocks(t)),
        "factors": (w, lambda t: mad.maddness_quantise_blocks(x, source=source, repeat=k, factors=t)),
        "A": (x, lambda t: mad.maddness_block_product(t, B)),
        "out": (out, lambda t: mad.maddness_block_product(x, B, out=t)),
        "logits": (logits, lambda t: mad.maddness_route(t, k)),
        "bias": (bias, lambda t: mad.maddness_route(logits, k, bias=t)),
        "logits of the gradient": (logits, lambda t: mad.maddness_route_gradient(t, ids, dw)),
        "weights_gradient": (dw, lambda t: mad.maddness_route_gradient(logits, ids, t)),
        "y": (y, lambda t: mad.maddness_combine(t, place, w)),
        "weights": (w, lambda t: mad.maddness_combine(y, place, t)),
        "weights without places": (w, lambda t: mad.maddness_combine(y, None, t)),
        "gradient": (grad, lambda t: mad.maddness_combine_gradient(t, y, place)),
        "y of the gradient": (y, lambda t: mad.maddness_combine_gradient(grad, t, place)),
        "layer's x": (x, lambda t: ExpertLayer(W, Wt, k).forward(t, logits)),
        "layer's logits": (logits, lambda t: ExpertLayer(W, Wt, k).forward(x, t, training=True)),
        "layer's weight": (weight, lambda t: ExpertLayer.from_weights(t, k)),
    }
    for name, (tensor, call) in calls.items():
        print("case requires grad", name, flush=True)
        call(tensor)
        with_gradient = tensor.clone().requires_grad_()
        with pytest.raises(ValueError, match="requires a gradient"):
            call(with_gradient)
        with torch.no_grad():
            call(with_gradient)
        call(torch.nn.Parameter(tensor, requires_grad=False))


def test_the_gradients_calls_in_an_autograd_function(mad):
    """The way that the error names: a Function's forward and backward run without recording."""
    import torch
    W, Wt = mad.maddness_quantise_blocks(torch.randn(40, 64, device="cuda"), 128, both=True)

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return mad.maddness_block_product(x, W, out_dtype=torch.float32)

        @staticmethod
        def backward(ctx, grad):
            return mad.maddness_block_product(grad.contiguous(), Wt, out_dtype=torch.float32)

    x = torch.randn(6, 64, device="cuda", requires_grad=True)
    grad = torch.randn(6, 40, device="cuda")
    Layer.apply(x).backward(grad)
    assert torch.equal(x.grad, mad.maddness_block_product(grad, Wt, out_dtype=torch.float32))
