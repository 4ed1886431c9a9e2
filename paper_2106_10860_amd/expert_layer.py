"""A layer of experts at 8 bits: every token goes through k of E matrices and the results are added up with the weights of the choice.

    layer = ExpertLayer.from_weights(weight, k=2)        # weight [experts, outputs, inputs]
    out, saved = layer.forward(x, logits, training=True)
    dx, dW, dlogits = layer.backward(saved, grad)

Run as a module it trains such a layer on a task that wants different matrices for different tokens, and prints the loss; ``--norm`` puts a layer
norm before it, ``--balance`` adds the loss that keeps the experts' tokens alike, ``--clip`` scales the gradients down to a norm.
"""
from __future__ import annotations

import dataclasses

import paper_2106_10860_amd as m


@dataclasses.dataclass
class Saved:
    """What the backward pass needs of a forward pass (without training: ids and weights)."""
    ids: object
    weights: object
    logits: object = None
    offsets: object = None
    source: object = None
    place: object = None
    x_t: object = None
    y: object = None
    tokens: int = 0
    balance_loss: object = None        # with ``balance``: the loss, the experts' tokens and what the gradient takes
    counts: object = None
    push: object = None


class ExpertLayer:
    """W: BlockMatrix [experts, outputs, inputs] in tiles of 128; Wt: the same transposed, for the backward pass (or None).
    The choice is that of ``maddness_route``.

    ``slot_dtype`` is what a token's k results are held in between their products and the weighted sum (and those of the backward pass).  In
    fp32, the default, out and the gradients are rounded once, to the types that they are returned in.  A narrower type halves the bytes of
    that step and rounds every one of the k; float16 makes a result beyond 65504 infinite, also where its weight is 0 or the sum would be in
    range.

    ``balance``: the factor of the loss of ``maddness_balance``, or 0 for none.  In training it is in ``Saved.balance_loss`` (an fp32 scalar tensor, to be added to the
    model's own loss), beside the experts' tokens in ``Saved.counts``, and its gradient is part of that of the logits."""

    def __init__(self, W: "m.BlockMatrix", Wt=None, k: int = 1, scores: str = "softmax", bias=None, groups: int = 1, kept_groups: int = 1,
                 renormalise: bool = True, factor: float = 1.0, slot_dtype=None, balance: float = 0.0):
        if len(W.shape) != 3:
            raise ValueError("W must be [experts, outputs, inputs]")
        if Wt is not None and Wt.shape != (W.shape[0], W.shape[2], W.shape[1]):
            raise ValueError("Wt must be the transpose of W")
        if slot_dtype is None:
            import torch
            slot_dtype = torch.float32
        m.blocks._float_code(slot_dtype, "slot_dtype")
        self.W, self.Wt, self.experts, self.k, self.slot_dtype = W, Wt, W.shape[0], k, slot_dtype
        self.choice = {"scores": scores, "renormalise": renormalise, "factor": factor}
        self.balance = float(balance)
        self.groups = {"bias": bias, "groups": groups, "kept_groups": kept_groups}

    @classmethod
    def from_weights(cls, weight, k: int = 1, **choice) -> "ExpertLayer":
        """From float matrices [experts, outputs, inputs]; after an update of them, again."""
        W, Wt = m.maddness_quantise_blocks(weight, tile=m.BLOCK, both=True)
        return cls(W, Wt, k, **choice)

    def by_choice(self, tokens: int) -> bool:
        """Whether the product finds an expert's slots by itself, without an order of them (a launch less): while an expert has 16 rows
        or so, which it multiplies at a time.  64 experts of 1024 x 512, 6 to a token: 4 tokens 16 us, 22 with an order, 85 tokens 22 and 25;
        8 of 4096 x 4096, 2 to a token: 64 tokens 61 and 70, 85 tokens 73 and 68.  Where all tokens choose the same experts it costs up to
        half as much again (85 tokens of the first layer 37 and 25)."""
        return tokens * self.k <= min(m.MAX_CHOSEN, 16 * self.experts)

    def forward(self, x, logits, training: bool = False):
        """x [T, inputs], logits [T, experts] -> (out [T, outputs] of x's dtype, Saved)."""
        if x.shape[0] != logits.shape[0] or logits.shape[1] != self.experts or x.shape[1] != self.W.shape[2]:
            raise ValueError(f"x must be [T, {self.W.shape[2]}] and logits [T, {self.experts}]")
        if training and self.Wt is None:
            raise ValueError("training needs Wt")
        ids, weights = m.maddness_route(logits, self.k, **self.choice, **self.groups)
        if not training and self.by_choice(x.shape[0]):
            y = m.maddness_block_product(x, self.W, by="choice", source=ids, out_dtype=self.slot_dtype)
            return m.maddness_combine(y, None, weights, out_dtype=x.dtype), Saved(ids, weights)
        # in training the sums over an expert's tokens are products by depth, which go by whole blocks
        offsets, _, source, place = m.maddness_order(ids, self.experts, m.BLOCK if training else 1)
        x_t = m.maddness_quantise_blocks(x, transposed=True, source=source, repeat=self.k) if training else None
        y = m.maddness_block_product(x, self.W, offsets, source=source, repeat=self.k, out_dtype=self.slot_dtype)
        out = m.maddness_combine(y, place, weights, out_dtype=x.dtype)
        if not training:
            return out, Saved(ids, weights)
        # (a copy: the caller may write to its logits before the backward pass)
        saved = Saved(ids, weights, logits.clone(), offsets, source, place, x_t, y, x.shape[0])
        if self.balance:
            saved.balance_loss, saved.counts, saved.push = m.maddness_balance(logits, ids, scores=self.choice["scores"], factor=self.balance)
        return out, saved

    def backward(self, saved: Saved, grad, weight_dtype=None, balance_gradient=None):
        """The gradient of out [T, outputs] -> those of x, of the matrices [experts, outputs, inputs] (of ``weight_dtype``, or grad's
        dtype) and of logits.  ``balance_gradient``: that of the balance's loss, an fp32 tensor of one element (1: what a loss is scaled by)."""
        if saved.y is None:
            raise ValueError("saved is of a forward pass without training=True")
        if tuple(grad.shape) != (saved.tokens, self.W.shape[1]):
            raise ValueError(f"grad must be [{saved.tokens}, {self.W.shape[1]}]")
        if grad.stride(1) != 1 or grad.stride(0) < grad.shape[1]:        # (the gradient of a sum is one number in every place)
            grad = grad.contiguous()
        dweights = m.maddness_combine_gradient(grad, saved.y, saved.place)
        dlogits = m.maddness_route_gradient(saved.logits, saved.ids, dweights, **self.choice)
        if saved.push is not None:
            m.maddness_balance_gradient(saved.logits, saved.push, scores=self.choice["scores"], loss_gradient=balance_gradient, add=dlogits, out=dlogits)
        dy, dy_t = m.maddness_quantise_blocks(grad, both=True, source=saved.source, repeat=self.k, factors=saved.weights)
        dx = m.maddness_combine(m.maddness_block_product(dy, self.Wt, saved.offsets, out_dtype=self.slot_dtype), saved.place, out_dtype=grad.dtype)
        dW = m.maddness_block_product(dy_t, saved.x_t, saved.offsets, by="depth", out_dtype=weight_dtype or grad.dtype)
        return dx, dW, dlogits


def train_example(steps: int = 60, tokens: int = 2048, inputs: int = 256, outputs: int = 192, experts: int = 8, k: int = 2, seed: int = 0, norm: bool = False,
                  balance: float = 0.0, clip=None):
    """Tokens of several kinds, each with a matrix of its own; a gate and a layer of experts learn them.  Returns the losses."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kinds, truth = normal(experts, inputs), normal(experts, outputs, inputs) / inputs ** 0.5
    weight, gate = normal(experts, outputs, inputs) * (0.3 / inputs ** 0.5), 0.3 * normal(experts, inputs)
    scale, shift = torch.ones(inputs, device="cuda"), torch.zeros(inputs, device="cuda")
    losses = []
    for step in range(steps):
        kind = torch.randint(experts, (tokens,), generator=g, device="cuda")
        x = kinds[kind] + 0.5 * normal(tokens, inputs)
        want = torch.bmm(truth[kind], x.unsqueeze(2)).squeeze(2)
        h = x
        if norm:
            h, mean, rstd = m.maddness_layer_norm(x, scale, shift, training=True)
        layer = ExpertLayer.from_weights(weight, k, balance=balance)
        out, saved = layer.forward(h, h @ gate.T, training=True)
        losses.append(float(((out - want) ** 2).mean()))
        dh, dW, dlogits = layer.backward(saved, 2 * (out - want) / out.numel())
        gradients = [dW, dlogits.T @ h]
        if norm:
            gradients += m.maddness_layer_norm_gradient(dh + dlogits @ gate, x, mean, rstd, scale)[1:]
        if clip is not None:
            m.maddness_clip_gradients(gradients, clip)
        weight -= 4.0 * gradients[0]
        gate -= 0.05 * gradients[1]
        if norm:
            scale -= 0.05 * gradients[2]
            shift -= 0.05 * gradients[3]
    return losses


if __name__ == "__main__":
    import argparse
    parser = argparse.ArgumentParser(description="Trains a layer of experts.")
    parser.add_argument("--norm", action="store_true", help="a layer norm before the layer")
    parser.add_argument("--balance", type=float, default=0.0, help="factor of the loss that keeps the experts' tokens alike")
    parser.add_argument("--clip", type=float, default=None, help="largest norm of a step's gradients")
    chosen = parser.parse_args()
    curve = train_example(norm=chosen.norm, balance=chosen.balance, clip=chosen.clip)
    print("mean squared error, every tenth step: " + " ".join(f"{v:.4f}" for v in curve[::10] + curve[-1:]))
