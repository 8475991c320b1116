"""A feed-forward layer of gated experts as a generating transformer runs it: a router chooses top_k of them for every token, weights and activations
are 8 bits with a scale for each channel and each token, so that a token's output does not depend on who else is in the batch.

    python examples/expert_layer.py

prints how far the layer's output is from the same layer in fp64 with the same choice of experts (the error of 8 bits on both sides), and that a token
alone gets the bits that it gets in its batch.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2311_15806_amd.binding as pipe  # noqa: E402


class ExpertLayer:
    """width -> experts of SiLU(gate) * up of `hidden` features -> width, top_k a token.  Keeps the full-precision weights for reference()."""

    def __init__(self, width, hidden, experts, top_k, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        draw = lambda *shape: torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5     # noqa: E731
        self.top_k = top_k
        self.W = draw(experts, width), draw(experts, 2 * hidden, width), draw(experts, width, hidden)
        self.router, self.up, self.down = (self._codes(W) for W in self.W)

    @staticmethod
    def _codes(W):
        """Rows of the weights in 8 bits with a scale each, shaped as W."""
        codes, scales = pipe.pipe_token_quantize(W.reshape(-1, W.shape[-1]))
        return codes.view(*W.shape[:-1], -1), scales.view(W.shape[:-1])

    def forward(self, x):
        """(y [tokens, width], the experts of every token and their weights)"""
        logits = pipe.pipe_token_forward(x, *self.router)
        experts, weights, starts, order, places = pipe.pipe_expert_route(logits, self.top_k)
        h = pipe.pipe_expert_forward(x, *self.up, starts, order=order, top_k=self.top_k, act=pipe.PIPE_ACT_SILU_GATED)
        y = pipe.pipe_expert_forward(h, *self.down, starts)
        return pipe.pipe_expert_combine(y, places, weights), experts, weights

    def reference(self, x, experts, weights):
        """The same in fp64 with the full-precision weights."""
        _, up, down = (W.double() for W in self.W)
        x, y = x.double(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
        for e in range(up.shape[0]):
            t, j = torch.nonzero(experts == e, as_tuple=True)
            gate, h = (x[t] @ up[e].t().contiguous()).chunk(2, dim=1)
            y.index_add_(0, t, weights[t, j, None].double() * ((gate * torch.sigmoid(gate) * h) @ down[e].t().contiguous()))
        return y


def main(tokens=(300, 1, 7, 64), width=1024, hidden=704, experts=16, top_k=4, dtype=torch.bfloat16, say=print):
    """Returns the relative errors of the batches and whether single tokens get the same bits."""
    layer = ExpertLayer(width, hidden, experts, top_k)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    errors, same = [], True
    for T in tokens:
        x = torch.randn(T, width, generator=g, device="cuda").to(dtype)
        y, chosen, weights = layer.forward(x)
        want = layer.reference(x, chosen, weights)
        errors.append(float((y.double() - want).norm() / want.norm()))
        alone = layer.forward(x[T // 2:T // 2 + 1].contiguous())[0]
        same = same and bool(torch.equal(alone[0], y[T // 2]))
        say("%d tokens: %.1e of the full-precision layer; a token alone %s" % (T, errors[-1], "gets the same bits" if same else "DIFFERS"))
    return errors, same


if __name__ == "__main__":
    main()
