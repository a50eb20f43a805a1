"""A pre-norm feed-forward block trained in 8-bit floating point: the operators around the layers, used together.

  Y = X + W2 relu(W1 layernorm(X))

Weights are float32; their codes (128 x 128 tiles, by row for the forward, by column for the input gradient) are
formed once a step and kept between steps that do not change them, as while serving.  Every product reads 8-bit
floating point operands with a scale for each block of 128 and sums in float32; gradients are quantized
stochastically, so that they stay unbiased (Sec. 2.2), with independent draws for grad_W and grad_X (App. E).
Gradients are clipped by their global norm before the update.

  python -m paper_2010_14298_amd.ffn [--tokens N] [--width D] [--hidden H] [--steps K]

trains one block to follow another of random weights and prints the loss; then serves single tokens.
"""
import argparse

import torch

from . import fqt


class FeedForward:
    """One block of width D and hidden width H.  dtype: the type of activations and their gradients."""

    def __init__(self, D, H, dtype=torch.bfloat16, device="cuda", seed=0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.dtype = dtype
        self.W1 = torch.randn((H, D), generator=gen, device=device) * (2.0 / D) ** 0.5
        self.W2 = torch.randn((D, H), generator=gen, device=device) * (0.5 / H) ** 0.5
        self.gamma, self.beta = torch.ones(D, device=device), torch.zeros(D, device=device)
        self.quantize()

    def parameters(self):
        return [self.W1, self.W2, self.gamma, self.beta]

    def quantize(self):
        """The codes of the weights as they are now."""
        self.W1_8, self.W1_8t = fqt.fqt_fp8_quantize(self.W1, tile=True, by_row=True, by_col=True)
        self.W2_8, self.W2_8t = fqt.fqt_fp8_quantize(self.W2, tile=True, by_row=True, by_col=True)

    def forward(self, X, keep=True):
        """(Y, what the backward reads); keep=False (serving) forms no operands for it."""
        Xn, mean, rstd = fqt.fqt_layernorm_forward(X, self.gamma, self.beta)
        H, Xn8t, _ = fqt.fqt_fp8_linear_forward(Xn, self.W1_8, relu=True, save=keep)
        Z, H8t, _ = fqt.fqt_fp8_linear_forward(H, self.W2_8, save=keep)
        return Z + X, (X, mean, rstd, Xn8t, H, H8t) if keep else None

    def backward(self, dY, kept, seed):
        """(gradients in the order of parameters(), dX)."""
        X, mean, rstd, Xn8t, H, H8t = kept
        dW2, dH, _ = fqt.fqt_fp8_linear_backward(dY, H8t, self.W2_8t, seed=2 * seed, relu_input=H)
        dW1, dXn, _ = fqt.fqt_fp8_linear_backward(dH, Xn8t, self.W1_8t, seed=2 * seed + 1)
        dX, dgamma, dbeta, _ = fqt.fqt_layernorm_backward(dXn, X, mean, rstd, self.gamma)
        return [dW1, dW2, dgamma, dbeta], dX + dY

    def step(self, X, target, lr, max_norm, seed):
        """One training step on 1/2 mean |Y - target|^2; returns (loss, gradient norm), device scalars.

        The backward runs on the loss times the power of two next to its number of elements: float16 would lose
        diff / numel below its smallest step.  The float32 gradients of the parameters are larger by as much, exactly,
        which the bound, the update and the norm take out again."""
        Y, kept = self.forward(X)
        diff = Y.float() - target.float()
        loss = 0.5 * diff.square().mean()
        scale = 2.0 ** (diff.numel() - 1).bit_length()
        grads, _ = self.backward((diff / diff.numel() * scale).to(self.dtype), kept, seed)
        norm, _ = fqt.fqt_grad_norm_clip(grads, max_norm * scale)
        for p, g in zip(self.parameters(), grads):
            p.add_(g, alpha=-lr / scale)
        self.quantize()
        return loss, norm / scale


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lr", type=float, default=2.0)
    a = ap.parse_args(argv)
    teacher, block = FeedForward(a.width, a.hidden, seed=1), FeedForward(a.width, a.hidden, seed=2)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    losses = []
    for i in range(a.steps):
        X = torch.randn((a.tokens, a.width), generator=gen, device="cuda").to(block.dtype)
        loss, norm = block.step(X, teacher.forward(X, keep=False)[0], a.lr, 1.0, seed=i)
        losses.append(loss)
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {float(loss):.5f}  gradient norm {float(norm):.4f}", flush=True)
    one = block.forward(X[:1], keep=False)[0]
    many = block.forward(X, keep=False)[0][:1]
    print(f"a single token against the same row of a batch: {float((one - many).abs().max()):.3g}", flush=True)
    return [float(v) for v in losses]


if __name__ == "__main__":
    main()
