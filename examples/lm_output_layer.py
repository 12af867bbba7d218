"""A model's output layer from training to serving, on synthetic data: states of which each knows its word more or less, learnt through the cross entropy
over the vocabulary (whose logits are never stored), then stored in 4 bits with a scale per group, loaded, scored and asked for one token at a time.

    python examples/lm_output_layer.py [--steps K] [--tokens M] [--width N] [--words P]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_13313_amd import lm  # noqa: E402


class Loss(torch.autograd.Function):
    """The mean cross entropy of the layer, for torch's autograd: the losses and the logarithms of the sums are all that is kept."""
    @staticmethod
    def forward(ctx, x, w, y):
        loss, lse = lm.cross_entropy(x, w, y)
        ctx.save_for_backward(x, w, y, lse)
        ctx.learnt = (y != lm.IGNORE).sum()
        return loss.sum() / ctx.learnt

    @staticmethod
    def backward(ctx, g):
        x, w, y, lse = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dw = lm.cross_entropy_backward((g / ctx.learnt).expand(len(y)), x, w, y, lse, need_dx=need[0], need_dw=need[1])
        return dx, dw, None


def train(x, y, words, steps, lr=4.0):
    """Gradient descent; the weights are kept in 32 bits and multiplied in 16."""
    master = torch.zeros((words, x.shape[1]), device=x.device)
    losses = []
    for _ in range(steps):
        w = master.bfloat16().requires_grad_()
        loss = Loss.apply(x, w, y)
        loss.backward()
        master -= lr * w.grad.float()
        losses.append(loss.detach())
    return master, torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=512)
    ap.add_argument("--words", type=int, default=8000)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    directions = torch.randn((a.words, a.width), device="cuda", generator=gen) / a.width ** 0.5
    y = torch.randint(0, a.words, (a.tokens,), device="cuda", generator=gen)
    x = (torch.randn((a.tokens, a.width), device="cuda", generator=gen) + 16 * directions[y]).bfloat16()
    y[::17] = lm.IGNORE                                              # (padding)
    master, losses = train(x, y, a.words, a.steps)
    print(f"cross entropy: {losses[0]:.3f} at first, {losses[-1]:.3f} after {a.steps} steps")

    # stored as codes, scales and zero points, and laid out again as a server would on loading them
    served = lm.pack(*lm.unpack(lm.quantize(master, group=64, zeros=True)), n=a.width, group=64)
    bits = 8 * served.data.numel() / master.numel()
    back = lm.dequantize(served, torch.bfloat16)
    scored = lm.cross_entropy(x, back, y)[0].sum().item() / (y != lm.IGNORE).sum().item()
    logits = torch.cat([lm.linear(x[i:i + 1], served) for i in range(64)])
    prompt = lm.linear(x[:64], served)
    off = (logits.float() - prompt.float()).abs().max().item() / prompt.float().abs().max().item()
    print(f"stored at {bits:.2f} bits a weight: cross entropy {scored:.3f}; logits token by token within {off:.4f} of the prompt's at once")
    return losses, scored, off


if __name__ == "__main__":
    main()
