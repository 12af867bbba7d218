"""A layer in the microscaled 4-bit form from training to serving, on synthetic data: y = W0 x, learnt by a layer that multiplies quantised
activations, weights and gradients, then stored, loaded and asked for one token at a time.

    python examples/mx_linear.py [--steps K] [--tokens M] [--inputs N] [--outputs P]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2409_13313_amd import mx  # noqa: E402


def train(x, y, steps, lr=0.5):
    """Gradient descent on the mean square error; the weights are kept in 32 bits and quantised, both ways, once a step."""
    m, n = x.shape
    p = y.shape[1]
    w = torch.zeros((p, n), device=x.device)
    room = mx.alloc_workspace(m, n, p, x.device, backward=True)
    losses = []
    for _ in range(steps):
        by_row, by_col = mx.quantize(w, rows=True, cols=True)
        error = mx.linear(x, by_row, workspace=room) - y
        losses.append(error.float().square().mean())
        _, dw = mx.linear_backward(error / m, x, by_col, workspace=room)
        w -= lr * dw
    return w, torch.stack(losses).tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--inputs", type=int, default=512)
    ap.add_argument("--outputs", type=int, default=384)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    w0 = torch.randn((a.outputs, a.inputs), device="cuda", generator=gen) / a.inputs ** 0.5
    x = torch.randn((a.tokens, a.inputs), device="cuda", generator=gen).bfloat16()
    y = (x.float() @ w0.t()).bfloat16()
    w, losses = train(x, y, a.steps)
    print(f"mean square error: {losses[0]:.4f} at first, {losses[-1]:.4f} after {a.steps} steps")

    # stored as codes and scales, and laid out again as a server would on loading them
    codes, scales = mx.unpack(mx.quantize(w)[0])
    served = mx.pack(codes, scales, a.inputs)
    bits = 8 * (codes.numel() + scales.numel()) / w.numel()
    prompt = mx.linear(x[:64], served)
    one = torch.cat([mx.linear(x[i:i + 1], served) for i in range(64)])
    off = (one.float() - prompt.float()).abs().max().item()
    rel = (prompt.float() - y[:64].float()).norm().item() / y[:64].float().norm().item()
    print(f"served at {bits:.2f} bits a weight: error {rel:.3f} of the outputs, token by token within {off:.4f} of the prompt at once")
    back = mx.dequantize(served)
    print(f"weights read back: {(back - w0).norm().item() / w0.norm().item():.3f} off the ones that made the data")
    return losses, rel


if __name__ == "__main__":
    main()
