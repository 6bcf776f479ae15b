"""A gated feed-forward block on 8-bit codes: trained for some steps, then run for single tokens.

    python3 examples/feed_forward.py [--tokens 4096] [--width 1024] [--hidden 4096] [--steps 30]

The block is  y = x + down(silu(gate(x)) * up(x)).  Weights are held as signed codes with a scale per output, next to the
32-bit master copies that the optimiser updates; tokens are brought to codes with a scale per token.  What a training step
keeps between its forward and backward pass are the codes of x and of h (a byte an element), not the pre-activations: those
are computed again from the codes inside the gradient's kernel.  The gradient passes through the rounding to codes as if it
were the identity."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2506_11728_b200 import binding as mg

BF16, F32 = mg.TYPES["bf16"], mg.TYPES["f32"]
SILU = mg.ACTIVATIONS["silu"]


def quantize(x):
    """Rows of x (bfloat16 or float32) as codes and a scale each."""
    M, N = x.shape
    q = torch.empty(M, N, dtype=torch.int8, device=x.device)
    s = torch.empty(M, dtype=torch.float32, device=x.device)
    mg.mipgemm_quantize_rows(BF16 if x.dtype == torch.bfloat16 else F32, M, N, x, N, q, N, s)
    return q, s


def product(a, b, b_scale, out, transposed=False, accumulate=False):
    """out (+)= a diag(b_scale) b, or a^T diag(b_scale) b: a bfloat16, b codes, b_scale one for each row of b."""
    K, N = b.shape
    M = out.shape[0]
    mg.mipgemm_bf16s8_product(BF16 if out.dtype == torch.bfloat16 else F32, mg.MN_CONTIGUOUS if transposed else mg.K_CONTIGUOUS, M, N, K,
                              a, a.shape[1], b, N, b_scale, out, N, accumulate)
    return out


class FeedForward:
    def __init__(self, width, hidden, generator=None):
        def master(rows, cols):
            return torch.randn(rows, cols, device="cuda", generator=generator) / cols ** 0.5
        self.width, self.hidden = width, hidden
        self.master = {"gate": master(hidden, width), "up": master(hidden, width), "down": master(width, hidden)}
        self.lay_out()

    def lay_out(self):
        """Codes of the master weights, one scale for each output."""
        self.codes = {k: quantize(w) for k, w in self.master.items()}

    def forward(self, x):
        """y and what the backward pass needs: any number of tokens (rows of x), one included."""
        M, D, F = x.shape[0], self.width, self.hidden
        (wg, sg), (wu, su), (wd, sd) = (self.codes[k] for k in ("gate", "up", "down"))
        xq, xs = quantize(x)
        h = torch.empty(M, F, dtype=torch.bfloat16, device=x.device)
        mg.mipgemm_s8s8_gated(BF16, SILU, M, F, D, xq, D, xs, wg, D, sg, wu, D, su, h, F)
        hq, hs = quantize(h)
        y = torch.empty_like(x)
        mg.mipgemm_s8s8_linear(BF16, mg.ACTIVATIONS["none"], M, D, F, hq, F, hs, wd, F, sd, None, x, D, y, D)
        return y, (xq, xs, hq, hs)

    def backward(self, dy, kept):
        """dx and the gradients of the three master weights."""
        xq, xs, hq, hs = kept
        M, D, F = dy.shape[0], self.width, self.hidden
        (wg, sg), (wu, su), (wd, sd) = (self.codes[k] for k in ("gate", "up", "down"))
        dh, dg, du = (torch.empty(M, F, dtype=torch.bfloat16, device=dy.device) for _ in range(3))
        product(dy, wd, sd, dh)
        mg.mipgemm_s8s8_gated_grad(BF16, SILU, M, F, D, xq, D, xs, wg, D, sg, wu, D, su, dh, F, dg, F, du, F)
        dx = dy.float()
        product(dg, wg, sg, dx, accumulate=True)
        product(du, wu, su, dx, accumulate=True)
        grads = {k: torch.empty_like(w) for k, w in self.master.items()}
        product(dg, xq, xs, grads["gate"], transposed=True)
        product(du, xq, xs, grads["up"], transposed=True)
        product(dy, hq, hs, grads["down"], transposed=True)
        return dx, grads

    def step(self, grads, rate):
        for k, w in self.master.items():
            w.sub_(grads[k], alpha=rate)
        self.lay_out()


def restore(q, s):
    """The bfloat16 rows that the codes stand for (a check-pointed activation read back)."""
    x = torch.empty(q.shape, dtype=torch.bfloat16, device=q.device)
    mg.mipgemm_dequantize_rows(BF16, q.shape[0], q.shape[1], q, q.shape[1], s, x, q.shape[1])
    return x


def train(tokens, width, hidden, steps, rate=0.2, seed=0):
    """Fits a block to another one's outputs; returns the block and the loss of every step."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher, block = FeedForward(width, hidden, g), FeedForward(width, hidden, g)
    x = torch.randn(tokens, width, device="cuda", generator=g).bfloat16()
    want = teacher.forward(x)[0]
    losses = []
    for _ in range(steps):
        y, kept = block.forward(x)
        error = y.float() - want.float()
        losses.append(error.square().mean())
        grads = block.backward((2 / tokens * error).bfloat16(), kept)[1]
        block.step(grads, rate)
    return block, [float(v) for v in losses], kept


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args()
    block, losses, kept = train(a.tokens, a.width, a.hidden, a.steps)
    print("loss: %.5f at the first step, %.5f at step %d" % (losses[0], losses[-1], a.steps))
    print("kept for the backward pass: %.1f MB as codes" % (sum(t.numel() * t.element_size() for t in kept) / 1e6))
    rows = restore(kept[0][:8], kept[1][:8])
    together = block.forward(rows)[0]
    apart = torch.cat([block.forward(rows[i:i + 1])[0] for i in range(len(rows))])      # token by token, as a decoder would
    print("8 tokens one by one: largest difference from the same tokens together %.4f" % float((together - apart).abs().max()))
    status = mg.mipgemm_device_status()
    assert status == mg.OK, mg.mipgemm_status_string(status)


if __name__ == "__main__":
    main()
