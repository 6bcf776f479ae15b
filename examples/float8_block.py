"""A block of a transformer layer in 8-bit floating point, forward and backward, and token by token.

    python3 examples/float8_block.py [--tokens 2048] [--width 1024] [--hidden 4096]

    h1 = norm(x),  u = h1 A^T,  h2 = norm(u),  z = h2 B^T,  y = x + dropout(gate * norm(z))

The norms write codes with a scale for each 128 channels, which the products read; weights are codes with a scale for each
square of 128 x 128, so that the same codes serve both passes.  Backward, the gradients are brought to codes along their rows
(for the products with the weights) and along their columns (for the weights' gradients) in one reading.  The gradient passes
through the rounding to codes as if it were the identity.  The dropout mask is never stored: the backward pass draws it again."""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2506_11728_b200 import binding as mg

BF16, F32 = mg.TYPES["bf16"], mg.TYPES["f32"]
E4M3, E5M2 = mg.F8_FORMATS["e4m3"], mg.F8_FORMATS["e5m2"]
NONE, RMS = mg.NORMS["none"], mg.NORMS["rms"]
SQUARES, COLUMNS = mg.F8_BLOCKS["squares"], mg.F8_BLOCKS["columns"]
K, MN = mg.K_CONTIGUOUS, mg.MN_CONTIGUOUS


def blocks(n):
    return (n + 127) // 128


def both_ways(x, fmt):
    """Codes of x (bfloat16) along its rows and along its columns."""
    m, n = x.shape
    r, c = (torch.empty(m, n, dtype=torch.uint8, device=x.device) for _ in range(2))
    rs, cs = torch.empty(blocks(n), m, device=x.device), torch.empty(blocks(m), n, device=x.device)
    mg.mipgemm_f8_quantize(BF16, fmt, m, n, x, n, r, n, rs, m, c, n, cs, n)
    return (r, rs), (c, cs)


def squares(w):
    """Codes of a weight matrix (float32)."""
    m, n = w.shape
    q, s = torch.empty(m, n, dtype=torch.uint8, device=w.device), torch.empty(blocks(m), blocks(n), device=w.device)
    mg.mipgemm_f8_quantize_squares(F32, E4M3, m, n, w, n, q, n, s, blocks(n))
    return q, s


class Block:
    def __init__(self, width, hidden, drop=0.1, generator=None):
        self.width, self.hidden, self.drop, self.seed = width, hidden, drop, 1234
        self.master = {"a": torch.randn(hidden, width, device="cuda", generator=generator) / width ** 0.5,
                       "b": torch.randn(width, hidden, device="cuda", generator=generator) / hidden ** 0.5}
        self.norm = {"in": torch.ones(width, device="cuda"), "mid": torch.ones(hidden, device="cuda"), "out": torch.ones(width, device="cuda")}
        self.gate = torch.ones(1, width, dtype=torch.bfloat16, device="cuda")
        self.codes = {k: squares(w) for k, w in self.master.items()}

    def _normed(self, x, w, keep):
        """norm(x) as codes along the rows; with `keep` also as values, and the statistics, for the backward pass."""
        m, n = x.shape
        q, s = torch.empty(m, n, dtype=torch.uint8, device=x.device), torch.empty(blocks(n), m, device=x.device)
        h, stats = (torch.empty_like(x), torch.empty(m, 4, device=x.device)) if keep else (None, None)
        mg.mipgemm_norm_step(BF16, NONE, RMS, m, n, X=x, ldx=n, pre_weight=w, H=h, ldh=n, codes=mg.CODES["e4m3"], Q=q, ldq=n, q_scale=s, ldqs=m,
                             stats=stats)
        return (q, s), h, stats

    def _product(self, codes, name):
        (q, s), (w, ws) = codes, self.codes[name]
        (m, k), n = q.shape, w.shape[0]
        y = torch.empty(m, n, dtype=torch.bfloat16, device=q.device)
        mg.mipgemm_f8f8_product(BF16, E4M3, E4M3, K, K, SQUARES, m, n, k, q, k, s, m, w, k, ws, ws.shape[1], None, None, 0, y, n)
        return y

    def forward(self, x, counter=None, train=True):
        """y, and what the backward pass needs."""
        m, n = x.shape
        c1, h1, s1 = self._normed(x, self.norm["in"], train)
        u = self._product(c1, "a")
        c2, h2, s2 = self._normed(u, self.norm["mid"], train)
        z = self._product(c2, "b")
        y, s3 = torch.empty_like(x), torch.empty(m, 4, device=x.device) if train else None
        mg.mipgemm_norm_step(BF16, RMS, NONE, m, n, X=x, ldx=n, Z=z, ldz=n, post_weight=self.norm["out"], gate=self.gate, ldgate=n, gate_rows=m,
                             drop=self.drop if train else 0.0, seed=self.seed, counter=counter, Y=y, ldy=n, stats=s3)
        return y, (x, h1, s1, u, h2, s2, z, s3, counter)

    def _back(self, d, kept_h, name):
        """Gradients of a product's input and weights from that of its output."""
        m, n = d.shape
        (r, rs), (c, cs) = both_ways(d, E5M2)
        (w, ws), k = self.codes[name], kept_h.shape[1]
        _, (hc, hs) = both_ways(kept_h, E4M3)
        dh, dw = torch.empty_like(kept_h), torch.empty(n, k, device=d.device)
        mg.mipgemm_f8f8_product(BF16, E5M2, E4M3, K, MN, SQUARES, m, k, n, r, n, rs, m, w, k, ws, ws.shape[1], None, None, 0, dh, k)
        mg.mipgemm_f8f8_product(F32, E5M2, E4M3, MN, MN, COLUMNS, n, k, m, c, n, cs, n, hc, k, hs, k, None, None, 0, dw, k)
        return dh, dw

    def backward(self, dy, kept):
        """dx, and the gradients of the weights, the norms' weights and the gate."""
        x, h1, s1, u, h2, s2, z, s3, counter = kept
        m, n = dy.shape
        g = {"in": torch.empty(self.width, device=dy.device), "mid": torch.empty(self.hidden, device=dy.device), "out": torch.empty(self.width, device=dy.device),
             "gate": torch.empty_like(self.gate)}
        dz, dx = torch.empty_like(z), torch.empty_like(x)
        mg.mipgemm_norm_step_grad(BF16, RMS, NONE, m, n, dY=dy, lddy=n, Z=z, ldz=n, post_weight=self.norm["out"], gate=self.gate, ldgate=n, gate_rows=m,
                                  drop=self.drop, seed=self.seed, counter=counter, stats=s3, dZ=dz, lddz=n, dgate=g["gate"], lddgate=n,
                                  dpost_weight=g["out"])
        dh2, g["b"] = self._back(dz, h2, "b")
        du = torch.empty_like(u)
        mg.mipgemm_norm_step_grad(BF16, NONE, RMS, m, self.hidden, dH=dh2, lddh=self.hidden, Y=u, ldy=self.hidden, pre_weight=self.norm["mid"], stats=s2,
                                  dX=du, lddx=self.hidden, dpre_weight=g["mid"])
        dh1, g["a"] = self._back(du, h1, "a")
        mg.mipgemm_norm_step_grad(BF16, NONE, RMS, m, n, dY=dy, lddy=n, dH=dh1, lddh=n, Y=x, ldy=n, pre_weight=self.norm["in"], stats=s1, dX=dx, lddx=n,
                                  dpre_weight=g["in"])
        return dx, g


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    a = ap.parse_args()
    gen = torch.Generator(device="cuda").manual_seed(0)
    block = Block(a.width, a.hidden, generator=gen)
    x = torch.randn(a.tokens, a.width, device="cuda", generator=gen).bfloat16()
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    y, kept = block.forward(x, counter)
    dx, grads = block.backward(torch.randn(a.tokens, a.width, device="cuda", generator=gen).bfloat16(), kept)
    print("norms of the gradients: " + ", ".join("%s %.3f" % (k, float(v.float().norm())) for k, v in sorted(grads.items())))
    few = x[:8].contiguous()
    together = block.forward(few, train=False)[0]
    apart = torch.cat([block.forward(few[i:i + 1].contiguous(), train=False)[0] for i in range(8)])      # token by token, as a decoder would
    print("8 tokens one by one: largest difference from the same tokens together %.4f" % float((together - apart).abs().max()))
    status = mg.mipgemm_device_status()
    assert status == mg.OK, mg.mipgemm_status_string(status)


if __name__ == "__main__":
    main()
