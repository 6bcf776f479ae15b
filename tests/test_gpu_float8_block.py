"""The example of a block in 8-bit floating point runs, and its stages fit together: each gradient is that of the stage's formula
on the values the stage was given, within what the rounding to codes can do."""
import os
import sys

import numpy as np
import pytest

import float8_util as f

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def values(t):
    return t.double().cpu().numpy()


def near(got, want, a, b, da, db, what):
    """A product of codes against the product of what they were made from: each operand is off by half a step of its format
    (2^-4 of itself in e4m3, 2^-3 in e5m2, or of the smallest step where it is tiny beside its block: below 2^-9 of the block's
    largest value here), the result is rounded once."""
    bound = (np.abs(a) * da + np.abs(a).max() * 2.0 ** -16) @ (np.abs(b) * (1 + db)) + np.abs(a) @ (np.abs(b) * db + np.abs(b).max() * 2.0 ** -16)
    assert (np.abs(got - want) <= bound + 2.0 ** -8 * np.abs(want) + 1e-30).all(), what


@pytest.mark.parametrize("tokens,width,hidden", [(200, 256, 392), (70, 136, 520), (300, 250, 130)])
def test_block_forward_and_backward(tokens, width, hidden):
    import torch
    from float8_block import Block, mg
    gen = torch.Generator(device="cuda").manual_seed(3)
    block = Block(width, hidden, 0.2, gen)
    for k in block.norm:
        block.norm[k].copy_(1 + 0.2 * torch.randn(block.norm[k].shape, device="cuda", generator=gen))
    block.gate.copy_(torch.randn(1, width, device="cuda", generator=gen))
    x = torch.randn(tokens, width, device="cuda", generator=gen).bfloat16()
    dy = torch.randn(tokens, width, device="cuda", generator=gen).bfloat16()
    counter = torch.tensor([9], dtype=torch.int64, device="cuda")
    y, kept = block.forward(x, counter)
    dx, g = block.backward(dy, kept)
    assert mg.mipgemm_device_status() == mg.OK
    _, h1, s1, u, h2, s2, z, s3, _ = kept
    w = {k: values(v) for k, v in block.norm.items()}
    A, B = values(block.master["a"]), values(block.master["b"])
    E4, E5, bf = 2.0 ** -4, 2.0 ** -3, 2.0 ** -8

    def rms(v, weight):
        hat, _, rstd = f.hat(v, "rms", 1e-5)
        return hat * weight, hat, rstd
    # forward: norms to bfloat16's rounding, products to the codes'
    for got, source, weight in ((h1, x, w["in"]), (h2, u, w["mid"])):
        want = rms(values(source), weight)[0]
        assert (np.abs(values(got) - want) <= bf * np.abs(want) * 1.01 + 1e-4 * np.abs(want).max()).all()
    # (the codes come from the unrounded norm: half a unit of bfloat16 from its stored values)
    near(values(u), values(h1) @ A.T, values(h1), A.T, E4 + 2 * bf, E4, "u")
    near(values(z), values(h2) @ B.T, values(h2), B.T, E4 + 2 * bf, E4, "z")
    mask = f.kept(tokens, width, 0.2, block.seed, 9)
    zn, zhat, zr = rms(values(z), w["out"])
    gate = values(block.gate)
    want = values(x) + mask * gate * zn
    assert (np.abs(values(y) - want) <= bf * np.abs(want) * 1.01 + 1e-4 * np.abs(mask * gate * zn).max()).all()
    # backward, stage by stage from the values each was given
    d = values(dy)
    dz = f.through(d * mask * gate * w["out"], zhat, zr, "rms")
    near(values(g["b"]), dz.T @ values(h2), dz.T, values(h2), E5 + 2 * bf, E4, "dB")
    for got, terms in ((g["out"], d * mask * gate * zhat), (g["gate"][0], d * mask * zn)):
        want = terms.sum(axis=0)
        assert (np.abs(values(got) - want) <= 2e-4 * np.abs(terms).sum(axis=0) + bf * np.abs(want)).all()
    # the whole: norm by norm, the relative error of the codes' roundings adds up in quadrature over the stages; straight
    # through the roundings.  Each of the four products has two rounded operands, 2^-4 / sqrt 3 (e4m3) or 2^-3 / sqrt 3 (e5m2)
    # of themselves at most in the mean square: below 0.19 after two products in a row
    dh2 = dz @ B
    _, uhat, ur = rms(values(u), w["mid"])
    du = f.through(dh2 * w["mid"], uhat, ur, "rms")
    dh1 = du @ A
    _, xhat, xr = rms(values(x), w["in"])
    full = d + f.through(dh1 * w["in"], xhat, xr, "rms")
    for got, want in ((dx, full), (g["a"], du.T @ values(h1)), (g["mid"], (dh2 * uhat).sum(axis=0)), (g["in"], (dh1 * xhat).sum(axis=0))):
        assert np.linalg.norm(values(got) - want) <= 0.19 * np.linalg.norm(want)


def test_single_tokens_are_the_batch():
    """The few-token and the dense kernel sum in other orders; their 16-bit results differ by roundings, and by the codes of
    the middle norm that such a rounding tips over (a step of 2^-3 of an element for few of them)."""
    import torch
    from float8_block import Block
    block = Block(384, 640, 0.0, torch.Generator(device="cuda").manual_seed(4))
    x = torch.randn(70, 384, device="cuda").bfloat16()
    together = block.forward(x, train=False)[0].float()
    apart = torch.cat([block.forward(x[i:i + 1].contiguous(), train=False)[0] for i in range(70)]).float()
    assert float((together - apart).norm()) <= 0.03 * float(together.norm())


def test_example_runs(capsys, monkeypatch):
    import float8_block
    monkeypatch.setattr(sys, "argv", ["float8_block.py", "--tokens", "130", "--width", "256", "--hidden", "512"])
    float8_block.main()
    assert "8 tokens one by one" in capsys.readouterr().out
