"""The feed-forward example: its gradients against those of the same block in 64 bits, and that training lowers the loss."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ff():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward.py")
    spec = importlib.util.spec_from_file_location("feed_forward", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("tokens", [1, 33, 300])
def test_gradients_of_the_block(ff, tokens):
    """Against automatic differentiation in 64 bits of the block whose weights and kept activations are the codes' values.

    Bounds: h, dh, dg, du, dy are rounded to bfloat16 (2^-8 of each value, dy given) and scale * code is rounded to
    bfloat16 inside the products (2^-8 again), every sum in 32 bits.  dx passes through at most four such roundings on a path
    (dh, dg or du, and a product's operand twice), the weights' gradients through the same number, so that their norms are
    within 4 * 2^-8 of the exact gradient's; h enters dW_down as codes: it is taken from them in the comparison too."""
    import torch
    D, F = 192, 320
    torch.manual_seed(0)
    block = ff.FeedForward(D, F)
    x = torch.randn(tokens, D, device="cuda").bfloat16()
    dy = torch.randn(tokens, D, device="cuda").bfloat16()
    y, kept = block.forward(x)
    dx, grads = block.backward(dy, kept)
    xq, xs, hq, hs = kept
    w = {k: (q.double() * s.double()[:, None]).requires_grad_() for k, (q, s) in block.codes.items()}
    xe = (xq.double() * xs.double()[:, None]).requires_grad_()
    he = hq.double() * hs.double()[:, None]
    h = torch.nn.functional.silu(xe @ w["gate"].t()) * (xe @ w["up"].t())
    h_codes = h + (he - h).detach()                           # the value of the codes, the gradient of h
    out = xe + h_codes @ w["down"].t()
    out.backward(dy.double())
    bound = 4 * 2.0 ** -8
    assert (y.double() - (x.double() + he @ w["down"].t())).abs().max() <= 2.0 ** -7 * (1 + y.double().abs().max())
    assert (dx.double() - xe.grad).norm() <= bound * xe.grad.norm()
    for k in grads:
        assert (grads[k].double() - w[k].grad).norm() <= bound * w[k].grad.norm(), k


def test_training_lowers_the_loss(ff):
    block, losses, kept = ff.train(512, 128, 256, 20)
    assert np.isfinite(losses).all() and losses[-1] < 0.8 * losses[0], losses
    x = ff.restore(kept[0][:1], kept[1][:1])
    one = block.forward(x)[0]
    many = block.forward(x.expand(40, -1).contiguous())[0]    # the few-token form and the dense one agree
    assert (one.float() - many.float()).abs().max() <= 2.0 ** -6 * (1 + one.float().abs().max())
