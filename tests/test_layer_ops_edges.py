"""The operators around the attention where they could go wrong and tests/test_layer_ops.py does not look: values that are not finite in the
last rows of weights, products walked in parts, the precision that each number of rows has, and calls that must not reach a kernel."""
import pytest
import torch

from paper_2511_20426_amd import binding as B
from tests.test_layer_ops import DEV, _act, _gen, _normal


def _given_gradients(g, u, dh, act):
    """dg and du of saved projections, in 64 bits"""
    g = g.double().requires_grad_()
    a = _act(g, act)
    slope = torch.autograd.grad(a.sum(), g)[0]
    return dh * u.double() * slope, dh * a.detach()


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["gate", "up"])
@pytest.mark.parametrize("F", [72, 136, 256])
@pytest.mark.parametrize("M", [3, 4, 5, 8, 16, 17, 20, 32, 40])
def test_an_infinity_in_the_last_row_of_weights(M, F, which):
    """... is an infinity in its column of dX, of the sign of its gradient, and nowhere else, for any number of rows and of columns f."""
    from paper_2511_20426_amd.runner import gated_linear_backward, gated_linear_train
    gen, K = _gen(M + F), 128
    x, wg, wu, dh = _normal(gen, M, K), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, F, K, scale=K ** -0.5), _normal(gen, M, F)
    _, saved = gated_linear_train(x, wg, wu)
    xd, gd, ud = (t.double().cpu() for t in (x, wg, wu))
    dg, du = _given_gradients(xd @ gd.T, xd @ ud.T, dh.double().cpu(), "silu")
    (wg if which == "gate" else wu)[F - 1, 5] = float("inf")
    dx, dwg, dwu = (t.double().cpu() for t in gated_linear_backward(dh, x, wg, wu, saved))
    d = (dg if which == "gate" else du)[:, F - 1]
    assert (d != 0).all() and (dx[:, 5] == d.sign() * float("inf")).all()
    dx[:, 5] = 0
    assert all(t.isfinite().all() for t in (dx, dwg, dwu))
