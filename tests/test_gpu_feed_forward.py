"""The layer operators together: the feed-forward layer's gradients against
autograd in 64 bits, and its training through the relay."""
import pytest
import torch

import paper_2110_04175_gb300 as rs  # noqa: F401  (the package builds its library first)
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import feed_forward as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _reference(layer, rows, x, r, dout, dtotal, lengths):
    """Output and gradients by autograd in float64; padding has no part in the loss."""
    rows = rows.double().detach().requires_grad_()
    x = x.double().detach().requires_grad_()
    w, gate_up, down = layer.weights(rows)
    h = x + r.double()
    y = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + layer.eps) * w[:, None]
    g, u = layer._halves(y @ gate_up.transpose(1, 2))
    out = (torch.nn.functional.silu(g) * u) @ down.transpose(1, 2)
    used = torch.arange(x.shape[1], device=x.device)[None, :, None] < lengths[:, None, None]
    ((out * dout.double() + h * dtotal.double()) * used).sum().backward()
    return out.detach(), rows.grad, x.grad


@pytest.mark.parametrize("dtype,least", [(torch.float32, 0.0), (torch.bfloat16, 2.0 ** -7)], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n,tokens,d,f", [(3, 130, 96, 200), (2, 257, 100, 75)])
def test_gradients(dtype, least, n, tokens, d, f):
    """fp32: only the 8 bits are between the two.  A block's largest value is some 2.6 of its rms,
    and a step 1/127 to 1/64 of it, so a value is off by 0.6 % to 1.2 % of the rms; a gradient takes
    in at most three such values (the norm's row, gate, up), each with a slope of order 1: within
    4 %.  bf16 adds the roundings of the products' inputs and outputs, 2^-8 each."""
    torch.manual_seed(0)
    layer = ff.FeedForward(n, tokens, d, f, dtype=dtype)
    rows = torch.randn(n, layer.size + 3, device="cuda") * 0.1
    layer.weights(rows)[0].add_(1.0)
    x, r, dout, dtotal = (torch.randn(n, tokens, d, device="cuda").to(dtype) for _ in range(4))
    lengths = torch.tensor([tokens, 50, 1][:n], dtype=torch.int32, device="cuda")
    grads = torch.full_like(rows, float("nan"))
    out, h = layer.forward(rows, x, residual=r)
    used = torch.arange(tokens, device="cuda")[None, :, None] < lengths[:, None, None]
    dx = layer.backward(rows, grads, torch.where(used, dout, 0), torch.where(used, dtotal, 0), lengths)
    want_out, want_rows, want_dx = _reference(layer, rows, x, r, dout, dtotal, lengths)

    def off(got, want):
        return float((got.double() - want).norm() / want.norm())

    assert off(h, (x.double() + r.double())) <= 2.0 ** -24 + least
    assert off(out, want_out) <= 1e-5 + 4 * least
    assert off(dx, want_dx) <= 0.04 + 2 * least
    for got, want in zip(layer.weights(grads), layer.weights(want_rows)):
        assert off(got, want) <= 0.04 + 2 * least
    assert not dx[~used.expand_as(dx)].any()


def test_training_through_the_relay():
    """Workers of different data come down together; the same bits every time."""
    losses = ff.train(n=5, tokens=64, d=64, f=96, steps=40)
    assert losses[-1] < 0.25 * losses[0] and all(loss == loss for loss in losses)
    assert ff.train(n=5, tokens=64, d=64, f=96, steps=40) == losses
