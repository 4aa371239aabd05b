"""What the feed-forward layer's training hands to the relay: the gradients' every bit, and models
without a hole."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import feed_forward as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def test_the_gradient_reaches_the_optimiser_whole(monkeypatch):
    """After the first step Adam's first moment is (1 - beta1) g, to two roundings of its own: also
    where g is far smaller than the spacing of the model's values."""
    moments, gradients = [], []
    step, backward = rs.RelayRun.step, ff.FeedForward.backward

    def recorded_step(run, *args, **kw):
        step(run, *args, **kw)
        if run.state:
            moments.append(run.state[0].clone())

    def recorded_backward(layer, rows, grads, *args, **kw):
        out = backward(layer, rows, grads, *args, **kw)
        gradients.append([v.clone() for v in layer.weights(grads)])
        return out

    monkeypatch.setattr(rs.RelayRun, "step", recorded_step)
    monkeypatch.setattr(ff.FeedForward, "backward", recorded_backward)
    n, d, f = 3, 32, 24
    ff.train(n=n, tokens=16, d=d, f=f, steps=1)
    layer = ff.FeedForward(n, 16, d, f)
    keep = 1 - float(torch.tensor(0.9))
    for m, g in zip(layer.weights(moments[0].reshape(n, -1)), gradients[0]):
        assert float(g.abs().max()) > 0
        # (the sign of what is handed over is the caller's)
        assert ((m.double().abs() - keep * g.double().abs()).abs() <= 2.0 ** -22 * keep * g.double().abs()).all()


def test_models_have_no_holes(monkeypatch):
    """With a width that leaves a gap before the next view, every coordinate of the models stays
    finite whatever fresh memory holds."""
    runs, step, empty = [], rs.RelayRun.step, torch.empty

    def recorded_step(run, *args, **kw):
        step(run, *args, **kw)
        runs.append(run)

    def dirty(*args, **kw):
        t = empty(*args, **kw)
        return t.fill_(float("nan")) if t.is_floating_point() else t

    monkeypatch.setattr(rs.RelayRun, "step", recorded_step)
    monkeypatch.setattr(torch, "empty", dirty)
    losses = ff.train(n=3, tokens=16, d=30, f=24, steps=3)
    assert all(loss == loss for loss in losses)
    for run in runs:
        assert run.x[:, :run.d].isfinite().all()


def test_gradients_by_hand_and_by_the_steps_objective_agree():
    """GradientRun on the quadratic's own gradient x - mu steps like RelayRun with Adam on that
    objective.  Of values up to 8 each step adds four roundings of 2^-21 at most, over 12 steps
    2.3e-5; the gradients stay at 1 and more, where Adam does not magnify that: twice as much."""
    n, d, lr, steps = 5, 38, 0.01, 12
    from paper_2110_04175_gb300 import workloads as wl
    whole = rs.RelayRun(n, d, wl.binary_tree(n), optimizer=("adam", 0.9, 0.99, 1e-8))
    apart = ff.GradientRun(n, d, wl.binary_tree(n))
    whole.init(0.5, 3, wl.identity_mix(n), 1.0, 3, 0.0)
    apart.init(0.5, 3)
    assert torch.equal(whole.x[:, :d], apart.x[:, :d])
    mu = whole.mu[:, :d]
    mu.copy_(whole.x[:, :d].sign() * (4 + torch.arange(n, device="cuda")[:, None] / 2))
    for _ in range(steps):
        apart.descent[:, :d] = mu - apart.x[:, :d]
        apart.step(lr)
        whole.step(lr, 0)
    assert float((whole.x[:, :d] - mu).abs().min()) > 1
    assert float((whole.x[:, :d] - apart.x[:, :d]).abs().max()) < 5e-5
    assert torch.equal(whole.counts, apart.relay.counts)
