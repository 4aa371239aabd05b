"""What the feed-forward layer's training hands to the relay: models without a hole."""
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
