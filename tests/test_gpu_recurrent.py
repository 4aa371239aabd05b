"""The operators of a recurrent block together: its gradients against autograd in 64 bits, sequences in stretches and
token by token, the orthogonal step in front of the relay, and a training run."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import feed_forward as ff
from paper_2110_04175_gb300 import recurrent
from paper_2110_04175_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _rms(x, eps):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)


def _reference(block, rows, r, initial, begins):
    """(out, last state) in the tensors' own precision, token by token."""
    w = block.weights(rows)
    y = _rms(r, block.eps) * w["norm"][:, None]
    forget, value, gate = block._thirds(y @ w["mix"].transpose(1, 2))
    f, h, states = torch.sigmoid(forget), initial, []
    for t in range(r.shape[1]):
        h = torch.where(begins[:, t, None] != 0, 0.0, f[:, t] * h) + (1 - f[:, t]) * value[:, t]
        states.append(h)
    mixed = torch.nn.functional.silu(gate) * torch.stack(states, 1)
    x = mixed @ w["mixed"].transpose(1, 2)
    total = w["scale"][:, None] * r + _rms(x, block.eps) * w["post"][:, None]
    g, u = block._halves((_rms(total, block.eps) * w["pre"][:, None]) @ w["gate_up"].transpose(1, 2))
    return total + (torch.nn.functional.silu(g) * u) @ w["down"].transpose(1, 2), h


def _model(block, seed=0, size=0.2):
    torch.manual_seed(seed)
    rows = torch.randn(block.n, block.size + 3, device="cuda") * size
    for name in block.VECTORS:
        block.weights(rows)[name].add_(1.0)
    return rows


def _off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("n,tokens,d,f", [(3, 70, 48, 40), (2, 131, 100, 75)])
def test_gradients(n, tokens, d, f):
    """fp32: only the 8 bits are between the two.  A value put away in 8 bits is off by 0.6 % to 1.2 % of its
    block's rms; a weight's gradient takes in at most four such values (its own inputs, the gate, up and the
    norm's rows), each with a slope of order 1: within 5 %.  What comes from rows alone (the post norm, the
    scale, the pre norm, by way of gate and up in 8 bits) is within 3 %."""
    block = recurrent.RecurrentBlock(n, tokens, d, f, dtype=torch.float32)
    rows = _model(block)
    r, dout = (torch.randn(n, tokens, d, device="cuda") for _ in range(2))
    initial, dlast = torch.randn(n, f, device="cuda"), torch.randn(n, f, device="cuda")
    begins = (torch.rand(n, tokens, device="cuda") < 0.05).to(torch.uint8)
    begins[:, 0] = 0
    last, dinitial, grads = torch.empty_like(initial), torch.empty_like(initial), torch.full_like(rows, float("nan"))
    out = block.forward(rows, r, initial=initial, last=last, begins=begins).clone()
    dr = block.backward(rows, grads, dout, dlast=dlast, dinitial=dinitial)
    wide = [x.double().requires_grad_() for x in (rows, r, initial)]
    want, want_last = _reference(block, *wide, begins)
    ((want * dout.double()).sum() + (want_last * dlast.double()).sum()).backward()
    assert _off(out, want.detach()) < 1e-5 and _off(last, want_last.detach()) < 1e-5
    assert _off(dr, wide[1].grad) < 0.05 and _off(dinitial, wide[2].grad) < 0.05
    for name, got in block.weights(grads).items():
        assert _off(got, block.weights(wide[0].grad)[name]) < 0.05, name


def test_lengths_leave_padding_out():
    n, tokens, d, f = 3, 60, 40, 24
    block = recurrent.RecurrentBlock(n, tokens, d, f, dtype=torch.float32)
    rows = _model(block)
    r, dout = (torch.randn(n, tokens, d, device="cuda") for _ in range(2))
    lengths = torch.tensor([tokens, 17, 0], dtype=torch.int32, device="cuda")
    used = torch.arange(tokens, device="cuda")[None, :, None] < lengths[:, None, None]
    grads, got = [], []
    for fill in (0.0, 50.0):
        g = torch.empty_like(rows)
        block.forward(rows, torch.where(used, r, fill), lengths=lengths)
        dr = block.backward(rows, g, torch.where(used, dout, 0.0))
        grads.append(g), got.append(torch.where(used, dr, 0.0).clone())
        assert not dr[~used.expand_as(dr)].any()
    assert torch.equal(got[0], got[1])
    for name, a in block.weights(grads[0]).items():
        assert torch.equal(a, block.weights(grads[1])[name]), name


@pytest.mark.parametrize("cuts", [[0, 30, 64], [0, 1, 2, 3, 64], list(range(65))], ids=["two", "few", "tokens"])
def test_stretches_and_single_tokens(cuts):
    """Generation: the same outputs as in one call, the state handed on in its own place."""
    n, d, f = 4, 96, 64
    whole = recurrent.RecurrentBlock(n, 64, d, f, dtype=torch.float32)
    rows = _model(whole)
    r = torch.randn(n, 64, d, device="cuda")
    want = whole.forward(rows, r).clone()
    state, blocks, out = torch.zeros(n, f, device="cuda"), {}, []
    for a, b in zip(cuts, cuts[1:]):
        block = blocks.setdefault(b - a, recurrent.RecurrentBlock(n, b - a, d, f, dtype=torch.float32))
        out.append(block.forward(rows, r[:, a:b], initial=state, last=state).clone())
    # fp32 products of other shapes and runs of other lengths: a few roundings of 2^-24 in each of eight operators
    assert _off(torch.cat(out, 1), want.double()) < 1e-5


def test_a_step_in_a_graph():
    """Forward and backward captured together and replayed on new inputs: the bits of eager calls."""
    n, tokens, d, f = 2, 50, 64, 48
    block = recurrent.RecurrentBlock(n, tokens, d, f)
    rows = _model(block)
    r, dout = (torch.randn(n, tokens, d, device="cuda").bfloat16() for _ in range(2))
    grads = torch.zeros_like(rows)
    for _ in range(2):  # the libraries' own workspaces
        block.forward(rows, r)
        block.backward(rows, grads, dout)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block.forward(rows, r)
        block.backward(rows, grads, dout)
    r.copy_(torch.randn(n, tokens, d, device="cuda"))
    graph.replay()
    got = out.clone(), grads.clone(), block.dr.clone()
    eager = block.forward(rows, r)
    grads.zero_()
    block.backward(rows, grads, dout)
    torch.cuda.synchronize()
    assert torch.equal(got[0], eager) and torch.equal(got[1], grads) and torch.equal(got[2], block.dr)


def test_orthogonal_steps_go_into_the_relay():
    """One step from equal models: the vectors move by Adam's step, which is lr sign(g) at first, the matrices by
    lr times the orthogonal update of (1 + momentum) (-g), and the relay joins them as it does any step."""
    n, rows, columns, lr = 3, 40, 24, 0.01
    size = 64 + rows * columns

    def matrices(x):
        return [x[:, 64:size].unflatten(1, (rows, columns))]

    run = ff.GradientRun(n, size, wl.binary_tree(n), matrices=matrices)
    plain = ff.GradientRun(n, size, wl.binary_tree(n))
    for which in (run, plain):
        which.init(0.1, 0)
    start = run.x.clone()
    g = torch.randn(n, size, device="cuda")
    run.descent[:, :size].copy_(-g)
    plain.descent[:, :size].copy_(-g)
    want = torch.empty(n, rows, columns, device="cuda")
    work = torch.empty(rs.relay_orthogonalise_workspace(n, rows, columns), dtype=torch.uint8, device="cuda")
    m = -matrices(g)[0]
    rs.relay_orthogonalise(m + 0.95 * m, want, work, scale=lr * (rows / columns) ** 0.5)
    run.step(lr)
    plain.step(lr)
    assert torch.equal(run.x[:, :64], plain.x[:, :64])
    assert torch.equal(run.velocity[:, 64:size], -g[:, 64:size])
    # the centre holds x + step; 0.95 m and the sum may round otherwise in one call: 2^-23 times 485
    step = matrices(run.relay.mu - start)[0]
    assert float((step - want).abs().max()) < 1e-4 * lr + 2.0 ** -24
    run.init(0.1, 0)
    assert not run.velocity.any()


def test_training_runs():
    losses = recurrent.train(n=5, tokens=64, d=48, f=40, steps=12)
    assert all(loss == loss for loss in losses)
    assert recurrent.train(n=5, tokens=64, d=48, f=40, steps=12) == losses
