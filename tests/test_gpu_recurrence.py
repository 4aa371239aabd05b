"""The gated linear recurrence on the GPU against its definition in 64 bits: types, layouts, sizes around a warp's
channels and runs, segments, sequences that begin anywhere, lengths that leave a worker empty, states, values that are
not numbers, offsets past 32 bits, streams and graphs."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

from . import layers_util as lu
from . import recurrence_util as ru
from .layers_util import LEAST, ROUND, TYPES, np64, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _held(values, dtype):
    return np64(torch.from_numpy(values).to(dtype))


def _inputs(seed, n, T, d, dtype):
    """Gates with memories from one token to a thousand, and values, as the type holds them."""
    r = np.random.default_rng(seed)
    gate = r.standard_normal((n, T, d)) + r.uniform(-2, 7, d)
    return _held(gate, dtype), _held(r.standard_normal((n, T, d)) * np.where(r.random(d) < 0.1, 20, 1), dtype)


def _work(n, T, d):
    return torch.empty(rs.relay_recurrence_workspace(n, T, d), dtype=torch.uint8, device="cuda")


def _cuda(x, dtype):
    return None if x is None else torch.from_numpy(np.asarray(x)).to(dtype).cuda()


def _rounded(want, dtype, bound):
    return bound + ROUND[dtype] * (np.abs(want) + bound) + LEAST[dtype]


def _options(seed, n, T, d, what):
    """initial, begins and lengths as `what` asks for them."""
    r = np.random.default_rng(seed + 1)
    initial = r.standard_normal((n, d)).astype(np.float32) if "state" in what else None
    begins = lengths = None
    if "packed" in what:
        begins = (r.random((n, T)) < 5 / (T + 5)).astype(np.uint8) * 7
        begins[0, 0], begins[-1, T - 1] = 1, 255
    if "lengths" in what:
        lengths = r.integers(0, T + 1, n).astype(np.int32)
        lengths[0], lengths[-1] = T + 3, (0 if n > 1 else T // 2)
        if n > 2:
            lengths[1] = -4
    return initial, begins, lengths


def _check(n, T, d, dtype, layout="dense", what=("state",), seed=0):
    g, v = _inputs(seed, n, T, d, dtype)
    initial, begins, lengths = _options(seed, n, T, d, what)
    gate, value = lu.rows(g, dtype, layout)[0], lu.rows(v, dtype, layout)[0]
    out, buf = lu.empty_rows(n, T, d, dtype, layout)
    state = None if initial is None else _cuda(np.pad(initial, ((0, 0), (3, 2))), torch.float32)[:, 3:3 + d]
    last = torch.full((n, d + 4), 77.0, device="cuda")[:, 1:1 + d]
    kw = dict(begins=_cuda(begins, torch.uint8), lengths=_cuda(lengths, torch.int32))
    rs.relay_recurrence(gate, value, out, _work(n, T, d), initial=state, last=last, **kw)
    h, end, bound, end_bound = ru.forward(g, v, initial, begins, lengths)
    within(out, h, _rounded(h, dtype, bound))
    within(last, end, end_bound + 2.0 ** -150)
    assert lu.only_rows_written(out, buf)

    r = np.random.default_rng(seed + 2)
    dh = _held(r.standard_normal((n, T, d)) * 0.1, dtype)
    dlast = r.standard_normal((n, d)).astype(np.float32) if "state" in what else None
    dgate, dbuf = lu.empty_rows(n, T, d, dtype, layout)
    dvalue, dbuf2 = lu.empty_rows(n, T, d, dtype, layout)
    dinitial = torch.full((n, d), 77.0, device="cuda")
    kept = np64(out)
    rs.relay_recurrence_backward(lu.rows(dh, dtype, layout)[0], gate, value, out, dgate, dvalue, _work(n, T, d),
                                 initial=state, dlast=_cuda(dlast, torch.float32), dinitial=dinitial, **kw)
    dg, dv, dm, bg, bv, bm = ru.backward(dh, g, v, kept, initial, dlast, begins, lengths)
    within(dgate, dg, _rounded(dg, dtype, bg))
    within(dvalue, dv, _rounded(dv, dtype, bv))
    within(dinitial, dm, bm + 2.0 ** -150)
    assert lu.only_rows_written(dgate, dbuf) and lu.only_rows_written(dvalue, dbuf2)
    return gate, value, out, last


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
def test_types_and_layouts(dtype, layout):
    for n, T, d in [(1, 1, 1), (3, 1, 70), (2, 2, 64), (3, 9, 66), (2, 33, 129), (5, 130, 31), (2, 300, 96)]:
        _check(n, T, d, dtype, layout, ("state", "packed", "lengths"), seed=T)


@pytest.mark.parametrize("what", [(), ("state",), ("packed",), ("lengths",), ("state", "packed"), ("packed", "lengths")],
                         ids=lambda w: "+".join(w) or "plain")
def test_options(what):
    for T in (4, 8, 9, 16, 17, 31, 32, 33, 127, 128, 129, 257):
        _check(3, T, 72, torch.bfloat16, what=what, seed=T)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("n,T,d", [(1, 1024, 64), (1, 5003, 33), (2, 2050, 130), (1, 1500, 9728), (7, 1025, 100)])
def test_long_sequences(dtype, n, T, d):
    """Few channels and many tokens: segments; and where there is just one."""
    _check(n, T, d, dtype, what=("state", "packed", "lengths"), seed=d)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("n,T,d", [(1, 2060, 200), (2, 1033, 136), (20, 300, 128), (3, 700, 1024), (1, 530, 4096), (65, 290, 64),
                                   (3, 261, 3200), (150, 140, 64), (1, 13000, 64), (2, 6200, 72)])
def test_clusters_and_segments_of_aligned_rows(dtype, n, T, d):
    """Rows by tensor copies: one, four and eight CTAs a strip, rounds that end anywhere, and segments."""
    if n * T * d > 2e6 and dtype is torch.float16:
        pytest.skip("as bf16")
    _check(n, T, d, dtype, what=("state", "packed", "lengths"), seed=d)
    if n * T * d < 3e5:
        _check(n, T, d, dtype, what=(), seed=d)


def test_many_sequences_of_one_token():
    _check(5000, 1, 40, torch.bfloat16, what=("state",))
    _check(70000, 2, 3, torch.float32, what=("state", "lengths"))


def test_no_tokens_hand_the_state_on():
    n, d = 3, 50
    x = torch.empty(n, 0, d, device="cuda", dtype=torch.bfloat16)
    state, last = torch.randn(n, d, device="cuda"), torch.full((n, d), 9.0, device="cuda")
    rs.relay_recurrence(x, x, x, _work(n, 0, d), initial=state, last=last)
    assert torch.equal(last, state)
    rs.relay_recurrence(x, x, x, _work(n, 0, d), last=last)
    assert not last.any()
    rs.relay_recurrence_backward(x, x, x, x, x, x, _work(n, 0, d), dlast=state, dinitial=last)
    assert torch.equal(last, state)


@pytest.mark.parametrize("T,cuts,d", [(40, [0, 1, 13, 14, 40], 70), (2600, [0, 1100, 1101, 2600], 70),
                                      (2600, [0, 1100, 1101, 1250, 2600], 72)])
def test_stretches_go_on_from_the_state(T, cuts, d):
    """Token by token or in stretches, the state in its own place: the same rows as in one call, within the bounds."""
    n, dtype = 2, torch.float32
    g, v = _inputs(5, n, T, d, dtype)
    gate, value = _cuda(g, dtype), _cuda(v, dtype)
    state = torch.zeros(n, d, device="cuda")
    out = torch.empty_like(gate)
    for a, b in zip(cuts, cuts[1:]):
        rs.relay_recurrence(gate[:, a:b], value[:, a:b], out[:, a:b], _work(n, b - a, d), initial=state, last=state)
    h, end, bound, end_bound = ru.forward(g, v)
    within(out, h, _rounded(h, dtype, bound))
    within(state, end, end_bound)


@pytest.mark.parametrize("T,d", [(1, 40), (9, 33), (300, 64), (1100, 33), (13000, 64)])
def test_the_states_gradient_in_its_own_place(T, d):
    """dinitial over dlast: one warp, a CTA, a cluster, segments."""
    n, dtype = 2, torch.bfloat16
    g, v = _inputs(9, n, T, d, dtype)
    gate, value = _cuda(g, dtype), _cuda(v, dtype)
    dout, dlast = torch.randn_like(gate), torch.randn(n, d, device="cuda")
    out, dg, dv = (torch.empty_like(gate) for _ in range(3))
    rs.relay_recurrence(gate, value, out, _work(n, T, d))
    want = torch.empty_like(dlast)
    rs.relay_recurrence_backward(dout, gate, value, out, dg, dv, _work(n, T, d), dlast=dlast, dinitial=want)
    rs.relay_recurrence_backward(dout, gate, value, out, dg, dv, _work(n, T, d), dlast=dlast, dinitial=dlast)
    assert torch.equal(dlast, want)


@pytest.mark.parametrize("T", [20, 1100])
def test_nothing_passes_a_beginning(T):
    """Infinities and NaN before a beginning, in the padding and in a state that is not taken leave no trace."""
    n, d, dtype = 2, 40, torch.bfloat16
    g, v = _inputs(3, n, T, d, dtype)
    begins = np.zeros((n, T), np.uint8)
    begins[0, [0, 11]], begins[1, [3, T - 2]] = 1, 1
    lengths = np.array([T - 4, T], np.int32)
    bad_g, bad_v = g.copy(), v.copy()
    bad_g[0, 2, :5], bad_v[0, 5, 5:9], bad_v[0, 8, 9:12], bad_g[0, 9, 12:14] = np.nan, np.inf, np.nan, -np.inf
    bad_g[0, T - 4:], bad_v[0, T - 4:] = np.nan, np.inf
    initial = np.ones((n, d), np.float32)
    initial[0], initial[1, 4] = np.inf, np.nan
    kw = dict(begins=_cuda(begins, torch.uint8), lengths=_cuda(lengths, torch.int32))

    def run(g, v, initial):
        gate, value, out = _cuda(g, dtype), _cuda(v, dtype), torch.empty(n, T, d, device="cuda", dtype=dtype)
        last, state = torch.empty(n, d, device="cuda"), _cuda(initial, torch.float32)
        rs.relay_recurrence(gate, value, out, _work(n, T, d), initial=state, last=last, **kw)
        grads = [torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(last)]
        dout = torch.ones_like(gate)
        rs.relay_recurrence_backward(dout, gate, value, out, grads[0], grads[1], _work(n, T, d), initial=state,
                                     dinitial=grads[2], **kw)
        return out, last, *grads

    clean, dirty = run(g, v, np.ones((n, d))), run(bad_g, bad_v, initial)
    assert torch.equal(clean[1][:, 5:], dirty[1][:, 5:]) and torch.equal(clean[1][0], dirty[1][0])
    for a, b in zip(clean[:1] + clean[2:4], dirty[:1] + dirty[2:4]):
        assert torch.equal(a[0, 11:], b[0, 11:]) and torch.equal(a[1, 3:], b[1, 3:])
        assert not b[0, T - 4:].any()
    assert torch.isinf(dirty[0][0, 5, 5:9]).all() and not torch.isfinite(dirty[0][0, 5:11, 5:9]).any()
    assert torch.isnan(dirty[0][0, 2:11, :5]).all() and torch.isnan(dirty[0][1, :3, 4]).all()
    assert not dirty[4][0].any()  # what worker 0's state was is never taken


def test_gates_at_the_ends_of_the_range():
    """Gates that keep or forget everything, and the types' largest: no NaN, and the formula's values."""
    big = float(torch.finfo(torch.bfloat16).max)
    gates = [0.0, -0.0, 20.0, -20.0, 88.0, -88.0, 200.0, -200.0, big, -big, np.inf, -np.inf]
    for dtype in (torch.bfloat16, torch.float32):
        g = np.tile(np.array(gates), (1, 6, 1))
        v = np.arange(1.0, 7.0)[None, :, None] * np.ones((1, 6, len(gates)))
        out = torch.empty(1, 6, len(gates), device="cuda", dtype=dtype)
        rs.relay_recurrence(_cuda(g, dtype), _cuda(v, dtype), out, _work(1, 6, len(gates)))
        clipped = np.clip(g, -500, 500)
        h, _, bound, _ = ru.forward(clipped, v)
        # exponentials below fp32's normal numbers count as 0
        within(out, h, _rounded(h, dtype, bound) + 12 * 2.0 ** -126)


def test_repeated_rows_and_a_shared_state():
    """Inputs may repeat rows (stride 0): one gate for all tokens, one state for all workers."""
    n, T, d = 3, 50, 33
    g, v = _inputs(1, n, 1, d, torch.float32)[0], _inputs(2, n, T, d, torch.float32)[1]
    state = np.random.default_rng(0).standard_normal((1, d)).astype(np.float32)
    out = torch.empty(n, T, d, device="cuda")
    rs.relay_recurrence(_cuda(g, torch.float32).expand(n, T, d), _cuda(v, torch.float32), out, _work(n, T, d),
                        initial=_cuda(state, torch.float32).expand(n, d))
    h, _, bound, _ = ru.forward(np.repeat(g, T, 1), v, np.repeat(state, n, 0))
    within(out, h, _rounded(h, torch.float32, bound))


def test_gradients_agree_with_differences():
    """Central differences of the forward pass in fp32, in three random directions."""
    n, T, d = 2, 45, 20
    torch.manual_seed(0)
    gate, value, dout = (torch.randn(n, T, d, device="cuda") for _ in range(3))
    initial, dlast = torch.randn(n, d, device="cuda"), torch.randn(n, d, device="cuda")
    begins = (torch.rand(n, T, device="cuda") < 0.1).to(torch.uint8)

    def forward(gate, value, initial):
        out, last = torch.empty_like(gate), torch.empty_like(initial)
        rs.relay_recurrence(gate, value, out, _work(n, T, d), initial=initial, last=last, begins=begins)
        return out, last

    out, _ = forward(gate, value, initial)
    grads = [torch.empty_like(gate), torch.empty_like(gate), torch.empty_like(initial)]
    rs.relay_recurrence_backward(dout, gate, value, out, grads[0], grads[1], _work(n, T, d), initial=initial, dlast=dlast,
                                 dinitial=grads[2], begins=begins)
    for _ in range(3):
        steps = [torch.randn_like(x) for x in (gate, value, initial)]
        want = sum(float((g.double() * s.double()).sum()) for g, s in zip(grads, steps))
        eps, total = 2.0 ** -8, []
        for sign in (eps, -eps):
            h, last = forward(*(x + sign * s for x, s in zip((gate, value, initial), steps)))
            total.append(float((h.double() * dout.double()).sum() + (last.double() * dlast.double()).sum()))
        got = (total[0] - total[1]) / (2 * eps)
        # rounding: 2^-20 of some 40 (the sum's spread) over 2 eps; curvature: eps^2 of a third derivative
        # of the order of the sum of magnitudes (n T d = 1,800 terms): 5e-3 and 3e-2
        assert abs(got - want) < 0.1 + 1e-3 * abs(want)


@pytest.mark.parametrize("d", [100, 64], ids=["segments", "clusters"])
def test_the_same_bits_every_time_on_any_stream_and_in_a_graph(d):
    """Streams at once with a workspace each, and a captured call on new inputs."""
    n, T, dtype = 1, 4000, torch.bfloat16
    (g, v), (g2, v2) = _inputs(1, n, T, d, dtype), _inputs(2, n, T, d, dtype)
    gate, value = _cuda(g, dtype), _cuda(v, dtype)
    outs = [torch.empty_like(gate) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in outs]
    works = [_work(n, T, d) for _ in outs]
    torch.cuda.synchronize()
    for out, work, stream in zip(outs, works, streams):
        rs.relay_recurrence(gate, value, out, work, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    graph = torch.cuda.CUDAGraph()
    dg, dv = torch.empty_like(gate), torch.empty_like(gate)
    with torch.cuda.graph(graph):
        rs.relay_recurrence(gate, value, outs[0], works[0])
        rs.relay_recurrence_backward(outs[0], gate, value, outs[0], dg, dv, works[0])
    gate.copy_(_cuda(g2, dtype))
    value.copy_(_cuda(v2, dtype))
    graph.replay()
    want = [torch.empty_like(gate) for _ in range(3)]
    rs.relay_recurrence(gate, value, want[0], works[1])
    rs.relay_recurrence_backward(want[0], gate, value, want[0], want[1], want[2], works[1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((outs[0], dg, dv), want))


def test_past_32_bit_offsets():
    """Rows more than 2^31 elements apart."""
    far, T, d = (1 << 31) + 64, 3, 64
    buf = torch.zeros(far + T * d, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, T, d), (far, d, 1))
    g, v = _inputs(7, 2, T, d, torch.bfloat16)
    x.copy_(_cuda(g, torch.bfloat16))
    out, value = torch.empty(2, T, d, dtype=torch.bfloat16, device="cuda"), _cuda(v, torch.bfloat16)
    rs.relay_recurrence(x, value, out, _work(2, T, d))
    h, _, bound, _ = ru.forward(g, v)
    within(out, h, _rounded(h, torch.bfloat16, bound))
    rs.relay_recurrence(out, value, x, _work(2, T, d))
    h, _, bound, _ = ru.forward(np64(out), v)
    within(x, h, _rounded(h, torch.bfloat16, bound))
    assert not buf[T * d:far].any()
