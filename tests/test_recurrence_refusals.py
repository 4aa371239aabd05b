"""What the recurrence refuses, without a GPU: every argument is checked on the host before anything is enqueued."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import layers

A = 1 << 20  # addresses that are never used, each a megabyte from the last
OK, BAD, BIG = rs.RELAY_OK, rs.RELAY_EINVAL, rs.RELAY_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    rs_build.build()
    return layers._library()


def _r(data, ws=640, ts=64):
    return layers._pack_rows(data or 0, ws, ts)


def test_sizes(lib):
    for type_, n, tokens, d, want in [(3, 1, 10, 64, BAD), (0, 0, 10, 64, BAD), (0, 1, -1, 64, BAD), (0, 1, 10, 0, BAD),
                                      (0, (1 << 20) + 1, 1, 64, BIG), (0, 1, 1 << 30, 64, BIG), (0, 1 << 19, 1 << 11, 1, BIG),
                                      (0, 1, 1, (1 << 24) + 1, BIG), (0, 1 << 20, 1, 1 << 17, BIG)]:
        assert lib.relay_recurrence(type_, n, tokens, d, _r(A), _r(2 * A), None, 0, None, None, _r(3 * A), None, 0, None, 0,
                                    None) == want
        assert lib.relay_recurrence_backward(type_, n, tokens, d, _r(A), _r(2 * A), _r(3 * A), _r(4 * A), None, 0, None, 0,
                                             None, None, _r(5 * A), _r(6 * A), None, 0, None, 0, None) == want
        if type_ == 0:
            assert lib.relay_recurrence_workspace(n, tokens, d) == want
    assert lib.relay_recurrence_workspace(257, 10, 64) == 0


def test_forward(lib):
    n, tokens, d = 2, 4000, 64
    need = lib.relay_recurrence_workspace(n, tokens, d)
    assert need > 0
    ws = tokens * d

    def call(gate=_r(A, ws), value=_r(2 * A, ws), initial=None, si=d, begins=None, lengths=None, out=_r(3 * A, ws), last=None,
             sl=d, work=4 * A, size=need, tokens=tokens):
        return lib.relay_recurrence(0, n, tokens, d, gate, value, initial, si, begins, lengths, out, last, sl, work, size, None)

    for kw in (dict(gate=None), dict(value=None), dict(out=None), dict(gate=_r(A + 1, ws)), dict(out=_r(3 * A, ws - 1)),
               dict(out=_r(3 * A, ws, 63)), dict(value=_r(2 * A, -1)), dict(out=_r(A, ws)), dict(out=_r(2 * A, ws)),
               dict(initial=5 * A + 2), dict(initial=5 * A, si=-1), dict(last=5 * A, sl=63), dict(last=5 * A + 1),
               dict(initial=5 * A, last=5 * A, si=0), dict(initial=5 * A, last=5 * A, sl=128), dict(lengths=6 * A + 2),
               dict(work=None), dict(work=4 * A + 8), dict(size=need - 1)):
        assert call(**kw) == BAD, kw
    assert call(tokens=0, work=None, size=0, gate=_r(None), value=_r(None), out=_r(None)) == OK  # nothing to do


def test_backward(lib):
    n, tokens, d = 2, 10, 64
    assert lib.relay_recurrence_workspace(n, tokens, d) == 0

    def call(dout=_r(A), gate=_r(2 * A), value=_r(3 * A), out=_r(4 * A), initial=None, si=d, dlast=None, sd=d, lengths=None,
             dgate=_r(5 * A), dvalue=_r(6 * A), dinitial=None, so=d):
        return lib.relay_recurrence_backward(0, n, tokens, d, dout, gate, value, out, initial, si, dlast, sd, None, lengths,
                                             dgate, dvalue, dinitial, so, None, 0, None)

    for kw in (dict(dout=None), dict(gate=None), dict(value=None), dict(out=None), dict(dgate=None), dict(dvalue=None),
               dict(dgate=_r(A)), dict(dgate=_r(2 * A)), dict(dvalue=_r(3 * A)), dict(dvalue=_r(4 * A)),
               dict(dvalue=_r(5 * A)), dict(dgate=_r(5 * A, 639)), dict(initial=7 * A, dinitial=7 * A),
               dict(dlast=7 * A, dinitial=7 * A, sd=128), dict(dinitial=7 * A, so=63), dict(dlast=7 * A + 1),
               dict(lengths=7 * A + 1), dict(initial=7 * A, si=-1)):
        assert call(**kw) == BAD, kw


def test_binding_refuses_tensors_that_do_not_fit(lib):
    x, w = torch.zeros(2, 3, 64), torch.empty(0, dtype=torch.uint8)
    with pytest.raises(ValueError, match="current CUDA device"):
        rs.relay_recurrence(x, x, x, w)
    for bad in (torch.zeros(3, 64), torch.zeros(2, 3, 64, dtype=torch.int32), None):
        with pytest.raises(ValueError):
            rs.relay_recurrence(bad, x, x, w)
        with pytest.raises(ValueError):
            rs.relay_recurrence_backward(bad, x, x, x, x, x, w)
    with pytest.raises(rs.RelayError):
        rs.relay_recurrence_workspace(0, 3, 64)


@pytest.mark.gpu
def test_binding_refuses_other_types_shapes_and_strides():
    x, w = torch.zeros(2, 3, 64, device="cuda"), torch.empty(0, dtype=torch.uint8, device="cuda")
    y, s = torch.zeros_like(x), torch.zeros(2, 64, device="cuda")
    for kw in (dict(initial=s.half()), dict(initial=s[:, :63]), dict(last=s.t().contiguous().t()),
               dict(begins=torch.zeros(2, 3, device="cuda")), dict(begins=torch.zeros(2, 4, dtype=torch.uint8, device="cuda")),
               dict(begins=torch.zeros(2, 3, dtype=torch.bool, device="cuda")),
               dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(initial=s.cpu())):
        with pytest.raises(ValueError):
            rs.relay_recurrence(x, x, y, w, **kw)
    with pytest.raises(ValueError):
        rs.relay_recurrence(x, x.half(), y, w)
    with pytest.raises(ValueError):
        rs.relay_recurrence(x, x, y[:, :2], w)
    with pytest.raises(rs.RelayError):  # in place
        rs.relay_recurrence(x, y, x, w)
