"""What the step from one block to the next refuses, without a GPU."""
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


def _forward(lib, type_=0, n=2, tokens=10, d=64, x=_r(A), gate=_r(2 * A), residual=_r(3 * A), post=4 * A, ps=64, pre=5 * A,
             es=64, scale=6 * A, ss=64, eps=1e-5, total=_r(7 * A), y=_r(8 * A), rstd=9 * A, codes=10 * A, scales=11 * A):
    return lib.relay_block_norm(type_, n, tokens, d, x, gate, residual, post, ps, pre, es, scale, ss, eps, total, y, rstd, codes,
                                scales, None)


def _backward(lib, type_=0, n=2, tokens=10, d=64, dy=_r(A), over=_r(2 * A), x=_r(3 * A), gate=_r(4 * A), residual=_r(5 * A),
              post=6 * A, ps=64, pre=7 * A, es=64, scale=8 * A, ss=64, rstd=9 * A, lengths=10 * A, dx=_r(11 * A),
              dgate=_r(12 * A), dr=_r(13 * A), dpost=14 * A, dps=64, dpre=15 * A, des=64, dscale=16 * A, dss=64, work=17 * A,
              size=1 << 40):
    return lib.relay_block_norm_backward(type_, n, tokens, d, dy, over, x, gate, residual, post, ps, pre, es, scale, ss, rstd,
                                         lengths, dx, dgate, dr, dpost, dps, dpre, des, dscale, dss, work, size, None)


def test_sizes(lib):
    for type_, n, tokens, d, want in [(3, 1, 10, 64, BAD), (-1, 1, 10, 64, BAD), (0, 0, 10, 64, BAD), (0, 1, -1, 64, BAD),
                                      (0, 1, 10, 0, BAD), (0, 257, 1, 64, BIG), (0, 1, 1 << 30, 64, BIG),
                                      (0, 1, 1, 32769, BIG)]:
        assert _forward(lib, type_, n, tokens, d) == want
        assert _backward(lib, type_, n, tokens, d) == want
        if type_ == 0:
            assert lib.relay_block_norm_backward_workspace(n, tokens, d) == want


def test_forward(lib):
    for kw in (dict(x=None), dict(residual=None), dict(y=None), dict(post=None), dict(pre=None), dict(ps=-1), dict(es=-1),
               dict(ss=-1), dict(post=A + 2), dict(scale=A + 1), dict(eps=0.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(gate=_r(None)), dict(gate=_r(A + 1)), dict(total=_r(7 * A, 64)),
               dict(y=_r(A)), dict(y=_r(2 * A)), dict(y=_r(3 * A)), dict(y=_r(7 * A)), dict(total=_r(2 * A)),
               dict(total=_r(A, 64, 128)), dict(total=_r(3 * A, 700)), dict(rstd=A + 2), dict(codes=None),
               dict(scales=None), dict(codes=A + 8)):
        assert _forward(lib, **kw) == BAD, kw
    assert _forward(lib, tokens=0) == OK  # nothing to do


def test_backward(lib):
    need = lib.relay_block_norm_backward_workspace(2, 10, 64)
    assert need > 0
    for kw in (dict(dy=None), dict(x=None), dict(residual=None), dict(dx=None), dict(dr=None), dict(gate=None),
               dict(dgate=None), dict(scale=None), dict(post=None), dict(pre=None), dict(rstd=None), dict(rstd=A + 1),
               dict(lengths=A + 2), dict(dpost=None), dict(dpre=None), dict(dpost=15 * A), dict(dscale=14 * A),
               dict(dscale=15 * A), dict(dps=63), dict(des=63), dict(dss=63), dict(dscale=A + 2), dict(work=None),
               dict(work=A + 8), dict(size=need - 1), dict(dx=_r(A)), dict(dx=_r(2 * A)), dict(dx=_r(3 * A)),
               dict(dr=_r(5 * A)), dict(dgate=_r(4 * A)), dict(dgate=_r(11 * A)), dict(dr=_r(11 * A)), dict(dr=_r(12 * A)),
               dict(dx=_r(11 * A, 639)), dict(over=_r(A, -1)), dict(ps=-1)):
        assert _backward(lib, **kw) == BAD, kw


def test_binding_refuses_tensors_that_do_not_fit(lib):
    x, w = torch.zeros(2, 3, 64), torch.zeros(2, 64)
    with pytest.raises(ValueError, match="current CUDA device"):
        rs.relay_block_norm(x, x, w, w, x, x, 1e-5)
    for bad in (torch.zeros(3, 64), torch.zeros(2, 3, 64, dtype=torch.int32), None):
        with pytest.raises(ValueError):
            rs.relay_block_norm(bad, x, w, w, x, x, 1e-5)
        with pytest.raises(ValueError):
            rs.relay_block_norm_backward(bad, x, x, w, w, w, x, x, w, w, w)
    with pytest.raises(rs.RelayError):
        rs.relay_block_norm_backward_workspace(2, 3, 40000)


@pytest.mark.gpu
def test_binding_refuses_other_types_shapes_and_strides():
    x, w = torch.zeros(2, 3, 64, device="cuda"), torch.zeros(2, 64, device="cuda")
    r, y, t = (torch.zeros_like(x) for _ in range(3))
    for kw in (dict(gate=x.half()), dict(gate=x[:, :2]), dict(scale=w[:, :63]), dict(scale=w.half()),
               dict(rstd=torch.zeros(2, 3, device="cuda")), dict(checkpoint=rs.ActivationCheckpoint(2, 3, 63))):
        with pytest.raises(ValueError):
            rs.relay_block_norm(x, r, w, w, t, y, 1e-5, **kw)
    with pytest.raises(rs.RelayError):
        rs.relay_block_norm(x, r, w, w, t, t, 1e-5)
