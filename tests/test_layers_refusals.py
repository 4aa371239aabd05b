"""What the layer operators refuse, and their 8-bit format's rule, without a GPU:
every argument is checked on the host before anything is enqueued."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import layers

from . import layers_util as lu

A, B, C, D, E = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20)  # addresses that are never used
OK, BAD, BIG = rs.RELAY_OK, rs.RELAY_EINVAL, rs.RELAY_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    rs_build.build()
    return layers._library()


def _r(data, ws, ts):
    return layers._pack_rows(data or 0, ws, ts)


def test_header_and_library_agree(lib):
    text = open(os.path.join(rs_build.INCLUDE, "relaylayers.h")).read()
    names = set(re.findall(r"\b(relay_[a-z_]+)\s*\(", text))
    assert names == set(layers._SIGNATURES)
    for name in names:
        assert hasattr(lib, name) and hasattr(rs, name) or name == "relay_checkpoint_pitch"


def test_scale_rule_is_the_least_scale():
    """The carry of relaylayers.h's rule equals the search for the least scale that fits, at the step
    from scale to scale, at random magnitudes, and at both ends."""
    g = np.random.default_rng(0)
    e = np.arange(-149, 128)
    edge = np.ldexp(np.float64(1), e)
    near = np.concatenate([edge * f for f in (1, 1 - 2.0 ** -24, 1.9921875, 1.9921875 - 2.0 ** -23, 1.99, 1.9999999)])
    near = np.concatenate([near, np.abs(g.standard_normal(2000)) * np.exp2(g.integers(-130, 127, 2000)), [0.0]])
    most = near.astype(np.float32)
    most = most[np.isfinite(most)]
    bits = most.view(np.uint32).astype(np.int64)
    rule = np.minimum(255, np.maximum(7, (bits + 0x10000) >> 23))
    assert np.array_equal(rule, lu.scale_bytes(most.astype(np.float64)))


def test_sizes_and_types(lib):
    rows = _r(A, 640, 64)
    for type_, n, tokens, d, want in [(3, 1, 10, 64, BAD), (-1, 1, 10, 64, BAD), (0, 0, 10, 64, BAD),
                                      (0, 1, -1, 64, BAD), (0, 1, 10, 0, BAD), (0, 257, 1, 64, BIG),
                                      (0, 1, 1 << 30, 64, BIG), (0, 16, 1 << 26, 64, BIG),
                                      (0, 1, 1, (1 << 24) + 1, BIG), (0, 1, 1 << 62, 64, BIG)]:
        assert lib.relay_checkpoint_pack(type_, n, tokens, d, rows, B, C, None) == want
        assert lib.relay_gated(type_, n, tokens, d, rows, rows, _r(B, 640, 64), None, None, None, None, None) == want
        assert lib.relay_rms_norm(type_, n, tokens, d, rows, None, B, 64, 1e-5, None, _r(C, 640, 64), None, None,
                                  None, None) == want
        assert lib.relay_rms_norm_backward(type_, n, tokens, d, rows, None, B, 64, C, rows, None, None, None,
                                           _r(D, 640, 64), E, 64, A, 1 << 40, None) == want
        assert lib.relay_weight_grad(type_, n, tokens, d, 64, rows, B, C, None, 0, None, D, 4096, 64, E, 1 << 40,
                                     None) == want
        if type_ == 0:
            assert lib.relay_rms_norm_backward_workspace(n, tokens, d) == want
            assert lib.relay_weight_grad_workspace(2, n, tokens, d, 64, None) == want
            assert lib.relay_weight_grad_workspace(2, n, tokens, 64, d, None) == want
    assert lib.relay_checkpoint_pitch(0) == BAD and lib.relay_checkpoint_pitch(1) == 128
    assert lib.relay_checkpoint_pitch(128) == 128 and lib.relay_checkpoint_pitch(129) == 256
    wide = _r(A, 0, 40000)
    assert lib.relay_rms_norm(0, 1, 2, 32769, wide, None, B, 0, 1e-5, None, _r(C, 0, 40000), None, None, None,
                              None) == BIG
    assert lib.relay_rms_norm_backward_workspace(1, 2, 32769) == BIG


def test_rows(lib):
    """Inputs may repeat rows, outputs may not; NULL, negative strides and odd addresses are refused."""
    def unpack(r, n=2, tokens=10, type_=0):
        return lib.relay_checkpoint_unpack(type_, n, tokens, 64, A, B, r, None)

    assert unpack(None) == BAD
    assert unpack(_r(None, 640, 64)) == BAD
    assert unpack(_r(C + 1, 640, 64)) == BAD
    assert unpack(_r(C + 2, 640, 64), type_=2) == BAD
    assert unpack(_r(C, 640, -64)) == BAD
    assert unpack(_r(C, -640, 64)) == BAD
    assert unpack(_r(C, 640, 63)) == BAD      # rows overlap
    assert unpack(_r(C, 639, 64)) == BAD      # workers overlap
    assert unpack(_r(C, 64, 127)) == BAD      # token by token, and overlapping
    assert unpack(_r(C, 0, 64)) == BAD
    assert lib.relay_checkpoint_unpack(0, 2, 0, 64, None, None, _r(None, 0, 0), None) == OK  # nothing to do
    assert lib.relay_checkpoint_pack(0, 2, 10, 64, _r(C, 640, 64), None, B, None) == BAD
    assert lib.relay_checkpoint_pack(0, 2, 10, 64, _r(C, 640, 64), A, None, None) == BAD
    assert lib.relay_checkpoint_pack(0, 2, 10, 64, _r(C, 640, 64), A + 8, B, None) == BAD
    assert lib.relay_checkpoint_pack(0, 2, 10, 64, _r(C, 640, 64), A, B + 4, None) == BAD


def test_norm_refusals(lib):
    def call(x=_r(A, 640, 64), r=None, w=B, ws=64, eps=1e-5, total=None, y=_r(C, 640, 64), rstd=None, q=None, c=None):
        return lib.relay_rms_norm(0, 2, 10, 64, x, r, w, ws, eps, total, y, rstd, q, c, None)

    for kw in (dict(x=None), dict(y=None), dict(w=None), dict(w=B + 2), dict(ws=-1), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(r=_r(None, 0, 0)), dict(total=_r(D, 64, 64)),
               dict(rstd=D + 2), dict(q=D), dict(c=D), dict(q=D + 1, c=E), dict(y=_r(A, 640, 64)),
               dict(r=_r(C, 640, 64)), dict(total=_r(C, 640, 64))):
        assert call(**kw) == BAD, kw


def test_norm_backward_refusals(lib):
    need = lib.relay_rms_norm_backward_workspace(2, 10, 64)
    assert need > 0

    def call(dy=_r(A, 640, 64), dh=None, w=B, rstd=C, total=_r(D, 640, 64), q=None, c=None, lengths=None,
             dx=_r(E, 640, 64), dw=6 << 20, ds=64, work=7 << 20, size=need):
        return lib.relay_rms_norm_backward(0, 2, 10, 64, dy, dh, w, 64, rstd, total, q, c, lengths, dx, dw, ds, work,
                                           size, None)

    for kw in (dict(dy=None), dict(dx=None), dict(w=None), dict(rstd=None), dict(rstd=C + 1), dict(total=None),
               dict(q=B), dict(q=B, c=C), dict(total=None, q=B), dict(total=None, c=B), dict(lengths=C + 2),
               dict(dx=_r(A, 640, 64)), dict(dx=_r(D, 640, 64)), dict(dh=_r(E, 640, 64)), dict(dw=None),
               dict(dw=C + 2), dict(ds=63), dict(work=None), dict(work=A + 4), dict(size=need - 1),
               dict(dh=_r(A, -1, 64))):
        assert call(**kw) == BAD, kw


def test_gated_refusals(lib):
    g, u, o = _r(A, 640, 64), _r(B, 640, 64), _r(C, 640, 64)
    f = lib.relay_gated
    none = (None, None, None, None, None)
    assert f(0, 2, 10, 64, None, u, o, *none) == BAD
    assert f(0, 2, 10, 64, g, None, o, *none) == BAD
    assert f(0, 2, 10, 64, g, u, None, *none) == BAD
    assert f(0, 2, 10, 64, g, u, g, *none) == BAD
    assert f(0, 2, 10, 64, g, u, u, *none) == BAD
    assert f(0, 2, 10, 64, g, u, o, D, None, None, None, None) == BAD
    assert f(0, 2, 10, 64, g, u, o, None, None, None, D, None) == BAD
    assert f(0, 2, 10, 64, g, u, o, D, E, D, E, None) == BAD
    h = lib.relay_gated_backward
    dg, du = _r(D, 640, 64), _r(E, 640, 64)
    eight = [6 << 20, 7 << 20, 8 << 20, 9 << 20]
    for args in ((None, g, u, *none[:4], dg, du, None, None), (o, g, None, *none[:4], dg, du, None, None),
                 (o, None, None, *none[:4], dg, du, None, None), (o, g, u, *eight, dg, du, None, None),
                 (o, None, None, *eight[:3], None, dg, du, None, None), (o, g, u, *none[:4], dg, dg, None, None),
                 (o, g, u, *none[:4], o, du, None, None), (o, g, u, *none[:4], dg, u, None, None),
                 (o, g, u, *none[:4], None, du, None, None), (o, None, None, *eight, dg, du, 10 << 20, None),
                 (o, None, None, *eight, dg, du, eight[0], 10 << 20)):
        assert h(0, 2, 10, 64, *args, None) == BAD, args


def test_weight_grad_refusals(lib):
    need = lib.relay_weight_grad_workspace(0, 2, 10, 48, 64, _r(A + 2, 480, 48))
    assert need == 2 * 2 * 10 * 48  # unaligned: copied
    assert lib.relay_weight_grad_workspace(0, 2, 10, 48, 64, _r(A, 480, 48)) == 0
    assert lib.relay_weight_grad_workspace(0, 2, 10, 48, 64, None) == need
    assert lib.relay_weight_grad_workspace(2, 2, 10, 48, 64, None) == 3 * need
    assert lib.relay_weight_grad_workspace(0, 2, 10, 48, 64, _r(A, 480, 0)) == need  # one row, repeated

    def call(dy=_r(A + 2, 480, 48), q=B, c=C, scale=None, ss=0, lengths=None, dw=D, ws=48 * 64, row=64, work=E,
             size=need):
        return lib.relay_weight_grad(0, 2, 10, 48, 64, dy, q, c, scale, ss, lengths, dw, ws, row, work, size, None)

    for kw in (dict(dy=None), dict(q=None), dict(c=None), dict(q=B + 8), dict(scale=A + 1), dict(scale=A, ss=-1),
               dict(lengths=A + 2), dict(dw=None), dict(dw=D + 2), dict(ws=48 * 64 - 1), dict(row=63), dict(row=-1),
               dict(size=need - 1), dict(work=None), dict(work=E + 8)):
        assert call(**kw) == BAD, kw


def test_binding_refuses_tensors_that_do_not_fit(lib):
    """On a machine without a GPU every tensor is on the wrong device; with one, the same calls are
    refused for it too (CPU tensors)."""
    x = torch.zeros(2, 3, 64)
    w, ckpt = torch.zeros(2, 64), rs.ActivationCheckpoint(2, 3, 64, device="cpu")
    with pytest.raises(ValueError, match="x"):
        rs.relay_rms_norm(x, w, torch.zeros_like(x), 1e-5)
    with pytest.raises(ValueError, match="current CUDA device"):
        rs.relay_checkpoint_pack(x, ckpt)
    for bad in (torch.zeros(3, 64), torch.zeros(2, 3, 64, dtype=torch.int32), None, 3, np.zeros((2, 3, 64))):
        with pytest.raises(ValueError):
            rs.relay_checkpoint_pack(bad, ckpt)
        with pytest.raises(ValueError):
            rs.relay_rms_norm(bad, w, x, 1e-5)
        with pytest.raises(ValueError):
            rs.relay_gated(bad, x, x)
        with pytest.raises(ValueError):
            rs.relay_weight_grad(bad, ckpt, x, w)
    with pytest.raises(rs.RelayError):
        rs.relay_rms_norm_backward_workspace(2, 3, 40000)
    with pytest.raises(rs.RelayError):
        rs.ActivationCheckpoint(2, 3, 0, device="cpu")


@pytest.mark.gpu
def test_binding_refuses_other_types_shapes_and_strides():
    x = torch.zeros(2, 3, 64, device="cuda")
    w, y = torch.zeros(2, 64, device="cuda"), torch.zeros_like(x)
    ckpt = rs.ActivationCheckpoint(2, 3, 64)
    work = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: rs.relay_rms_norm(x, w, y.half(), 1e-5), lambda: rs.relay_rms_norm(x, w, y[:, :2], 1e-5),
                 lambda: rs.relay_rms_norm(x, w.half(), y, 1e-5), lambda: rs.relay_rms_norm(x, w[:, :63], y, 1e-5),
                 lambda: rs.relay_rms_norm(x, w.t().contiguous().t(), y, 1e-5),
                 lambda: rs.relay_rms_norm(x.transpose(1, 2).contiguous().transpose(1, 2), w, y, 1e-5),
                 lambda: rs.relay_rms_norm(x, w, y, 1e-5, rstd=torch.zeros(3, 2, device="cuda").t()),
                 lambda: rs.relay_rms_norm(x, w, y, 1e-5, checkpoint=rs.ActivationCheckpoint(2, 3, 63)),
                 lambda: rs.relay_rms_norm(x, w, y, 1e-5, checkpoint=rs.ActivationCheckpoint(2, 4, 64)),
                 lambda: rs.relay_weight_grad(x, ckpt, w, work),
                 lambda: rs.relay_weight_grad(x, ckpt, torch.zeros(2, 63, 64, device="cuda"), work),
                 lambda: rs.relay_weight_grad(x, ckpt, torch.zeros(2, 64, 64, device="cuda"), work,
                                              lengths=torch.zeros(2, dtype=torch.int64, device="cuda")),
                 lambda: rs.relay_weight_grad(x, ckpt, torch.zeros(2, 64, 64, device="cuda"), work.cpu())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(rs.RelayError):  # total's buffer as y
        rs.relay_rms_norm(x, w, y, 1e-5, total=y)
    with pytest.raises(rs.RelayError):  # no workspace
        rs.relay_rms_norm_backward(x, w, torch.zeros(2, 3, device="cuda"), y, w.clone(), work[:64], total=x)
