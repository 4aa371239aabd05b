"""The layer operators at the ends of their range: gates down to the type's lowest value, weights
that are not finite beside padding."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

from . import layers_util as lu
from .layers_util import LEAST, ROUND, TYPES, U, np64, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _held_by(v, dtype):
    return np64(torch.from_numpy(np.asarray(v, np.float64)).to(dtype))


def _rounded(want, dtype, bound):
    return bound + ROUND[dtype] * (np.abs(want) + bound) + LEAST[dtype]


# ------------------------------------------------------------------ gates


def _gates(dtype):
    """(gate, up, output's gradient) [1][T][64]: in each row one gate of the list at feature 0, with
    ordinary ones beside it."""
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    rows = [(g, u) for g in (low, -1e38, -1e36, -1e30, -1e4, -300.0, -100.0, -95.0, -90.0, -88.5, -88.0, -87.5, -87.0,
                             -80.0, -20.0, -0.0, 20.0, 88.0, 1e4, high, np.inf, -np.inf, np.nan)
            for u in (1.0, -0.375) + ((1e30,) if g < -50 and dtype is not torch.float16 else ())]
    g = np.random.default_rng(0).standard_normal((1, len(rows), 64))
    u, da = np.roll(g, 1, 2) + 2.0, np.full_like(g, 0.5)
    g[0, :, 0], u[0, :, 0] = [r[0] for r in rows], [r[1] for r in rows]
    return _held_by(g, dtype), _held_by(u, dtype), da


def _sigma_error(g, dtype):
    """Relative error of g sigma(g): as for moderate gates (16 roundings, and in 16 bits the rounded
    product by log2(e), which |g| magnifies); one part in 2^20 more where sigma is subnormal in fp32
    (below -87.3, where its 2^-149 are that part of it or less); all of it where sigma is less
    than 2^-128 (below -88.7) and may be taken as 0."""
    with np.errstate(invalid="ignore"):
        e = (16 + (4 * np.abs(np.where(np.isfinite(g), g, 0)) if dtype != torch.float32 else 0)) * U
        return np.where(g < -88.7, 1.0, e + np.where(g < -87.3, 2.0 ** -20, 0.0))


def _same(got, want, bound):
    """Within the bound, with infinities and NaN in the same places."""
    got = np64(got) if isinstance(got, torch.Tensor) else got
    assert np.array_equal(np.where(np.isinf(got), got, 0), np.where(np.isinf(want), want, 0))
    with np.errstate(invalid="ignore"):
        within(got, want, np.where(np.isfinite(want), bound, 0))


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "odd"])
def test_gates_of_any_size(dtype, layout):
    """g sigma(g) u goes to 0 as g falls, down to the lowest value that the type has; NaN at minus
    infinity, where the formula has infinity times 0, and at NaN."""
    g, u, da = _gates(dtype)
    n, T, d = g.shape
    with np.errstate(invalid="ignore", over="ignore"):
        s, rest = lu.sigmoid(g), lu.sigmoid(-g)
        act, du = g * s * u, da * (g * s)
        dg = da * u * (s * (1 + g * rest))
        act_bound, du_bound = _sigma_error(g, dtype) * np.abs(act), _sigma_error(g, dtype) * np.abs(du)
        dg_bound = 1.5 * _sigma_error(g, dtype) * np.abs(da * u * s) * (1 + np.abs(g) * rest)
        gv, uv, dv = (lu.rows(v, dtype, layout)[0] for v in (g, u, da))
        out, kg, ku = lu.empty_rows(n, T, d, dtype, layout)[0], *(rs.ActivationCheckpoint(n, T, d) for _ in range(2))
        rs.relay_gated(gv, uv, out, gate_checkpoint=kg, up_checkpoint=ku)
        _same(out, act, _rounded(act, dtype, act_bound))
        (ov, _), (pv, _) = lu.empty_rows(n, T, d, dtype, layout), lu.empty_rows(n, T, d, dtype, layout)
        kept = rs.ActivationCheckpoint(n, T, d)
        rs.relay_gated_backward(dv, ov, pv, gate=gv, up=uv, out_checkpoint=kept)
        _same(pv, du, _rounded(du, dtype, du_bound))
        _same(ov, dg, _rounded(dg, dtype, dg_bound))
        got = lu.held(kept.codes.cpu().numpy(), kept.scales.cpu().numpy(), d)
        fits = np.repeat(lu.scale_bytes(np.abs(act.reshape(n, T, 2, 32)).max(-1)) < 255, 32, -1)
        assert np.array_equal(np.isnan(got), ~fits)
        within(got[fits], act[fits], (lu.half_step(act) * (1 + 2.0 ** -10) + act_bound)[fits])

        # from 8 bits: the gates that those hold
        pairs = [(k.codes.cpu().numpy(), k.scales.cpu().numpy()) for k in (kg, ku)]
        g, u = (lu.held(q, c, d) for q, c in pairs)
        s, rest = lu.sigmoid(g), lu.sigmoid(-g)
        du, dg = da * (g * s), da * u * (s * (1 + g * rest))
        dg_bound = 1.5 * _sigma_error(g, dtype) * np.abs(da * u * s) * (1 + np.abs(g) * rest)
        rs.relay_gated_backward(dv, ov, pv, gate_checkpoint=kg, up_checkpoint=ku)
        _same(pv, du, _rounded(du, dtype, _sigma_error(g, dtype) * np.abs(du)))
        _same(ov, dg, _rounded(dg, dtype, dg_bound))


# ------------------------------------------------------------------ padding


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("source", ["checkpoint", "total"])
@pytest.mark.parametrize("d", [64, 500, 1000, 2048, 4096, 8192, 16384, 20000])
def test_padding_is_zero_whatever_the_weight(dtype, layout, source, d):
    """dx past the lengths is 0 also where a worker's weight holds an infinity or a NaN, which
    reaches that worker's other rows only."""
    n, T, lengths = 3, 4, [2, 0, 3]
    g = np.random.default_rng(0)
    h, dy, dh = (_held_by(g.standard_normal((n, T, d)), dtype) for _ in range(3))
    rstd = torch.from_numpy(1 / np.sqrt((h * h).mean(-1) + EPS)).float().cuda()
    kw = {"lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"), "dtotal": lu.rows(dh, dtype, layout)[0]}
    if source == "checkpoint":
        kw["checkpoint"] = rs.ActivationCheckpoint(n, T, d).pack(lu.rows(h, dtype, "dense")[0])
    else:
        kw["total"] = lu.rows(h, dtype, layout)[0]
    good = torch.ones(n, d, device="cuda")
    bad = good.clone()
    bad[0, d // 2], bad[1, 0], bad[1, d - 1] = float("inf"), float("nan"), float("-inf")
    work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    results = []
    for w in (good, bad):
        dx, dw = lu.empty_rows(n, T, d, dtype, layout)[0], torch.empty(n, d, device="cuda")
        rs.relay_rms_norm_backward(lu.rows(dy, dtype, layout)[0], w, rstd, dx, dw, work, **kw)
        for i, m in enumerate(lengths):
            assert not dx[i, m:].any()  # (NaN is true)
        results.append((dx, dw))
    (dx, dw), (dx_bad, dw_bad) = results
    assert torch.equal(dw, dw_bad) and torch.equal(dx[2], dx_bad[2])
    assert dx_bad[0, :2, d // 2].isnan().all()
