"""The layer operators of relaylayers.h on the GPU against their definitions in
64 bits: types, layouts, odd sizes, lengths that leave a worker empty, values
that are not numbers, offsets past 32 bits, streams and graphs."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

from . import layers_util as lu
from .layers_util import CHAIN, LEAST, ROUND, TYPES, U, np64, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _values(seed, n, T, d, dtype, size=1.0):
    """Normal values that the type holds, one feature in 16 much louder, as float64."""
    g = np.random.default_rng(seed)
    v = g.standard_normal((n, T, d)) * np.where(g.random(d) < 1 / 16, 20.0, 1.0) * size
    return np64(torch.from_numpy(v).to(dtype))


def _weight(seed, n, d, first=0):
    """fp32 [n][d] in wider rows, from column `first` on."""
    w = torch.from_numpy(1 + 0.3 * np.random.default_rng(seed).standard_normal((n, first + d + 7))).float().cuda()
    return w[:, first:first + d]


def _rounded(want, dtype, bound):
    return bound + ROUND[dtype] * (np.abs(want) + bound) + LEAST[dtype]


# ------------------------------------------------------------------ the 8-bit format

WIDTHS = [1, 7, 31, 32, 33, 127, 128, 129, 255, 256, 264, 515, 1000, 1537]


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
def test_checkpoint_codes_are_the_formats(dtype, layout):
    for d in WIDTHS:
        n, T = 3, 5
        x = _values(d, n, T, d, dtype) * np.exp2(np.random.default_rng(d).integers(-9, 9, (n, T, 1)))
        x = np64(torch.from_numpy(x).to(dtype))
        x[0, 0] = 0
        want_q, want_c = lu.pack(x)
        ckpt = rs.ActivationCheckpoint(n, T, d)
        ckpt.codes.fill_(55)
        ckpt.scales.fill_(55)
        view, _ = lu.rows(x, dtype, layout)
        rs.relay_checkpoint_pack(view, ckpt)
        assert np.array_equal(ckpt.codes.cpu().numpy(), want_q), d
        assert np.array_equal(ckpt.scales.cpu().numpy(), want_c), d
        out, buf = lu.empty_rows(n, T, d, dtype, layout)
        rs.relay_checkpoint_unpack(ckpt, out)
        want = torch.from_numpy(lu.held(want_q, want_c, d)).to(dtype)
        assert torch.equal(out.cpu(), want), d
        assert lu.only_rows_written(out, buf)


def test_checkpoint_at_the_ends_of_the_range():
    """Ties, the step to the next scale, subnormals, the largest magnitudes, infinities and NaN,
    each in a block of its own: only the blocks that hold no number read as NaN."""
    big = float(np.finfo(np.float32).max)
    first = [0.0, 127.0, 127.49999, 127.5, 127.5 * 2.0 ** -40, 2.0 ** -126, 2.0 ** -149, 2.0 ** -120, 1e-40,
             127.0 * 2.0 ** 121, 127.49999 * 2.0 ** 121, 127.5 * 2.0 ** 121, big, np.inf, -np.inf, np.nan, 0.5, 126.5]
    x = np.zeros((1, len(first), 64))
    x[0, :, 0] = first
    x[0, :, 1] = np.float64(np.float32(first)) / 254  # small codes beside it
    x[0, :, 40] = 3.0  # the next block
    x = np64(torch.from_numpy(x).float())
    want_q, want_c = lu.pack(x)
    for layout in ("dense", "odd"):
        ckpt = rs.ActivationCheckpoint(1, len(first), 64).pack(lu.rows(x, torch.float32, layout)[0])
        assert np.array_equal(ckpt.codes.cpu().numpy(), want_q)
        assert np.array_equal(ckpt.scales.cpu().numpy(), want_c)
        out = np64(ckpt.unpack(torch.float32))
        assert np.array_equal(out, lu.held(want_q, want_c, 64), equal_nan=True)
        assert (out[..., 40] == 3.0).all()
        assert np.isnan(out[0, 11:16, :32]).all() and not np.isnan(out[0, :11]).any()
        half = np64(ckpt.unpack(torch.float16))
        assert np.isfinite(half[~np.isnan(out)]).all() and np.array_equal(np.isnan(half), np.isnan(out))
        assert half[0, 9, 0] == 65504.0


def test_checkpoint_reads_foreign_scale_bytes_as_the_smallest():
    ckpt = rs.ActivationCheckpoint(1, 1, 32)
    ckpt.codes.fill_(3)
    for c in (0, 5, 6, 7):
        ckpt.scales.fill_(c)
        assert (np64(ckpt.unpack(torch.float32)) == 3 * 2.0 ** -126).all()


def test_checkpoint_past_32_bit_offsets():
    """More than 2^32 codes, and rows more than 2^31 elements apart."""
    T, d = (1 << 18) + 3, 16384
    row = torch.randn(1, 1, d, device="cuda")
    ckpt = rs.ActivationCheckpoint(1, T, d).pack(row.expand(1, T, d))
    q, c = lu.pack(np64(row))
    assert np.array_equal(ckpt.codes[0, [0, T // 2, T - 1]].cpu().numpy(), np.repeat(q[0], 3, 0))
    assert np.array_equal(ckpt.scales[0, [0, T // 2, T - 1]].cpu().numpy(), np.repeat(c[0], 3, 0))
    del ckpt
    far = (1 << 31) + 64
    buf = torch.zeros(far + 256, dtype=torch.bfloat16, device="cuda")
    out = buf.as_strided((2, 1, 256), (far, 256, 1))
    x = _values(1, 2, 1, 256, torch.bfloat16)
    rs.ActivationCheckpoint(2, 1, 256).pack(torch.from_numpy(x).cuda().bfloat16())
    small = rs.ActivationCheckpoint(2, 1, 256).pack(torch.from_numpy(x).cuda().bfloat16())
    rs.relay_checkpoint_unpack(small, out)
    assert np.array_equal(np64(out), lu.held(*lu.pack(x), 256))
    assert float(buf[256:far].abs().max()) == 0


# ------------------------------------------------------------------ the norm


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
@pytest.mark.parametrize("d", [1, 7, 32, 257, 512, 1000, 1024, 1537, 2048, 4096, 5000, 8192, 12000, 16384, 20001, 32768])
def test_norm(dtype, layout, d):
    n, T = (3, 5) if d < 3000 else (2, 2)
    for residual, first in ((True, 4), (False, 1)):
        x, r = _values(1, n, T, d, dtype), _values(2, n, T, d, dtype) if residual else None
        x[0, 0] = 0
        if residual:
            r[0, 0] = 0  # a row of zeros: y = 0, not NaN
        w = _weight(3, n, d, first)
        h, s, xhat, y = lu.norm(x, r, np64(w), float(np.float32(EPS)))
        xv = lu.rows(x, dtype, layout)[0]
        rv = lu.rows(r, dtype, layout)[0] if residual else None
        (yv, ybuf), (tv, tbuf) = lu.empty_rows(n, T, d, dtype, layout), lu.empty_rows(n, T, d, dtype, layout)
        rstd, ckpt = torch.empty(n, T, device="cuda"), rs.ActivationCheckpoint(n, T, d)
        rs.relay_rms_norm(xv, w, yv, EPS, residual=rv, total=tv, rstd=rstd, checkpoint=ckpt)
        within(tv, h, _rounded(h, dtype, U * np.abs(h)))
        within(rstd, s, CHAIN * U * s)
        within(yv, y, _rounded(y, dtype, CHAIN * U * np.abs(y)))
        got = lu.held(ckpt.codes.cpu().numpy(), ckpt.scales.cpu().numpy(), d)
        within(got, xhat, lu.half_step(xhat) * (1 + 2.0 ** -10) + CHAIN * U * np.abs(xhat))
        assert not ckpt.codes[..., d:].any() and lu.only_rows_written(yv, ybuf) and lu.only_rows_written(tv, tbuf)
        again, none = torch.empty_like(yv), lu.empty_rows(n, T, d, dtype, layout)[0]
        rs.relay_rms_norm(xv, w, again, EPS, residual=rv)  # only y
        assert torch.equal(again, yv)
        if residual:  # in place on the residual stream
            rs.relay_rms_norm(xv, w, none, EPS, residual=rv, total=rv)
            assert torch.equal(rv, tv) and torch.equal(none, yv)


def test_norm_of_rows_that_are_not_numbers():
    """An infinity or a NaN spoils its own row only."""
    x = _values(5, 1, 6, 515, torch.float32)
    x[0, 1, 7], x[0, 3, 500], x[0, 4] = np.inf, np.nan, 1e-30
    w = _weight(3, 1, 515)
    y, ckpt = torch.empty(1, 6, 515, device="cuda"), rs.ActivationCheckpoint(1, 6, 515)
    rs.relay_rms_norm(torch.from_numpy(x).float().cuda(), w, y, EPS, checkpoint=ckpt)
    h, s, xhat, want = lu.norm(x[:, [0, 2, 4, 5]], None, np64(w), float(np.float32(EPS)))
    within(y[:, [0, 2, 4, 5]], want, _rounded(want, torch.float32, CHAIN * U * np.abs(want)))
    assert np.isnan(np64(y)[0, 1, 7]) and np.isnan(np64(y)[0, 3]).all()
    held = np64(ckpt.unpack(torch.float32))
    assert np.isnan(held[0, 1, :32]).all() and np.isnan(held[0, 3]).all()
    assert np.isfinite(held[0, [0, 2, 4, 5]]).all()


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
@pytest.mark.parametrize("source", ["checkpoint", "total"])
@pytest.mark.parametrize("d", [1, 7, 32, 257, 512, 1000, 1024, 1537, 2048, 4096, 8192, 12000, 16384, 20001, 32768])
def test_norm_backward(dtype, layout, source, d):
    n, T = (5, 9) if d < 3000 else (3, 2)
    lengths = [T, 0, 1, T + 5, -3][:n]
    for given, with_dh in ((None, True), (lengths, False), (lengths, True)):
        used = lu.used_rows(None if given is None else np.array(given), n, T)
        h, dy = _values(1, n, T, d, dtype), _values(2, n, T, d, dtype, 0.01)
        dh = _values(4, n, T, d, dtype, 0.01) if with_dh else None
        w = _weight(3, n, d, 4)
        s = np64(torch.from_numpy(1 / np.sqrt((h * h).mean(-1) + EPS)).float())
        for v in (h, dy) + ((dh,) if with_dh else ()):
            v[~used[..., 0]] = np.nan  # padding is not read
        s[~used[..., 0]] = np.nan
        if source == "checkpoint":
            xhat0 = np.where(np.isnan(h), 0, h) * np.where(np.isnan(s), 0, s)[..., None]
            codes, scales = lu.pack(xhat0)
            scales[~used[..., 0]] = 255
            xhat = lu.held(codes, scales, d)
            kw = {"checkpoint": (torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())}
        else:
            xhat, kw = h * s[..., None], {"total": lu.rows(h, dtype, layout)[0]}
        dx, dw, dx_bound, dw_bound = lu.norm_backward(dy, np64(w), s, xhat, dh, used)
        out, buf = lu.empty_rows(n, T, d, dtype, layout)
        flat = torch.full((n, d + 9), 77.0, device="cuda")
        grad = flat[:, 5:5 + d]
        work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
        kw.update(dtotal=lu.rows(dh, dtype, layout)[0] if with_dh else None,
                  lengths=None if given is None else torch.tensor(given, dtype=torch.int32, device="cuda"))
        args = (lu.rows(dy, dtype, layout)[0], w, torch.from_numpy(s).float().cuda())
        rs.relay_rms_norm_backward(*args, out, grad, work, **kw)
        # xhat from the total is one more rounding of each product
        within(out, dx, _rounded(dx, dtype, dx_bound * 2))
        within(grad, dw, dw_bound)
        assert lu.only_rows_written(out, buf) and lu.only_rows_written(grad, flat.view(-1))
        again, grad2 = torch.empty_like(out), torch.empty_like(grad)
        rs.relay_rms_norm_backward(*args, again, grad2, work, **kw)
        assert torch.equal(again, out) and torch.equal(grad2, grad)  # the same bits


@pytest.mark.parametrize("n,T", [(1, 1), (1, 700), (4, 1000), (256, 3)])
def test_norm_backward_over_many_tokens(n, T):
    d, dtype = 136, torch.float32
    h, dy, w = _values(1, n, T, d, dtype), _values(2, n, T, d, dtype), _weight(3, n, d)
    s = np64(torch.from_numpy(1 / np.sqrt((h * h).mean(-1) + EPS)).float())
    dx, dw, dx_bound, dw_bound = lu.norm_backward(dy, np64(w), s, h * s[..., None], None, lu.used_rows(None, n, T))
    out, grad = torch.empty(n, T, d, device="cuda"), torch.empty(n, d, device="cuda")
    work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    rs.relay_rms_norm_backward(torch.from_numpy(dy).float().cuda(), w, torch.from_numpy(s).float().cuda(), out, grad,
                               work, total=torch.from_numpy(h).float().cuda())
    within(out, dx, _rounded(dx, dtype, dx_bound * 2))
    within(grad, dw, dw_bound)


def test_norm_gradient_against_differences():
    """d/de of sum(gy y + gt total) along random directions of x and of the weight: central
    differences of the forward call at +-2^-6 are within (2^-6)^2 of the slope, relative to its
    scale, and the forward's rounding adds 2^6 2^-23 of the sums' magnitudes at most."""
    n, T, d, e = 2, 3, 96, 2.0 ** -6
    g = np.random.default_rng(0)
    x, r, gy, gt, vx = (torch.from_numpy(g.standard_normal((n, T, d))).float().cuda() for _ in range(5))
    w, vw = (torch.from_numpy(g.standard_normal((n, d))).float().cuda() for _ in range(2))

    def loss(x, w):
        y, total, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, T, device="cuda")
        rs.relay_rms_norm(x, w, y, EPS, residual=r, total=total, rstd=rstd)
        return float((gy.double() * y).sum() + (gt.double() * total).sum()), total, rstd

    _, total, rstd = loss(x, w)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    rs.relay_rms_norm_backward(gy, w, rstd, dx, dw, work, total=total, dtotal=gt)
    size = float((gy * gy).sum().sqrt() + (gt * gt).sum().sqrt()) * float((vx * vx).sum().sqrt()) / d ** 0.5
    tol = size * 4 * e * e + n * T * d * 8 * 2.0 ** -23 / e
    slope = (loss(x + e * vx, w)[0] - loss(x - e * vx, w)[0]) / (2 * e)
    assert abs(slope - float((dx.double() * vx).sum())) < tol
    slope = (loss(x, w + e * vw)[0] - loss(x, w - e * vw)[0]) / (2 * e)
    assert abs(slope - float((dw.double() * vw).sum())) < tol


# ------------------------------------------------------------------ the gated activation


def _gate_values(seed, n, T, d, dtype):
    g = _values(seed, n, T, d, dtype)
    flat = g.reshape(-1)
    ends = [0.0, -0.0, 30.0, -30.0, 100.0, -100.0, 1e-6, -1.2784645]
    flat[:min(len(ends), flat.size)] = ends[:flat.size]
    return np64(torch.from_numpy(g).to(dtype))


def _sigma_error(g, dtype):
    """Relative error of sigma(g), 1 - sigma(g) and their few products: 16 roundings; 16-bit rows
    also take exp from a product by log2(e) that is rounded, which |g| magnifies."""
    return (16 + (4 * np.abs(g) if dtype != torch.float32 else 0)) * U


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
def test_gated(dtype, layout):
    for d in (1, 8, 33, 128, 257, 1000, 2048):
        n, T = 3, 4
        g, u = _gate_values(1, n, T, d, dtype), _values(2, n, T, d, dtype)
        want = g * lu.sigmoid(g) * u
        bound = _sigma_error(g, dtype) * np.abs(want) + 1e-37 * np.abs(g * u)
        gv, uv = lu.rows(g, dtype, layout)[0], lu.rows(u, dtype, layout)[0]
        out, buf = lu.empty_rows(n, T, d, dtype, layout)
        kg, ku = rs.ActivationCheckpoint(n, T, d), rs.ActivationCheckpoint(n, T, d)
        rs.relay_gated(gv, uv, out, gate_checkpoint=kg, up_checkpoint=ku)
        within(out, want, _rounded(want, dtype, bound))
        assert lu.only_rows_written(out, buf)
        for kept, v in ((kg, g), (ku, u)):
            q, c = lu.pack(v)
            assert np.array_equal(kept.codes.cpu().numpy(), q) and np.array_equal(kept.scales.cpu().numpy(), c)
        again = torch.empty_like(out)
        rs.relay_gated(gv, uv, again)
        assert torch.equal(again, out)
        only = rs.ActivationCheckpoint(n, T, d)
        rs.relay_gated(gv, uv, again, up_checkpoint=only)
        assert torch.equal(only.codes, ku.codes) and torch.equal(again, out)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
@pytest.mark.parametrize("source", ["checkpoint", "rows"])
def test_gated_backward(dtype, layout, source):
    for d in (1, 8, 33, 128, 257, 1000, 2048):
        n, T = 3, 4
        g, u, da = _gate_values(1, n, T, d, dtype), _values(2, n, T, d, dtype), _values(3, n, T, d, dtype, 0.01)
        if source == "checkpoint":
            pairs = [lu.pack(v) for v in (g, u)]
            g, u = (lu.held(q, c, d) for q, c in pairs)
            kw = {k: tuple(torch.from_numpy(t).cuda() for t in p)
                  for k, p in zip(("gate_checkpoint", "up_checkpoint"), pairs)}
        else:
            kw = {"gate": lu.rows(g, dtype, layout)[0], "up": lu.rows(u, dtype, layout)[0]}
        dg, du = lu.gated_backward(da, g, u)
        s, rest = lu.sigmoid(g), lu.sigmoid(-g)
        dg_bound = 1.5 * _sigma_error(g, dtype) * np.abs(da * u * s) * (1 + np.abs(g) * rest) + 1e-37 * np.abs(da * u) * (1 + np.abs(g))
        du_bound = _sigma_error(g, dtype) * np.abs(du) + 1e-37 * np.abs(da * g)
        act = g * s * u
        (gv, gbuf), (uv, ubuf) = lu.empty_rows(n, T, d, dtype, layout), lu.empty_rows(n, T, d, dtype, layout)
        dv, kept = lu.rows(da, dtype, layout)[0], rs.ActivationCheckpoint(n, T, d)
        rs.relay_gated_backward(dv, gv, uv, out_checkpoint=kept, **kw)
        within(gv, dg, _rounded(dg, dtype, dg_bound))
        within(uv, du, _rounded(du, dtype, du_bound))
        assert lu.only_rows_written(gv, gbuf) and lu.only_rows_written(uv, ubuf)
        got = lu.held(kept.codes.cpu().numpy(), kept.scales.cpu().numpy(), d)
        within(got, act, lu.half_step(act) * (1 + 2.0 ** -10) + _sigma_error(g, dtype) * np.abs(act)
               + 1e-37 * np.abs(g * u))
        assert not kept.codes[..., d:].any()
        g2, u2 = torch.empty_like(gv), torch.empty_like(uv)
        rs.relay_gated_backward(dv, g2, u2, **kw)
        assert torch.equal(g2, gv) and torch.equal(u2, uv)


def test_gated_backward_of_a_block_that_is_not_a_number():
    """A NaN block gives NaN in its own features only, also where the row ends inside the block."""
    n, T, d = 1, 2, 40
    g, u = rs.ActivationCheckpoint(n, T, d), rs.ActivationCheckpoint(n, T, d)
    x = torch.ones(n, T, d, device="cuda")
    x[0, 1, 35] = float("nan")
    g.pack(x)
    u.pack(torch.ones(n, T, d, device="cuda"))
    dg, du, kept = torch.empty_like(x), torch.empty_like(x), rs.ActivationCheckpoint(n, T, d)
    rs.relay_gated_backward(torch.ones_like(x), dg, du, gate_checkpoint=g, up_checkpoint=u, out_checkpoint=kept)
    for t in (dg, du, kept.unpack(torch.float32)):
        assert torch.isnan(t[0, 1, 32:]).all() and torch.isfinite(t[0, 1, :32]).all() and torch.isfinite(t[0, 0]).all()


def test_gated_gradient_against_differences():
    """Central differences at +-2^-6 of sum(w a) along random directions, as for the norm: a's third
    derivatives are of order 1."""
    n, T, d, e = 1, 4, 64, 2.0 ** -6
    r = np.random.default_rng(1)
    g, u, w, vg, vu = (torch.from_numpy(r.standard_normal((n, T, d))).float().cuda() for _ in range(5))

    def loss(g, u):
        out = torch.empty_like(g)
        rs.relay_gated(g, u, out)
        return float((w.double() * out).sum())

    dg, du = torch.empty_like(g), torch.empty_like(g)
    rs.relay_gated_backward(w, dg, du, gate=g, up=u)
    tol = float((w * w).sum().sqrt()) * float((vg * vg).sum().sqrt()) * 4 * e * e + n * T * d * 8 * 2.0 ** -23 / e
    slope = (loss(g + e * vg, u + e * vu) - loss(g - e * vg, u - e * vu)) / (2 * e)
    assert abs(slope - float((dg.double() * vg).sum() + (du.double() * vu).sum())) < tol


# ------------------------------------------------------------------ the weight gradient


def _weight_grad(dtype, layout, n, T, outputs, inputs, lengths=None, scaled=False, first=5, gap=0, seed=0, dead=None):
    """relay_weight_grad on random inputs against 64 bits; rows past the lengths hold NaN."""
    dy = _values(seed + 1, n, T, outputs, dtype, 0.01)
    codes, scales = lu.pack(_values(seed + 2, n, T, inputs, torch.float32))
    if dead is not None:
        scales[dead] = 255
    used = lu.used_rows(None if lengths is None else np.array(lengths), n, T)
    dy[~used[..., 0]] = np.nan
    scales[~used[..., 0]] = 255
    xhat = np.where(used, lu.held(codes, scales, inputs), 0)
    w = _weight(seed + 3, n, inputs, 3) if scaled else None
    scale = np.ones((n, inputs)) if w is None else np64(w)
    clean = np.where(used, dy, 0)
    want = np.matmul(clean.transpose(0, 2, 1), xhat) * scale[:, None]
    bound = np.matmul(np.abs(clean).transpose(0, 2, 1), np.abs(xhat)) * np.abs(scale[:, None])
    # products are exact; each of T additions is off by one unit of the last place of a partial sum at most
    bound = (T + 16) * 2 * U * bound + 4 * U * np.abs(want)
    flat = torch.full((n, first + outputs * (inputs + gap) + 3), 77.0, device="cuda")
    out = flat[:, first:first + outputs * (inputs + gap)].unflatten(1, (outputs, inputs + gap))[..., :inputs]
    size = rs.relay_weight_grad_workspace(n, T, outputs, inputs)
    args = (lu.rows(dy, dtype, layout)[0], (torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()))
    kw = dict(column_scale=w,
              lengths=None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda"))
    rs.relay_weight_grad(*args, out, torch.full((size,), 255, dtype=torch.uint8, device="cuda"), **kw)
    within(out, want, bound)
    fine = np.isfinite(want)
    off = np.linalg.norm((np64(out) - want)[fine])
    assert off <= (T ** 0.5 + 1) * 2 * U * np.linalg.norm(want[fine])
    assert lu.only_rows_written(out, flat.view(-1))
    again = torch.empty_like(out)
    rs.relay_weight_grad(*args, again, torch.zeros(size, dtype=torch.uint8, device="cuda"), **kw)
    assert np.array_equal(np64(again), np64(out), equal_nan=True)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
@pytest.mark.parametrize("T,outputs,inputs", [(1, 1, 1), (1, 128, 256), (2, 7, 33), (15, 64, 64), (16, 129, 130),
                                              (17, 200, 128), (63, 128, 257), (64, 256, 512), (65, 72, 1000),
                                              (130, 136, 264), (515, 300, 200)])
def test_weight_grad(dtype, layout, T, outputs, inputs):
    _weight_grad(dtype, layout, 2, T, outputs, inputs, scaled=T % 2 == 0, gap=T % 3)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "odd"])
@pytest.mark.parametrize("T", [1, 40, 64, 200, 1000])
def test_weight_grad_lengths(dtype, layout, T):
    lengths = [T, 0, 1, T + 9, -2, T // 2, max(T - 1, 0)]
    _weight_grad(dtype, layout, len(lengths), T, 130, 140, lengths=lengths, scaled=True)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("n,T,outputs,inputs", [(1, 4099, 130, 257), (1, 3000, 64, 64), (3, 2500, 640, 520),
                                                (1, 2048, 2048, 1024), (256, 5, 9, 11), (3, 1000, 1111, 1537),
                                                (2, 700, 4100, 2600), (40, 200, 520, 300)])
def test_weight_grad_long_and_wide(dtype, n, T, outputs, inputs):
    _weight_grad(dtype, "dense", n, T, outputs, inputs, first=4)


def test_weight_grad_of_a_block_that_is_not_a_number():
    """A NaN block reaches the gradients of its own features only."""
    _weight_grad(torch.bfloat16, "dense", 1, 70, 40, 96, dead=(0, 33, 1))


def test_weight_grad_without_tokens_is_zero():
    out = torch.full((2, 5, 7), 3.0, device="cuda")
    dy = torch.empty(2, 0, 5, dtype=torch.bfloat16, device="cuda")
    work = torch.empty(rs.relay_weight_grad_workspace(2, 0, 5, 7), dtype=torch.uint8, device="cuda")
    rs.relay_weight_grad(dy, rs.ActivationCheckpoint(2, 0, 7), out, work)
    assert not out.any()


def test_weight_grad_past_32_bit_offsets():
    """Codes past 2^31, a gradient whose workers lie 2^31 elements apart, sums that fp32 holds exactly."""
    T, inputs = (1 << 17) + 5, 16384
    row = torch.randint(-100, 101, (1, 1, inputs), device="cuda").float()
    ckpt = rs.ActivationCheckpoint(1, T, inputs).pack(row.expand(1, T, inputs))
    dy = torch.ones(1, 1, 8, dtype=torch.bfloat16, device="cuda").expand(1, T, 8)
    out = torch.empty(1, 8, inputs, device="cuda")
    work = torch.empty(rs.relay_weight_grad_workspace(1, T, 8, inputs), dtype=torch.uint8, device="cuda")
    rs.relay_weight_grad(dy, ckpt, out, work)
    assert torch.equal(out, (row * T).expand_as(out))
    del ckpt
    far = (1 << 31) + 16
    buf = torch.zeros(far + 64, device="cuda")
    out = buf.as_strided((2, 4, 8), (far, 8, 1))
    ckpt = rs.ActivationCheckpoint(2, 1, 8).pack(torch.full((2, 1, 8), 3.0, device="cuda"))
    rs.relay_weight_grad(torch.ones(2, 1, 4, device="cuda"), ckpt, out, work)
    assert (out == 3).all() and float(buf[32:far].abs().max()) == 0


# ------------------------------------------------------------------ tokens of none, streams, graphs


def test_no_tokens():
    for dtype in TYPES.values():
        x = torch.empty(2, 0, 24, dtype=dtype, device="cuda")
        none = rs.ActivationCheckpoint(2, 0, 24)
        rstd = torch.empty(2, 0, device="cuda")
        rs.relay_rms_norm(x, _weight(0, 2, 24), x.clone(), EPS, residual=x, total=x, rstd=rstd, checkpoint=none)
        none.pack(x).unpack(dtype)
        rs.relay_gated(x, x, x.clone(), gate_checkpoint=none)
        rs.relay_gated_backward(x, x, x, gate=x, up=x)
        dw = torch.full((2, 24), 5.0, device="cuda")
        work = torch.empty(rs.relay_rms_norm_backward_workspace(2, 0, 24), dtype=torch.uint8, device="cuda")
        rs.relay_rms_norm_backward(x, _weight(0, 2, 24), rstd, x.clone(), dw, work, total=x)
        assert not dw.any()


def _step(x, dy, w, buffers, stream=None):
    """Norm, weight gradient and norm backward, as a training step makes them."""
    y, rstd, ckpt, dw, work, dx, dn, nwork = buffers
    rs.relay_rms_norm(x, w, y, EPS, rstd=rstd, checkpoint=ckpt, stream=stream)
    rs.relay_weight_grad(dy, ckpt, dw, work, column_scale=w, stream=stream)
    rs.relay_rms_norm_backward(dy, w, rstd, dx, dn, nwork, checkpoint=ckpt, stream=stream)


def _step_buffers(n, T, d):
    new = dict(device="cuda")
    return (torch.empty(n, T, d, dtype=torch.bfloat16, **new), torch.empty(n, T, **new),
            rs.ActivationCheckpoint(n, T, d), torch.empty(n, d, d, **new),
            torch.empty(rs.relay_weight_grad_workspace(n, T, d, d), dtype=torch.uint8, **new),
            torch.empty(n, T, d, dtype=torch.bfloat16, **new), torch.empty(n, d, **new),
            torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, **new))


def test_streams_and_graphs():
    """The calls run in the order of the stream that they are given, and are recorded into a graph
    (no allocation, no synchronisation); the same bits as on the default stream."""
    n, T, d = 2, 333, 264
    x, dy = (torch.from_numpy(_values(s, n, T, d, torch.bfloat16)).cuda().bfloat16() for s in (1, 2))
    w = _weight(3, n, d)
    want = _step_buffers(n, T, d)
    _step(x, dy, w, want)
    torch.cuda.synchronize()
    side, late = torch.cuda.Stream(), _step_buffers(n, T, d)
    held = torch.zeros_like(x)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        held.copy_(x)  # the input is there only once the side stream gets to it
        _step(held, dy, w, late)
    side.synchronize()
    given = _step_buffers(n, T, d)
    _step(x, dy, w, given, stream=side)
    side.synchronize()
    graph, replayed = torch.cuda.CUDAGraph(), _step_buffers(n, T, d)
    with torch.cuda.graph(graph):
        _step(x, dy, w, replayed)
    graph.replay()
    torch.cuda.synchronize()
    for got in (late, given, replayed):
        for a, b in zip(got[:2] + got[3:4] + got[5:7], want[:2] + want[3:4] + want[5:7]):
            assert torch.equal(a, b)
