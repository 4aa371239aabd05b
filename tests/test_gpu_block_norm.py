"""The step from one block to the next on the GPU against its definition in 64 bits: types, layouts, widths at every
instance's border, with and without gate, scale, checkpoint and lengths; gradients against differences; values that are
not numbers; streams and graphs."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

from . import layers_util as lu
from .layers_util import CHAIN, LEAST, ROUND, TYPES, U, np64, sigmoid, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _held(values, dtype):
    return np64(torch.from_numpy(values).to(dtype))


def _values(seed, n, T, d, dtype, size=1.0):
    g = np.random.default_rng(seed)
    return _held(g.standard_normal((n, T, d)) * np.where(g.random(d) < 1 / 16, 20.0, 1.0) * size, dtype)


def _weight(seed, n, d, first=0):
    w = torch.from_numpy(1 + 0.3 * np.random.default_rng(seed).standard_normal((n, first + d + 7))).float().cuda()
    return w[:, first:first + d]


def _rounded(want, dtype, bound):
    return bound + ROUND[dtype] * (np.abs(want) + bound) + LEAST[dtype]


def _used(lengths, n, T):
    return lu.used_rows(lengths, n, T)


def _gate_off(z):
    """As if the gate were moved by this: the exponential's argument, the exponential, sum and reciprocal."""
    return 0 if z is None else (4 + np.abs(z)) * 2.0 ** -23


def _forward(x, z, r, post, pre, rho):
    """The definition, and bounds of h, y, s_x and s_h before the outputs' rounding.

    s_x is off by half of what its mean is, CHAIN U, and a few roundings; m and the gate's product by
    their factors' errors (4 roundings, the gate's slope); h's error, weighed as its squares are, is half
    of what moves s_h: |h| <= H = rho |r| + p |m|, so mean(h^2) is off by 2 mean(|h| e_h)."""
    d = x.shape[-1]
    sx = 1 / np.sqrt((x * x).mean(-1) + EPS)
    sx_off = (CHAIN / 2 + 6) * U
    m = x * sx[..., None] * post[:, None]
    p, q = (np.ones_like(x), 0) if z is None else (sigmoid(z), sigmoid(-z))
    a, b = p * m, r * (1 if rho is None else rho[:, None])
    h = a + b
    eh = np.abs(a) * (sx_off + 5 * U + _gate_off(z) * q) + 2 * U * (np.abs(a) + np.abs(b))
    sh = 1 / np.sqrt((h * h).mean(-1) + EPS)
    sh_off = (CHAIN / 2 + 6) * U + (np.abs(h) * eh).sum(-1) / d * sh * sh
    y = h * sh[..., None] * pre[:, None]
    ey = np.abs(pre[:, None]) * sh[..., None] * (eh + np.abs(h) * (sh_off[..., None] + 4 * U))
    return h, y, sx, sh, eh, ey, sx * sx_off, sh * sh_off


def _backward(dy, over, x, z, r, post, pre, rho, sx, sh, used):
    """(dx, dz, dr, dpost, dpre, drho) and their bounds before the rounding of 16-bit outputs."""
    T, d = x.shape[1:]
    dy, over = np.where(used, dy, 0), np.where(used, 0 if over is None else over, 0)
    x, r = np.where(used, x, 0), np.where(used, r, 0)
    sx, sh = np.where(used, sx[..., None], 0), np.where(used, sh[..., None], 0)
    post, pre = post[:, None], pre[:, None]
    rho = np.ones_like(post) if rho is None else rho[:, None]
    p, q = (np.ones_like(x), np.zeros_like(x)) if z is None else (sigmoid(z), sigmoid(-z))
    off = _gate_off(None if z is None else np.where(used, z, 0))
    xhat = x * sx
    m = xhat * post
    hhat = (rho * r + p * m) * sh
    H = (np.abs(rho * r) + np.abs(p * m)) * sh  # what hhat is a difference of
    eH = (6 * U + off * q) * H
    u = dy * pre
    along = (u * hhat).sum(-1, keepdims=True) / d
    spread = (np.abs(u) * (CHAIN * U * np.abs(hhat) + eH + 4 * U * np.abs(hhat))).sum(-1, keepdims=True) / d
    dh = sh * (u - hhat * along) + over
    edh = sh * (4 * U * (np.abs(u) + np.abs(hhat * along)) + eH * np.abs(along) + np.abs(hhat) * spread) + 2 * U * np.abs(over)
    Dh = sh * (np.abs(u) + np.abs(hhat * along)) + np.abs(over)  # dh's own magnitudes
    edh = edh + 2 * U * Dh
    v = dh * p * post
    ev = np.abs(p * post) * (edh + (off * q + 4 * U) * np.abs(dh))
    along_x = (v * xhat).sum(-1, keepdims=True) / d
    # The kernels sum a (s_h u + dtotal), a hhat and u hhat, a = p xhat w_post, in one pass: their difference is
    # the mean of v xhat, and its terms are as large as a Dh, however small v is (one feature: v is nearly 0).  Each
    # sum is off by CHAIN U of its terms' magnitudes, products and the difference by a few U, and hhat and `along`
    # by what edh has of them.
    a = np.abs(p * m)
    spread_x = (ev * np.abs(xhat) + a * ((CHAIN + 10) * U * Dh + off * q * Dh) + sh * a * (np.abs(hhat) * spread + eH * np.abs(along))
                ).sum(-1, keepdims=True) / d
    dx = sx * (v - xhat * along_x)
    edx = sx * (ev + 4 * U * (np.abs(v) + np.abs(xhat * along_x)) + np.abs(xhat) * spread_x)
    dz = dh * m * p * q
    edz = np.abs(m * p * q) * (edh + (2 * off + 8 * U) * np.abs(dh))
    dr, edr = rho * dh, np.abs(rho) * (edh + 2 * U * np.abs(dh))
    sums = []
    for a, ea, b, eb in ((dh * p, np.abs(p) * (edh + (off * q + 3 * U) * np.abs(dh)), xhat, 2 * U * np.abs(xhat)),
                         (dy, 0, hhat, eH + 2 * U * np.abs(hhat)), (dh, edh, r, 0)):
        want = (a * b).sum(1)
        sums.append((want, ((T + 64) * U * np.abs(a * b) + ea * np.abs(b) + np.abs(a) * eb).sum(1)))
    return [(dx, edx), (dz, edz), (dr, edr), *sums]


def _check(n, T, d, dtype, layout="dense", gate=True, scale=True, ckpt=True, over=True, lengths=None, first=0, seed=0):
    x, r = _values(seed, n, T, d, dtype, 0.7), _values(seed + 1, n, T, d, dtype)
    z = _held(np.random.default_rng(seed + 2).standard_normal((n, T, d)) * 2, dtype) if gate else None
    post, pre = _weight(seed + 3, n, d, first), _weight(seed + 4, n, d, first)
    rho = _weight(seed + 5, n, d, first) if scale else None
    w, v, rh = np64(post), np64(pre), None if rho is None else np64(rho)

    def put(a):
        return None if a is None else lu.rows(a, dtype, layout)[0]

    X, R, Z = put(x), put(r), put(z)
    total, tbuf = lu.empty_rows(n, T, d, dtype, layout)
    y, ybuf = lu.empty_rows(n, T, d, dtype, layout)
    rstd = torch.full((2, n, T), 77.0, device="cuda")
    kept = rs.ActivationCheckpoint(n, T, d) if ckpt else None
    rs.relay_block_norm(X, R, post, pre, total, y, EPS, gate=Z, scale=rho, rstd=rstd, checkpoint=kept)
    h, want, sx, sh, eh, ey, esx, esh = _forward(x, z, r, w, v, rh)
    within(total, h, _rounded(h, dtype, eh))
    within(y, want, _rounded(want, dtype, ey))
    within(rstd, np.stack([sx, sh]), np.stack([esx, esh]))
    assert lu.only_rows_written(total, tbuf) and lu.only_rows_written(y, ybuf)
    if ckpt:
        hhat = h * sh[..., None]
        step = lu.half_step(hhat) * (1 + 1e-5)
        within(torch.from_numpy(lu.held(kept.codes.cpu().numpy(), kept.scales.cpu().numpy(), d)), hhat,
               step + ey / np.abs(v[:, None]))

    dy = _values(seed + 6, n, T, d, dtype, 0.05)
    dh = _values(seed + 7, n, T, d, dtype, 0.05) if over else None
    S = np64(rstd)
    outs = [lu.empty_rows(n, T, d, dtype, layout) for _ in range(3 if gate else 2)]
    grads = [torch.full((n, d + 5), 77.0, device="cuda")[:, first % 4:first % 4 + d] for _ in range(3)]
    work = torch.empty(rs.relay_block_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    size = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    rs.relay_block_norm_backward(put(dy), X, R, post, pre, rstd, outs[0][0], outs[1][0], grads[0], grads[1], work, gate=Z,
                                 scale=rho, dtotal=put(dh), dgate=outs[2][0] if gate else None,
                                 dscale=grads[2] if scale else None, lengths=size)
    used = _used(None if lengths is None else np.array(lengths), n, T)
    (dx, edx), (dz, edz), (dr, edr), *sums = _backward(dy, dh, x, z, r, w, v, rh, S[0], S[1], used)
    within(outs[0][0], dx, _rounded(dx, dtype, edx))
    within(outs[1][0], dr, _rounded(dr, dtype, edr))
    if gate:
        within(outs[2][0], dz, _rounded(dz, dtype, edz))
    for got, (want, bound), there in zip(grads, sums, (True, True, scale)):
        if there:
            within(got, want, bound + 2.0 ** -149)
        else:
            assert bool((got == 77).all())
    assert all(lu.only_rows_written(*o) for o in outs)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("layout", ["dense", "wide", "odd", "tokens"])
def test_types_and_layouts(dtype, layout):
    for d in (1, 7, 64, 100, 256, 264, 515, 1000):
        _check(3, 5, d, dtype, layout, lengths=[5, 0, 3], first=d % 3, seed=d)


@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("d", [256, 257, 512, 1024, 1025, 2048, 2050, 4096, 4104, 8192, 8200, 16384, 16385, 32768])
def test_widths(dtype, d):
    _check(2, 11, d, dtype, lengths=[11, 4], seed=d)


@pytest.mark.parametrize("gate", [False, True], ids=["", "gate"])
@pytest.mark.parametrize("scale", [False, True], ids=["", "scale"])
@pytest.mark.parametrize("over", [False, True], ids=["", "dtotal"])
def test_options(gate, scale, over):
    for T in (1, 9):
        _check(3, T, 328, torch.bfloat16, gate=gate, scale=scale, over=over, ckpt=gate, seed=T)
        _check(2, T, 333, torch.float32, gate=gate, scale=scale, over=over, ckpt=scale, seed=T)


@pytest.mark.parametrize("n,T,d", [(2, 1500, 200), (3, 700, 1000), (1, 900, 2048), (1, 700, 4096), (200, 9, 64), (1, 90000, 8)])
def test_many_rows(n, T, d):
    """CTAs that take rows one after the other."""
    _check(n, T, d, torch.bfloat16, seed=T)


# the backward pass takes rows by bulk copies from 2^20 features on: 152 / n CTAs of 16 warps (8 in fp32), one to 16 a row
@pytest.mark.parametrize("dtype", TYPES.values(), ids=TYPES)
@pytest.mark.parametrize("n,T,d", [(150, 67, 200), (77, 131, 512), (151, 35, 520), (151, 35, 1024), (152, 18, 1032), (120, 17, 2048),
                                   (152, 9, 2056), (140, 11, 4096), (100, 7, 4104), (90, 5, 8192), (3, 1100, 4096), (256, 66, 64)])
def test_rows_through_shared_memory(dtype, n, T, d):
    if n * T * d > 4e6 and dtype is torch.float16:
        pytest.skip("as bf16")
    lengths = np.random.default_rng(d).integers(0, T + 1, n)
    lengths[0], lengths[-1] = T, 0
    _check(n, T, d, dtype, lengths=list(lengths), first=d % 3, seed=d)


@pytest.mark.parametrize("gate,scale,over", [(False, False, False), (True, False, True), (False, True, False)])
def test_options_of_backward_rows_through_shared_memory(gate, scale, over):
    for dtype in (torch.bfloat16, torch.float32):
        _check(151, 35, 1000, dtype, gate=gate, scale=scale, over=over, ckpt=over, seed=3)


# and the forward pass of 16-bit rows from 2^24 on: 24 warps a CTA, one to 8 a row
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n,T,d,gate,scale", [(3, 10000, 568, True, True), (150, 112, 1024, True, True), (2, 8200, 1032, False, True),
                                              (5, 1700, 2000, True, False), (4, 1025, 4096, True, True), (1, 4100, 4104, True, True),
                                              (256, 9, 8192, False, False)])
def test_forward_rows_through_shared_memory(dtype, n, T, d, gate, scale):
    """The definition and _forward's bounds, in 64 bits on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(d)

    def values(size):
        v = torch.randn(n, T, d, generator=g, device="cuda") * torch.where(torch.rand(d, generator=g, device="cuda") < 1 / 16, 20.0, 1.0)
        return (v * size).to(dtype)

    x, r, z = values(0.7), values(1.0), values(0.5) if gate else None
    post, pre, rho = (_weight(k, n, d, first=k) for k in range(3))
    total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(2, n, T, device="cuda")
    kept = rs.ActivationCheckpoint(n, T, d)
    rs.relay_block_norm(x, r, post, pre, total, y, EPS, gate=z, scale=rho if scale else None, rstd=rstd, checkpoint=kept)
    X, R, W, V = x.double(), r.double(), post.double()[:, None], pre.double()[:, None]
    sx, sx_off = 1 / (X.square().mean(-1, keepdim=True) + EPS).sqrt(), (CHAIN / 2 + 6) * U
    p = torch.sigmoid(z.double()) if gate else torch.ones_like(X)
    off = (4 + z.double().abs()) * 2.0 ** -23 * torch.sigmoid(-z.double()) if gate else 0
    a, b = p * X * sx * W, R * (rho.double()[:, None] if scale else 1)
    h = a + b
    eh = a.abs() * (sx_off + 5 * U + off) + 2 * U * (a.abs() + b.abs())
    sh = 1 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()
    sh_off = (CHAIN / 2 + 6) * U + (h.abs() * eh).sum(-1, keepdim=True) / d * sh * sh
    want, ey = h * sh * V, V.abs() * sh * (eh + h.abs() * (sh_off + 4 * U))

    def near(got, want, bound):
        far = (got.double() - want).abs() - bound
        assert bool((far <= 0).all()), (int((far > 0).sum()), float(far.max()))

    def rounded(want, bound):
        return bound + ROUND[dtype] * (want.abs() + bound) + LEAST[dtype]

    near(total, h, rounded(h, eh))
    near(y, want, rounded(want, ey))
    near(rstd, torch.stack([sx, sh])[..., 0], torch.stack([sx * sx_off, sh * sh_off])[..., 0])
    hhat = h * sh
    wide = torch.nn.functional.pad(hhat, (0, -d % 32)).unflatten(-1, (-1, 32))
    step = (wide.abs().amax(-1) / 127.5).clamp(min=2.0 ** -127).repeat_interleave(32, -1)[..., :d]
    near(kept.unpack(torch.float32), hhat, step * (1 + 1e-5) + ey / V.abs() + U * hhat.abs())
    there = r.clone()
    rs.relay_block_norm(x, there, post, pre, there, y, EPS, gate=z, scale=rho if scale else None)  # the sum in the residual's rows
    assert torch.equal(there, total)


def test_no_tokens():
    n, d = 2, 40
    x = torch.empty(n, 0, d, device="cuda")
    w = torch.ones(n, d, device="cuda")
    rstd, grads = torch.empty(2, n, 0, device="cuda"), [torch.full((n, d), 5.0, device="cuda") for _ in range(3)]
    rs.relay_block_norm(x, x, w, w, x, x, EPS, rstd=rstd)
    work = torch.empty(rs.relay_block_norm_backward_workspace(n, 0, d), dtype=torch.uint8, device="cuda")
    rs.relay_block_norm_backward(x, x, x, w, w, rstd, x, x, *grads[:2], work, scale=w, dscale=grads[2])
    assert not any(g.any() for g in grads)


def test_total_in_place_shared_weights_and_repeated_rows():
    """The sum in the residual's or x's own rows, one weight for all workers, one residual row for all tokens."""
    n, T, d = 3, 17, 200
    x, r = (torch.randn(n, T, d, device="cuda") for _ in range(2))
    w = _weight(0, 1, d).expand(n, d)
    want = [torch.empty_like(x) for _ in range(2)]
    rs.relay_block_norm(x, r, w, w, *want, EPS, scale=w)
    for which in (0, 1):
        a, b, y = x.clone(), r.clone(), torch.empty_like(x)
        rs.relay_block_norm(a, b, w, w, (a, b)[which], y, EPS, scale=w)
        assert torch.equal((a, b)[which], want[0]) and torch.equal(y, want[1])
    one = r[:1, :1].expand(n, T, d)
    got = [torch.empty_like(x) for _ in range(4)]
    rs.relay_block_norm(x, one, w, w, *got[:2], EPS)
    rs.relay_block_norm(x, one.contiguous(), w, w, *got[2:], EPS)
    assert torch.equal(got[0], got[2]) and torch.equal(got[1], got[3])


@pytest.mark.parametrize("n,T,d", [(2, 12, 264), (152, 70, 264)])
def test_padding_may_hold_anything(n, T, d):
    for dtype in (torch.bfloat16, torch.float32):
        args = [torch.randn(n, T, d, device="cuda").to(dtype) for _ in range(5)]  # dy, dtotal, x, gate, residual
        w, rstd = torch.ones(n, d, device="cuda"), torch.rand(2, n, T, device="cuda")
        lengths = torch.tensor([7, 0] + [T] * (n - 2), dtype=torch.int32, device="cuda")
        work = torch.empty(rs.relay_block_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")

        def run():
            outs = [torch.empty(n, T, d, device="cuda", dtype=dtype) for _ in range(3)]
            grads = [torch.empty(n, d, device="cuda") for _ in range(3)]
            dy, over, x, z, r = args
            rs.relay_block_norm_backward(dy, x, r, w, w, rstd, outs[0], outs[1], grads[0], grads[1], work, gate=z, scale=w,
                                         dtotal=over, dgate=outs[2], dscale=grads[2], lengths=lengths)
            return outs, grads

        clean = run()
        for a, bad in zip(args, (np.nan, np.inf, -np.inf, np.nan, np.inf)):
            a[0, 7:], a[1] = bad, bad
        rstd[:, 0, 7:] = np.nan
        dirty = run()
        for a, b in zip(clean[0] + clean[1], dirty[0] + dirty[1]):
            assert torch.equal(a, b)
        assert not any(o[0, 7:].any() or o[1].any() for o in dirty[0])
        assert not any(g[1].any() for g in dirty[1])


def test_gradients_agree_with_differences():
    n, T, d = 2, 9, 40
    torch.manual_seed(0)
    x, r, z, dy, over = (torch.randn(n, T, d, device="cuda") for _ in range(5))
    post, pre, rho = (1 + 0.2 * torch.randn(n, d, device="cuda") for _ in range(3))

    def forward(x, r, z, post, pre, rho):
        total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(2, n, T, device="cuda")
        rs.relay_block_norm(x, r, post, pre, total, y, EPS, gate=z, scale=rho, rstd=rstd)
        return float((y.double() * dy.double()).sum() + (total.double() * over.double()).sum()), rstd

    args = (x, r, z, post, pre, rho)
    rstd = forward(*args)[1]
    g = [torch.empty_like(a) for a in args]
    work = torch.empty(rs.relay_block_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    rs.relay_block_norm_backward(dy, x, r, post, pre, rstd, g[0], g[1], g[3], g[4], work, gate=z, scale=rho, dtotal=over,
                                 dgate=g[2], dscale=g[5])
    for k in range(len(args)):
        step = torch.randn_like(args[k])
        want = float((g[k].double() * step.double()).sum())
        eps = 2.0 ** -8
        a, b = (forward(*[v + s * eps * step if j == k else v for j, v in enumerate(args)])[0] for s in (1, -1))
        # rounding: 2^-20 of some 40 over 2 eps; curvature: eps^2 of third derivatives of the order of
        # the sum of magnitudes (720 terms): 5e-3 and 1e-2
        assert abs((a - b) / (2 * eps) - want) < 0.05 + 1e-3 * abs(want), k


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph():
    n, T, d, dtype = 2, 300, 520, torch.bfloat16
    x, r, z, dy = (torch.randn(n, T, d, device="cuda").to(dtype) for _ in range(4))
    w = 1 + 0.1 * torch.randn(n, d, device="cuda")

    def buffers():
        return ([torch.empty_like(x) for _ in range(5)] + [torch.empty(2, n, T, device="cuda")] +
                [torch.empty(n, d, device="cuda") for _ in range(2)] +
                [torch.empty(rs.relay_block_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")])

    def run(b, stream=None):
        total, y, dx, dr, dz, rstd, dpost, dpre, work = b
        rs.relay_block_norm(x, r, w, w, total, y, EPS, gate=z, rstd=rstd, stream=stream)
        rs.relay_block_norm_backward(dy, x, r, w, w, rstd, dx, dr, dpost, dpre, work, gate=z, dgate=dz, stream=stream)

    sets, streams = [buffers() for _ in range(3)], [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for b, s in zip(sets, streams):
        run(b, s)
    torch.cuda.synchronize()
    for b in sets[1:]:
        assert all(torch.equal(p, q) for p, q in zip(b[:-1], sets[0][:-1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(sets[0])
    x.copy_(torch.randn(n, T, d, device="cuda"))
    graph.replay()
    run(sets[1])
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(sets[0][:-1], sets[1][:-1]))


def test_past_32_bit_offsets():
    """Rows more than 2^31 elements apart."""
    far, T, d = (1 << 31) + 64, 3, 256
    buf = torch.zeros(far + T * d, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((2, T, d), (far, d, 1))
    x.copy_(torch.randn(2, T, d, device="cuda"))
    w, dense = torch.ones(2, d, device="cuda"), x.clone()
    got, want = ([torch.empty_like(dense) for _ in range(2)] for _ in range(2))
    rs.relay_block_norm(x, dense, w, w, *got, EPS)
    rs.relay_block_norm(dense, dense, w, w, *want, EPS)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    rs.relay_block_norm(dense, dense, w, w, got[0], x, EPS)
    assert torch.equal(x, want[1]) and not buf[T * d:far].any()
