"""The norm where a CTA takes several groups of rows one after the other, forward (rows asked for
ahead) and backward, at every width's instance, against 64 bits; and how far the weight's gradient
is off where one worker has very many rows.  References in float64 on the GPU."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

from .layers_util import CHAIN, LEAST, ROUND, U

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _within(got, want, bound):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (float((off - bound).max()), int((off > bound).sum()))


def _rounded(want, dtype, bound):
    return bound + ROUND[dtype] * (want.abs() + bound) + LEAST[dtype]


def _random(seed, *shape, dtype, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * size).to(dtype)


def _held(ckpt, d):
    """A checkpoint's values in float64, by the format's formula."""
    unit = torch.pow(2.0, ckpt.scales.double() - 133).repeat_interleave(32, -1)
    return (ckpt.codes.double() * unit)[..., :d]


# CTAs that stay take 456 / n groups of max(1, 8 / warps of a row) rows of a worker at a time
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("n,T,d,residual", [(4, 1203, 200, False), (4, 1203, 512, False), (4, 1203, 1000, False),
                                            (4, 1203, 2048, False), (4, 1203, 4096, False), (2, 601, 8192, False),
                                            (2, 601, 8192, True), (2, 601, 5000, True), (256, 19, 256, False),
                                            (300 // 2, 13, 4096, False), (4, 1203, 4096, True)])
def test_norm_of_many_rows(dtype, n, T, d, residual):
    x, w = _random(1, n, T, d, dtype=dtype), 1 + _random(2, n, d, dtype=torch.float32, size=0.3)
    r = _random(3, n, T, d, dtype=dtype) if residual else None
    x *= torch.exp2(torch.arange(T, device="cuda") % 5 - 2)[:, None].to(dtype)  # each row its own size
    y, total = torch.empty_like(x), torch.empty_like(x)
    rstd, ckpt = torch.empty(n, T, device="cuda"), rs.ActivationCheckpoint(n, T, d)
    rs.relay_rms_norm(x, w, y, EPS, residual=r, total=total, rstd=rstd, checkpoint=ckpt)
    h = x.double() if r is None else x.double() + r.double()
    s = 1 / (h.square().mean(-1) + float(torch.tensor(EPS))).sqrt()
    xhat = h * s[..., None]
    want = xhat * w.double()[:, None]
    _within(total, h, _rounded(h, dtype, U * h.abs()))
    _within(rstd, s, CHAIN * U * s)
    _within(y, want, _rounded(want, dtype, CHAIN * U * want.abs()))
    got = _held(ckpt, d)
    most = torch.nn.functional.pad(xhat.abs(), (0, -d % 32)).unflatten(-1, (-1, 32)).amax(-1)
    step = (most / 127.5).repeat_interleave(32, -1)[..., :d]
    _within(got, xhat, step * (1 + 2.0 ** -10) + CHAIN * U * xhat.abs())
    only = torch.empty_like(y)
    rs.relay_rms_norm(x, w, only, EPS, residual=r)
    assert torch.equal(only, y)
    if r is not None:
        rs.relay_rms_norm(x, w, only, EPS, residual=r, total=x)  # in place
        assert torch.equal(only, y) and torch.equal(x, total)


# a worker has 304 / 16 = 19 CTAs; T is past twice what they take side by side, and ends within a group
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("source", ["checkpoint", "total"])
@pytest.mark.parametrize("d,T", [(200, 315), (94, 315), (512, 315), (500, 315), (1000, 157), (1001, 157), (2048, 79),
                                 (1999, 79), (4096, 41), (4001, 41), (8192, 41), (8001, 41), (16384, 41), (12001, 41),
                                 (32768, 41), (20001, 41), (201, 16387)])
def test_norm_backward_of_many_rows(dtype, source, d, T):
    n = 16
    h, dy = _random(1, n, T, d, dtype=dtype), _random(2, n, T, d, dtype=dtype, size=0.01)
    dh, w = _random(3, n, T, d, dtype=dtype, size=0.01), 1 + _random(4, n, d, dtype=torch.float32, size=0.3)
    lengths = torch.tensor([T, T - 1, T // 2 + 3, 1, 0, 19, 20, 38, 39, T - 2, T // 3, T, 5, T - 7, 2, T],
                           dtype=torch.int32, device="cuda")
    used = (torch.arange(T, device="cuda")[None] < lengths[:, None])[..., None]
    s = (1 / (h.double().square().mean(-1) + EPS).sqrt()).float()
    kw = {}
    if source == "checkpoint":
        kept = rs.ActivationCheckpoint(n, T, d).pack((h.float() * s[..., None]).to(dtype))
        xhat, kw["checkpoint"] = _held(kept, d), kept
    else:
        xhat, kw["total"] = h.double() * s.double()[..., None], h
    for t in (h, dy, dh, s):
        t.masked_fill_(~(used if t.dim() == 3 else used[..., 0]), float("nan"))  # padding is not read
    dx, dw = torch.empty_like(dy), torch.empty(n, d, device="cuda")
    work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    rs.relay_rms_norm_backward(dy, w, s, dx, dw, work, dtotal=dh, lengths=lengths, **kw)
    g, add, s64 = (torch.where(used, t, 0).double() for t in (dy, dh, s[..., None]))
    xhat = torch.where(used, xhat, 0)
    u = g * w.double()[:, None]
    along, spread = ((f(u * xhat)).sum(-1, keepdim=True) / d for f in (lambda v: v, torch.abs))
    want = s64 * (u - xhat * along) + add
    bound = U * (8 * (s64 * (u.abs() + (xhat * along).abs()) + add.abs()) + CHAIN * s64 * xhat.abs() * spread)
    _within(dx, want, _rounded(want, dtype, 2 * bound))  # xhat from the total is one more rounding
    _within(dw, (g * xhat).sum(1), (T + 64) * U * (g * xhat).abs().sum(1))
    assert not torch.where(used, 0, dx).any()


# the sum of N products of random sign in a chain of fp32 additions is off by U sqrt(N / 6) of itself
# (each addition rounds by U / sqrt(3) of a partial sum, which grows like a random walk); chains of 256,
# and their join in 8 shorter ones: 3.9e-7 and less than 2e-7
@pytest.mark.parametrize("n,T,d", [(160, 4096, 2304), (256, 2051, 4096), (16, 16384, 4096), (1, 30000, 8200)])
def test_norm_weight_gradient_of_many_rows(n, T, d):
    dtype = torch.bfloat16
    h, dy = _random(1, n, T, d, dtype=dtype), _random(2, n, T, d, dtype=dtype)
    s = torch.ones(n, T, device="cuda")
    dx, dw = torch.empty_like(dy), torch.empty(n, d, device="cuda")
    work = torch.empty(rs.relay_rms_norm_backward_workspace(n, T, d), dtype=torch.uint8, device="cuda")
    rs.relay_rms_norm_backward(dy, torch.ones(n, d, device="cuda"), s, dx, dw, work, total=h)
    for i in sorted({0, n // 2, n - 1}):
        want = (dy[i].double() * h[i].double()).sum(0)
        assert float((dw[i].double() - want).norm() / want.norm()) < 5e-7
