"""The orthogonal update on the GPU against its definition in 64 bits: shapes on both sides of the tiles' borders and of
the square, views, values of any size, matrices that hold no number, streams and graphs."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

pytestmark = pytest.mark.gpu
A, B, C = 3.4445, -4.7750, 2.0315
EPS = 1e-7


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


def _work(n, rows, columns):
    return torch.empty(rs.relay_orthogonalise_workspace(n, rows, columns), dtype=torch.uint8, device="cuda")


def _definition(u, steps=5, eps=EPS):
    """The result in 64 bits, and a bound of the kernel's error in the Frobenius norm.

    One product is off by `u` relative to the norms of its operands: two operands of 22 bits and the
    term left out (2^-23, 2^-23, 2^-22), the tensor cores' sums (36 additions of 2^-24 cut, then rounded
    additions), together 1e-6 with some room.  A step passes an error on by at most its largest slope,
    a = 3.4445 (of p(s) / s, and of p at 0), and adds its own three products'."""
    off = 1e-6
    x = u.double() / (torch.linalg.matrix_norm(u.double())[..., None, None] + eps)
    if x.shape[1] > x.shape[2]:
        got, bound = _definition(u.transpose(1, 2), steps, eps)
        return got.transpose(1, 2), bound

    def two(m):  # an upper bound of the spectral norm
        return torch.minimum(torch.linalg.matrix_norm(m), torch.sqrt(m.abs().sum(-1).amax(-1) * m.abs().sum(-2).amax(-1)))

    error = 4 * off * torch.linalg.matrix_norm(x)
    for _ in range(steps):
        g = x @ x.transpose(1, 2)
        p = B * g + C * g @ g
        fx, fg = torch.linalg.matrix_norm(x), torch.linalg.matrix_norm(g)
        sx, sg = two(x).clamp(max=1.25), two(g).clamp(max=1.6)
        of_g = off * sx * fx
        of_p = (abs(B) + 2 * C * sg) * of_g + off * (abs(B) + C * sg) * fg
        error = A * error + off * A * fx + sx * of_p + off * 2.9 * fx
        x = A * x + p @ x
    return x, error


def _matrices(seed, n, rows, columns, size=1.0):
    """Some strong directions over weaker ones, as gradients have them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = max(1, min(rows, columns) // 4)
    strong = torch.randn(n, rows, k, generator=g, device="cuda") @ torch.randn(n, k, columns, generator=g, device="cuda")
    return (strong / k ** 0.5 + 0.3 * torch.randn(n, rows, columns, generator=g, device="cuda")) * size


def _check(u, out=None, steps=5, scale=1.0):
    n, rows, columns = u.shape
    out = torch.full_like(u, 77.0) if out is None else out
    want, bound = _definition(u.clone(), steps)
    rs.relay_orthogonalise(u, out, _work(n, rows, columns), steps=steps, eps=EPS, scale=scale)
    off = torch.linalg.matrix_norm(out.double() - scale * want)
    bound = abs(scale) * (bound + 2.0 ** -23 * torch.linalg.matrix_norm(want))
    assert bool((off <= bound).all()), (float((off / bound).max()), u.shape)
    # element by element no entry is far from its place
    spread = torch.sqrt((want * want).mean((1, 2), keepdim=True)) * abs(scale)
    assert float(((out.double() - scale * want).abs() / spread.clamp(min=1e-30)).max()) < 0.05
    return out


SHAPES = [(512, 530), (513, 530), (1, 1), (1, 9), (9, 1), (2, 3), (16, 16), (15, 64), (64, 65), (65, 64), (128, 128), (127, 300), (300, 129), (256, 256),
          (257, 256), (256, 513), (511, 257), (640, 640), (200, 4001), (4001, 100), (1000, 777), (1025, 1300)]


@pytest.mark.parametrize("rows,columns", SHAPES)
def test_shapes(rows, columns):
    _check(_matrices(rows, 2, rows, columns))


@pytest.mark.parametrize("n,rows,columns", [(1, 128, 9728), (1, 128, 9729), (152, 64, 64), (153, 65, 64), (76, 100, 128), (3, 120, 3000),
                                            (5, 129, 300), (1, 1, 5000), (38, 33, 257)])
def test_up_to_128_rows(n, rows, columns):
    """A step in one launch (in slices of 64 or 128 columns), and where that does not fit."""
    _check(_matrices(n, n, rows, columns))
    if n * rows * columns < 3e6:
        _check(_matrices(n, n, columns, rows))


@pytest.mark.parametrize("n", [1, 3, 5, 200, 256])
def test_many_matrices(n):
    u = _matrices(n, n, 40, 72) * torch.exp(torch.arange(n, device="cuda") % 7 - 3.0)[:, None, None]
    _check(u)


def test_singular_values_come_near_one():
    u = _matrices(0, 2, 300, 500)
    s = torch.linalg.svdvals(_check(u).double())
    least = torch.linalg.svdvals(u.double()) / torch.linalg.matrix_norm(u.double())[:, None]
    assert float(s.max()) < 1.21 and float(s[least > 0.003].min()) > 0.67


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
def test_steps_and_scale(steps):
    _check(_matrices(steps, 2, 90, 140), steps=steps, scale=-0.25)
    _check(_matrices(steps, 2, 140, 90), steps=steps, scale=3.0)
    _check(_matrices(steps, 2, 90, 90), steps=steps, scale=0.0)


@pytest.mark.parametrize("rows,columns", [(70, 130), (130, 70), (33, 64), (257, 100)])
def test_views_and_in_place(rows, columns):
    """Matrices in model rows at any offset, rows apart, and the result over the update."""
    n, first = 3, 5
    u = _matrices(1, n, rows, columns)
    want = _check(u)
    buf = torch.full((n, first + rows * columns + 9), 77.0, device="cuda")
    view = buf[:, first:first + rows * columns].unflatten(1, (rows, columns))
    view.copy_(u)
    rs.relay_orthogonalise(view, view, _work(n, rows, columns))
    assert torch.equal(view, want)
    assert bool((buf[:, :first] == 77).all()) and bool((buf[:, first + rows * columns:] == 77).all())
    wide = torch.full((rows, n, columns + 3), 77.0, device="cuda")
    apart = wide.transpose(0, 1)[..., 1:1 + columns]
    rs.relay_orthogonalise(u, apart, _work(n, rows, columns))
    assert torch.equal(apart, want) and bool((wide[..., 0] == 77).all()) and bool((wide[..., 1 + columns:] == 77).all())
    one = u[:1].expand(n, rows, columns)
    rs.relay_orthogonalise(one, apart, _work(n, rows, columns))
    assert torch.equal(apart, want[:1].expand(n, rows, columns))


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-15, 1e15, 1e30, 1e37])
def test_values_of_any_size(size):
    """Squares that leave fp32: the same result as for ordinary values, apart from eps and subnormals."""
    u = _matrices(2, 2, 60, 90)
    want = torch.empty_like(u)
    rs.relay_orthogonalise(u, want, _work(2, 60, 90), eps=0.0)
    out = torch.empty_like(u)
    rs.relay_orthogonalise(u * size, out, _work(2, 60, 90), eps=0.0)
    # the product by `size` rounds: 2^-24 of each value, or half of 2^-149; five steps pass on up to 485 times that
    assert float(torch.linalg.matrix_norm(out - want).max()) < 485 * 2 * max(2.0 ** -24, 2.0 ** -150 * 75 / size)


def test_zeros_and_values_that_are_not_numbers():
    u = _matrices(3, 5, 50, 80)
    want = _check(u)
    u[0] = 0
    u[1, 3, 7], u[2, 49, 79], u[3, 0, 0] = float("nan"), float("inf"), -float("inf")
    for eps in (EPS, 0.0):
        out = torch.empty_like(u)
        rs.relay_orthogonalise(u, out, _work(5, 50, 80), eps=eps)
        assert not out[0].any() and torch.isnan(out[1:4]).all()
        assert eps == 0 or torch.equal(out[4], want[4])


def test_large():
    _check(_matrices(4, 1, 2048, 2304))


def test_past_32_bit_offsets():
    rows, columns, far = 40, 60, (1 << 31) + 96
    buf = torch.zeros(far + rows * columns, device="cuda")
    view = buf.as_strided((2, rows, columns), (far, columns, 1))
    u = _matrices(5, 2, rows, columns)
    want = _check(u)
    view.copy_(u)
    rs.relay_orthogonalise(view, view, _work(2, rows, columns))
    assert torch.equal(view, want) and not buf[rows * columns:far].any()


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph():
    n, rows, columns = 2, 200, 330
    u = _matrices(6, n, rows, columns)
    outs, works = [torch.empty_like(u) for _ in range(3)], [_work(n, rows, columns) for _ in range(3)]
    streams = [torch.cuda.Stream() for _ in outs]
    torch.cuda.synchronize()
    for out, work, stream in zip(outs, works, streams):
        rs.relay_orthogonalise(u, out, work, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rs.relay_orthogonalise(u, outs[0], works[0])
    u.copy_(_matrices(7, n, rows, columns))
    graph.replay()
    rs.relay_orthogonalise(u, outs[1], works[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
