"""What the orthogonal update refuses, without a GPU."""
import numpy as np
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import layers

A = 1 << 20  # addresses that are never used
OK, BAD, BIG = rs.RELAY_OK, rs.RELAY_EINVAL, rs.RELAY_EUNSUPPORTED


@pytest.fixture(scope="module")
def lib():
    rs_build.build()
    return layers._library()


def _call(lib, n=2, rows=30, columns=50, update=A, uw=1500, ur=50, steps=5, eps=1e-7, scale=1.0, out=64 * A, ow=1500, orow=50,
          work=128 * A, size=1 << 40):
    return lib.relay_orthogonalise(n, rows, columns, update, uw, ur, steps, eps, scale, out, ow, orow, work, size, None)


def test_arguments(lib):
    need = lib.relay_orthogonalise_workspace(2, 30, 50)
    nan, inf = float("nan"), float("inf")
    for kw in (dict(n=0), dict(rows=0), dict(columns=0), dict(rows=-1), dict(update=None), dict(update=A + 2), dict(uw=-1),
               dict(ur=-1), dict(out=None), dict(out=64 * A + 1), dict(ow=1499), dict(orow=49), dict(steps=0), dict(steps=101),
               dict(eps=-1e-9), dict(eps=nan), dict(eps=inf), dict(scale=nan), dict(scale=inf), dict(scale=-inf),
               dict(work=None), dict(work=A + 8), dict(size=need - 1), dict(out=A, ow=1600), dict(out=A, orow=100, ow=3000)):
        assert _call(lib, **kw) == BAD, kw
    for kw in (dict(n=257), dict(rows=65537), dict(columns=65537)):
        assert _call(lib, **kw) == BIG, kw
        assert lib.relay_orthogonalise_workspace(*{**dict(n=2, rows=30, columns=50), **kw}.values()) == BIG
    assert lib.relay_orthogonalise_workspace(2, 0, 5) == BAD


def test_workspace_is_that_of_the_transpose(lib):
    r = np.random.default_rng(0)
    for _ in range(200):
        n, a, b = int(r.integers(1, 257)), int(2 ** r.uniform(0, 13)), int(2 ** r.uniform(0, 13))
        size = lib.relay_orthogonalise_workspace(n, a, b)
        assert size == lib.relay_orthogonalise_workspace(n, b, a) and size % 4 == 0
        assert size >= 8 * n * a * b + 8 * n * min(a, b) ** 2


def test_binding_refuses_tensors_that_do_not_fit(lib):
    x = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError, match="current CUDA device"):
        rs.relay_orthogonalise(x, x, x)
    for bad in (torch.zeros(3, 4), None, 3):
        with pytest.raises(ValueError):
            rs.relay_orthogonalise(bad, x, x)
    with pytest.raises(rs.RelayError):
        rs.relay_orthogonalise_workspace(0, 3, 4)


@pytest.mark.gpu
def test_binding_refuses_other_types_shapes_and_strides():
    x = torch.zeros(2, 30, 50, device="cuda")
    work = torch.empty(rs.relay_orthogonalise_workspace(2, 30, 50), dtype=torch.uint8, device="cuda")
    for args in ((x.half(), x.half()), (x, x[:, :29]), (x, x.half()), (x.transpose(1, 2), x.transpose(1, 2))):
        with pytest.raises(ValueError):
            rs.relay_orthogonalise(*args, work)
    with pytest.raises(rs.RelayError):
        rs.relay_orthogonalise(x, x, work[:1000])
    with pytest.raises(rs.RelayError):
        rs.relay_orthogonalise(x, x, work, steps=0)
