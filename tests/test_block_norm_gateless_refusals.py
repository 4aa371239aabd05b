"""What the backward step between blocks refuses where there is no gate, without a GPU: the gradients of x and of the
residual are needed whether or not that of the gate is."""
import pytest

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import layers

A = 1 << 20  # addresses that are never used, each a megabyte from the last


@pytest.fixture(scope="module")
def lib():
    rs_build.build()
    return layers._library()


def _r(data, ws=640, ts=64):
    return layers._pack_rows(data, ws, ts)


def _backward(lib, tokens=10, dx=_r(5 * A), dr=_r(6 * A), dgate=None):
    return lib.relay_block_norm_backward(0, 2, tokens, 64, _r(A), None, _r(2 * A), None, _r(3 * A), 7 * A, 64, 8 * A, 64, None, 0,
                                         9 * A, None, dx, dgate, dr, 10 * A, 64, 11 * A, 64, None, 0, 12 * A, 1 << 40, None)


@pytest.mark.parametrize("tokens", [0, 1, 10])
def test_rows_that_are_needed(lib, tokens):
    for kw in (dict(dx=None), dict(dr=None), dict(dx=None, dr=None), dict(dgate=_r(4 * A))):
        assert _backward(lib, tokens, **kw) == rs.RELAY_EINVAL, kw


def test_rows_that_do_not_fit(lib):
    for kw in (dict(dx=_r(0)), dict(dr=_r(0)), dict(dx=_r(5 * A + 1)), dict(dr=_r(6 * A, 639)), dict(dr=_r(6 * A, 640, 63)),
               dict(dx=_r(A)), dict(dr=_r(3 * A)), dict(dr=_r(5 * A))):
        assert _backward(lib, **kw) == rs.RELAY_EINVAL, kw
