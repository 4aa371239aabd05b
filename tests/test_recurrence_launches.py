"""What the recurrence enqueues and in which order, on the CPU with a runtime that launches nothing: tensor maps (M) before the
first launch (L), so that nothing is enqueued where one cannot be made, and no launch behind one that failed."""
import ctypes

import pytest

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import layers

from .fake_cuda import library

A = 1 << 30  # addresses that are never used, each 16 GB from the last


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    fake = library(tmp_path_factory.mktemp("recurrence"), "recurrence.cu")
    layers._library()
    for name in ("relay_recurrence_workspace", "relay_recurrence", "relay_recurrence_backward"):
        fn = getattr(fake, name)
        fn.restype, fn.argtypes = layers._SIGNATURES[name]
    return fake


# tokens and width of one sequence in bf16: segments by tensor copies, segments of rows that are not aligned, one strip of
# tokens by a cluster, and by single loads
SEGMENTS, ODD, CLUSTER, FEW = (16384, 256), (16384, 257), (4096, 1024), (8, 256)


def _call(lib, back, tokens, d, bad_launch=-1, bad_map=-1):
    def rows(i):
        return layers._pack_rows(A * 16 * i, tokens * d, d)
    need = lib.relay_recurrence_workspace(1, tokens, d)
    lib.fake_start(bad_launch, bad_map)
    if back:
        rc = lib.relay_recurrence_backward(0, 1, tokens, d, rows(1), rows(2), rows(3), rows(4), None, 0, None, 0, None, None,
                                           rows(5), rows(6), None, 0, A, need, None)
    else:
        rc = lib.relay_recurrence(0, 1, tokens, d, rows(1), rows(2), None, 0, None, None, rows(3), None, 0, A, need, None)
    return rc, lib.fake_log().decode()


@pytest.mark.parametrize("back", [False, True], ids=["forward", "backward"])
def test_order(lib, back):
    maps = "MMMM" if back else "MM"
    assert _call(lib, back, *SEGMENTS) == (rs.RELAY_OK, maps + "LL")
    assert _call(lib, back, *ODD) == (rs.RELAY_OK, "LL")
    assert _call(lib, back, *CLUSTER) == (rs.RELAY_OK, maps + "L")
    assert _call(lib, back, *FEW) == (rs.RELAY_OK, "L")


@pytest.mark.parametrize("back", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("size", [SEGMENTS, ODD, CLUSTER, FEW], ids=["segments", "odd", "cluster", "few"])
def test_a_launch_that_fails_is_the_last(lib, back, size):
    launches = _call(lib, back, *size)[1].count("L")
    for bad in range(launches):
        rc, log = _call(lib, back, *size, bad_launch=bad)
        assert rc == rs.RELAY_ECUDA and log.count("L") == bad + 1
    assert _call(lib, back, *size)[0] == rs.RELAY_OK  # no error stays behind


@pytest.mark.parametrize("back", [False, True], ids=["forward", "backward"])
@pytest.mark.parametrize("size", [SEGMENTS, CLUSTER], ids=["segments", "cluster"])
def test_nothing_is_enqueued_without_maps(lib, back, size):
    for bad in range(4 if back else 2):
        rc, log = _call(lib, back, *size, bad_map=bad)
        assert rc == rs.RELAY_ECUDA and "L" not in log
