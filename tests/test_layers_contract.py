"""What relaylayers.h promises about sizes and arguments, without a GPU."""
import random

import pytest

from paper_2110_04175_gb300 import build as rs_build
from paper_2110_04175_gb300 import layers

A = 1 << 20  # an address that is never used


@pytest.fixture(scope="module")
def lib():
    rs_build.build()
    return layers._library()


def _shapes(count):
    r = random.Random(0)
    yield from [(3, 13866, 72, 6969), (4, 11644, 71, 6002), (1, 9195, 88, 522), (1, 9639, 88, 522)]
    for _ in range(count):
        yield (r.choice([1, 2, 3, 4, 8, 16, 256]), int(2 ** r.uniform(0, 15)), int(2 ** r.uniform(0, 12)),
               int(2 ** r.uniform(0, 13)))


def test_workspace_without_rows_is_enough_for_every_call(lib):
    """The size for RELAY_FP32 and no dy covers each type, with rows that are copied and rows that are
    not, at as many tokens and at fewer."""
    size, r = lib.relay_weight_grad_workspace, random.Random(1)
    for n, tokens, outputs, inputs in _shapes(3000):
        most = size(layers.RELAY_FP32, n, tokens, outputs, inputs, None)
        for type_ in (layers.RELAY_BF16, layers.RELAY_FP16, layers.RELAY_FP32):
            bound = size(type_, n, tokens, outputs, inputs, None)
            assert bound <= most, (n, tokens, outputs, inputs)
            wide = (outputs + 7) // 8 * 8
            for t in (tokens, r.randint(1, tokens), max(tokens - 64, 1), max(tokens - 500, 1), 0):
                for address in (A, A + 4):  # (bf16: by TMA, and copied)
                    rows = layers._pack_rows(address, tokens * wide, wide)
                    assert 0 <= size(type_, n, t, outputs, inputs, rows) <= bound, (type_, n, tokens, t, outputs, inputs)
                assert size(type_, n, t, outputs, inputs, None) <= bound


def test_total_on_other_rows_of_an_inputs_buffer_is_refused(lib):
    """total may be the view of x or of the residual; one that starts where they do with other strides
    would overwrite rows that are still to be read (x repeated for all workers, its first row as total's)."""
    x, r, other = layers._pack_rows(A, 0, 64), layers._pack_rows(2 * A, 640, 64), layers._pack_rows(3 * A, 640, 64)

    def call(x, residual, total, n=2, tokens=10):
        return lib.relay_rms_norm(0, n, tokens, 64, x, residual, 4 * A, 64, 1e-5, total, other, None, None, None, None)

    repeated, crosswise = layers._pack_rows(A, 640, 64), layers._pack_rows(2 * A, 64, 128)
    assert call(x, r, repeated) == -1  # RELAY_EINVAL
    assert call(repeated, r, crosswise) == -1
    assert call(r, None, crosswise) == -1
