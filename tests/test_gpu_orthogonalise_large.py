"""The orthogonal update of matrices with a side of up to 65,536, and with both sides above 2,048, against 64 bits."""
import pytest
import torch

from paper_2110_04175_gb300 import build as rs_build

from .test_gpu_orthogonalise import _check, _matrices

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


# the longest side, few and more than 128 rows, either way round; tiles of 256 columns that end inside, and a square of them
@pytest.mark.parametrize("rows,columns", [(1, 65536), (16, 65536), (65536, 16), (130, 65535), (65536, 200), (2305, 2560), (3000, 2500),
                                          (4096, 4096), (2050, 9000)])
def test_large_sides(rows, columns):
    _check(_matrices(rows, 1, rows, columns))
