"""Instances of the recurrence and of the step between blocks that fp16 rows alone reach, at sizes that the other tests leave
to bf16: whole rows through shared memory for every number of warps a row, and strips shared by one, four and eight CTAs with
beginnings and without."""
import pytest
import torch

from paper_2110_04175_gb300 import build as rs_build

from . import test_gpu_block_norm, test_gpu_recurrence

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


# 2^20 features and more: the backward pass takes 1, 2, 4, 8 and 16 warps a row, all their quads there and not
@pytest.mark.parametrize("n,T,d", [(3, 700, 512), (3, 790, 448), (3, 350, 1024), (3, 380, 968), (2, 260, 2048), (2, 300, 1800),
                                   (2, 130, 4096), (2, 140, 3976), (1, 130, 8192), (1, 160, 6600)])
def test_block_norm_backward(n, T, d):
    test_gpu_block_norm._check(n, T, d, torch.float16, lengths=[T, T // 2, 1][:n], first=d % 3, seed=d)


@pytest.mark.parametrize("gate,scale,over", [(False, True, True), (True, False, False)])
@pytest.mark.parametrize("n,T,d", [(3, 700, 512), (2, 130, 4096)])
def test_options_of_block_norm_backward(n, T, d, gate, scale, over):
    test_gpu_block_norm._check(n, T, d, torch.float16, gate=gate, scale=scale, over=over, ckpt=over, seed=1)


@pytest.mark.parametrize("what", [(), ("state", "packed", "lengths")], ids=["plain", "all"])
@pytest.mark.parametrize("n,T,d", [(1, 530, 4096), (3, 261, 3200), (20, 300, 128), (150, 140, 64), (2, 1033, 136), (1, 13000, 64)])
def test_recurrence(n, T, d, what):
    test_gpu_recurrence._check(n, T, d, torch.float16, what=what, seed=d)
