"""What the step between blocks writes of its 8-bit output past a row's features: code 0 and scale 7, also where the row is not
finite, whichever of its kernels takes the rows."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    rs_build.build()


# few rows, and 2^24 elements and more, which go through shared memory in 16 bits: warps with all their features and
# without, whole blocks of 32 past d (d mod 128 up to 96) and none
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,T,d", [(2, 9, 1032), (2, 8200, 1032), (2, 4400, 1928), (2, 4300, 2016), (2, 4090, 2088), (2, 1150, 7400),
                                   (3, 700, 8072)])
def test_features_past_the_row(dtype, n, T, d):
    g = torch.Generator(device="cuda").manual_seed(d)
    x, r, z = (torch.randn(n, T, d, device="cuda", generator=g).to(dtype) for _ in range(3))
    x[0, 1, 5] = float("nan")
    x[1, 3, d - 1] = float("inf")
    r[0, 5, 40] = float("-inf")
    z[1, 7, d // 2] = float("nan")
    odd = [(0, 1), (1, 3), (0, 5), (1, 7)]  # every feature of such a row is NaN, or all but where h is infinite, through s_h
    w = 1 + 0.1 * torch.randn(n, d, device="cuda", generator=g)
    kept, y, total = rs.ActivationCheckpoint(n, T, d), torch.empty_like(x), torch.empty_like(x)
    kept.codes.fill_(99)
    kept.scales.fill_(99)
    rs.relay_block_norm(x, r, w, w, total, y, 1e-5, gate=z, checkpoint=kept)
    past = -(-d // 32)  # the first block without a feature
    assert (kept.codes[..., d:] == 0).all()
    assert (kept.scales[..., past:] == 7).all()
    here = torch.zeros(n, T, dtype=torch.bool, device="cuda")
    for i, t in odd[:2] + odd[3:]:
        here[i, t] = True
        assert (kept.scales[i, t, :past] == 255).all() and (kept.codes[i, t] == 0).all()
    here[0, 5] = True  # h is infinite at one place, where h s_h is NaN, and 0 elsewhere
    assert kept.scales[0, 5, 40 // 32] == 255 and (kept.codes[0, 5] == 0).all()
    assert (kept.scales[..., :past][~here] < 255).all()
