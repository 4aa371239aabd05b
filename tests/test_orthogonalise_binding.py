"""What the binding of the orthogonal update refuses before it asks where the tensors are, without a GPU."""
import pytest
import torch

import paper_2110_04175_gb300 as rs
from paper_2110_04175_gb300 import build as rs_build


@pytest.fixture(scope="module", autouse=True)
def _library():
    rs_build.build()


@pytest.mark.parametrize("bad", [None, 1.0, torch.zeros(2, 3), torch.zeros(1, 1, 2, 3)], ids=["none", "number", "matrix", "four"])
@pytest.mark.parametrize("name", ["update", "out"])
def test_tensors_that_are_none(name, bad):
    given = dict(update=torch.zeros(1, 2, 3), out=torch.zeros(1, 2, 3))
    given[name] = bad
    with pytest.raises(ValueError, match=f"{name}: an fp32 tensor"):
        rs.relay_orthogonalise(given["update"], given["out"], torch.zeros(8, dtype=torch.uint8))


@pytest.mark.gpu
def test_no_output():
    u = torch.zeros(1, 2, 3, device="cuda")
    work = torch.empty(rs.relay_orthogonalise_workspace(1, 2, 3), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError, match="out"):
        rs.relay_orthogonalise(u, None, work)
