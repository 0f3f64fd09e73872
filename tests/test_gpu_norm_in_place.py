"""Outputs of the norm over its own inputs, element for element, in every pairing that
the call takes."""
import pytest
import torch

import paper_2609_38823_gb300 as dm

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(9, 64), (400, 2048), (5, 40000)])
@pytest.mark.parametrize("sum_on,y_on", [("x", "res"), ("res", "x"), (None, "res"), ("x", None), ("res", None)])
def test_outputs_over_inputs(dtype, T, d, sum_on, y_on):
    x, res = (torch.randn(T, d, device=DEV).to(dtype) for _ in range(2))
    w = torch.rand(d, device=DEV).to(dtype) + 0.5
    s, y = torch.empty_like(x), torch.empty_like(x)
    dm.decomoe_add_rmsnorm_q8(x, res, w, s, y)
    at = {"x": x.clone(), "res": res.clone(), None: torch.empty_like(x)}
    s2, y2 = at[sum_on], at[y_on] if y_on else torch.empty_like(x)
    dm.decomoe_add_rmsnorm_q8(at["x"], at["res"], w, s2, y2)
    assert torch.equal(s2, s) and torch.equal(y2, y)
