"""Attention over 4-bit pages where scale times a query is next to nothing or next to the
largest number: results of finite queries stay finite."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from tests.helpers import f64
from tests.test_gpu_paged_q4 import DEV, I32, _attend, _case, _ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


@pytest.mark.parametrize("group", [32, 128])
@pytest.mark.parametrize("scale", [2.0 ** -48, 1e-30, 1e-38])
def test_a_scale_next_to_nothing(scale, group):
    """All weights are equal, also those of a query head of zeros, and a last tile that is not full."""
    lens, hide = [37, 64, 5, 90], [(0, 0), (3, 7), (0, 0), (10, 40)]
    q, pool, table = _case(lens, 8, 2, 128, group, 16, 21, hide)
    q[0], q[1, 3], q[2, 7] = 0, 0, 2.0 ** -130
    out = _attend(q.to(DEV), pool, table, lens, hide, scale=scale)
    ref, tol = _ref(q, pool, table, lens, group, hide, scale=scale)
    assert torch.isfinite(out).all()
    assert (np.abs(f64(out) - ref) <= tol).all()
