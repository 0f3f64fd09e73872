"""Attention over 4-bit pages where scale times a query is next to nothing or next to the
largest number: results of finite queries stay finite."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
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


@pytest.mark.parametrize("group", [32, 64])
@pytest.mark.parametrize("size", [2.0 ** 117, 2.0 ** 120, 2.0 ** 122])
def test_queries_next_to_the_largest_number(size, group):
    """Finite queries whose factor fp32 cannot hold: the key of the largest score takes all the weight."""
    lens = [37, 200, 1]
    q, pool, table = _case(lens, 8, 2, 128, group, 16, 22)
    q = (q.double() * size).to(torch.bfloat16)
    assert torch.isfinite(q).all()
    out = f64(_attend(q.to(DEV), pool, table, lens))
    assert np.isfinite(out).all()
    q, (kd, vd, span, code) = f64(q), O.q4_values(pool.cpu().numpy(), 128, group)
    seen = 0
    for b, n in enumerate(lens):
        at = (table[b, np.arange(n) // 16], np.arange(n) % 16)
        for h in range(8):
            k, v, vs = (x[at][:, h // 4] for x in (kd, vd, code))
            s = k @ q[b, h]
            best, size_of = int(s.argmax()), ((span[at][:, h // 4] + np.abs(k - span[at][:, h // 4])) @ np.abs(q[b, h])).max()
            # (128 + 32) 2^-23: what a score is off by at most, of the sum of its terms
            if n > 1 and s[best] - np.sort(s)[-2] <= 2 * 160 * 2.0 ** -23 * size_of:
                continue
            tol = 2.0 ** -8 * np.abs(v[best]) + 2.0 ** -11 * vs[best] + n * 2.0 ** -26 * vs.max() + 2.0 ** -20 * np.abs(v[best])
            assert (np.abs(out[b, h] - v[best]) <= tol).all()
            seen += 1
    assert seen >= 20
