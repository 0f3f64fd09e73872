"""Rows outside the plain range (nothing but masks, lowest values, logits of 2^97 and more), which a warp
computes again: exact where they are special, sums in chains of V / 128 additions elsewhere, and one of them
does not hold a batch up for twelve times its own time (6.3 measured, read element by element 16)."""
import pytest
import torch

import paper_2609_38823_gb300 as dm
from tests.test_gpu_logprobs import BF16, DEV, F32, I32, _run, _shifted
from tests.test_gpu_logprobs_ranges import _us
from tests.test_gpu_logprobs_sizes import _compare

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [1, 5, 14, 127, 500, 4099, 40003])
def test_rows_outside_the_plain_range(V, dtype):
    """At every alignment: the sums, and special values at any place of the row."""
    scale = 2.0 ** -98
    for off in range(0, 9, 2 if V > 1000 else 1):
        g = torch.Generator().manual_seed(V + off)
        T = 6
        x = (torch.randn(T, V + off, generator=g, dtype=torch.float64) * 2.0 ** 98 + 2.0 ** 100).to(dtype)[:, off:]
        tokens = torch.randint(0, V, (T,), generator=g).to(I32)
        x[1] = -INF
        x[2, ::2] = -INF  # (all of V = 1)
        x[3, V // 2], x[4, V - 1] = NAN, INF
        wide = torch.zeros(T, V + off + 3, dtype=dtype, device=DEV)
        wide[:, off:off + V] = x.to(DEV)
        n = min(V, 3)
        got = _run(wide[:, off:off + V], tokens.to(DEV), n, scale=scale)
        plain = [0, 5] + ([2] if V > 1 and int(tokens[2]) % 2 else [])
        _compare(x[plain], tokens[plain].tolist(), [t[plain] for t in got], n, scale, V / 128)
        assert torch.isneginf(got[0][1]) and got[1][1] == 0 and torch.isneginf(got[3][1]).all() and got[2][1].tolist() == list(range(n))
        assert torch.isnan(got[0][3:5]).all() and torch.isnan(got[1][3:5]).all() and torch.isnan(got[3][3:5]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_equal_logits_but_one(dtype):
    V, scale = 151001, 2.0 ** -98
    for below in (0.4375, 0.8125, 1.25):
        x = (torch.full((2, V), 4.0 - below, dtype=torch.float64) * 2.0 ** 98).to(dtype)
        x[:, V // 3] = 2.0 ** 100
        got = _run(_shifted(x), torch.tensor([7, V // 3], dtype=I32, device=DEV), 3, scale=scale)
        _compare(x, [7, V // 3], got, 3, scale, V / 128)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_empty_row_of_a_batch(dtype):
    T, V, n = 24, 151001, 20
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    us = [_us(x, n)]
    x[3] = -INF
    us.append(_us(x, n))
    assert us[1] <= 12 * us[0], us
