"""Log probabilities where scale or logits lie near the ends of fp32, and where many terms of
a sum round the same way.

A row's sums (z of the exponentials e = 2^d, w of e d) are added up by threads, each with two partial sums, in
chains of at most L additions, and trees of 15 additions or fewer follow. An addition is off by at most
2^-24 of what has been added up so far, so the sum by (L + 16) 2^-24 of itself at most. d = c (x - m) is off
by four roundings at most, |d| 2^-22, an exponential by 2^-22 of itself, and where the largest logit comes last a
sum is multiplied with another one. L = V / 32 for a warp that has one sum a thread (rows whose size lies outside
the plain range), V / 64 for a warp of a short row, V / 256 for a block of four warps, at most that for more. So ln z
is off by z = (L + 16) 2^-24 + 2^-21 + mean |d| 2^-21, the mean being under p, and by its own rounding; a log
probability by that and three roundings of numbers as large as |lp| + |ln z|
"""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from tests.helpers import f64
from tests.test_gpu_logprobs import BF16, DEV, F32, I32, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _compare(x, tokens, got, n, scale, L):
    """Against the oracle within the bounds above, the scale being the fp32 number that the call gets."""
    lp, ent, ids, top = (f64(t) for t in got)
    scale = float(np.float32(scale))
    x64 = f64(x)
    rlp, rent, rids, rtop = O.token_logprobs(x64, tokens, n, scale)
    assert np.array_equal(ids.astype(np.int64), rids)
    for t in range(x.shape[0]):
        y = scale * (x64[t] - x64[t].max())
        p = np.exp(y)
        lnz, mean = np.log(p.sum()), -(p[p > 0] * y[p > 0]).sum() / p.sum()
        z = (L + 16) * 2.0 ** -24 + 2.0 ** -21 + 1.45 * mean * 2.0 ** -21 + 2.0 ** -24 * lnz
        for g, r in [(lp[t], rlp[t])] + list(zip(top[t], rtop[t])):
            if abs(r) > 3.4e38:
                assert g == -np.inf
            else:
                assert abs(g - r) <= z + 3 * 2.0 ** -24 * (abs(r) + lnz), (t, g, r)
        # the entropy is ln z - sum e y / z: the second sum as the first, and each of its terms
        assert abs(ent[t] - rent[t]) <= 2 * z + (lnz + 2 * mean) * (z + 2.0 ** -21), (t, ent[t], rent[t])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [3.4e38, 3e38, 2.4e38, 1e38, 2.0 ** 100])
def test_scales_up_to_the_largest(scale, dtype):
    """Logits that differ by little enough to share the probability, and by more: one token takes all."""
    g = torch.Generator().manual_seed(1)
    T, V, n = 4, 700, 5
    x = torch.randn(T, V, generator=g)
    x[1] = x[1] / scale / 4  # (2^-130 or so: numbers with few digits)
    x[2] = 2.5
    x[3, ::2] = float("-inf")
    x = x.to(dtype)
    tokens = torch.tensor([int(x[0].argmax()), 5, 9, 1], dtype=I32)
    got = _run(x.to(DEV), tokens.to(DEV), n, scale=scale)
    assert not any(torch.isnan(t).any() for t in got)
    _compare(x, tokens.tolist(), got, n, scale, V / 32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [2.0 ** -126, 5e-39, 2.0 ** -127, 1e-39])
def test_scales_down_to_subnormal_ones(scale, dtype):
    """Logits over all of the type's range, from the lowest value to the largest."""
    T, V, n = 3, 900, 6
    top = torch.finfo(dtype).max
    x = torch.linspace(-1, 1, V, dtype=torch.float64).repeat(T, 1)
    x = (x[:, torch.randperm(V, generator=torch.Generator().manual_seed(2))] * top).clamp(-top, top)
    x[1] *= 2.0 ** -7
    x[2, ::3] = float("-inf")
    x = x.to(dtype)
    tokens = torch.tensor([1, V - 1, 4], dtype=I32)
    got = _run(x.to(DEV), tokens.to(DEV), n, scale=scale)
    assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all()
    _compare(x, tokens.tolist(), got, n, scale, V / 32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,L", [(2, 40000, 40000 / 256), (2, 500, 500 / 64), (400, 2047, 2047 / 64), (400, 9001, 9001 / 256),
                                   (1, 151001, 151001 / 256)])
def test_rows_of_equal_logits_but_one(T, V, L, dtype):
    """All exponentials but one are the same number, so that their additions round the same way for long."""
    for below in (0.4375, 0.8125, 1.25, 4.0):
        x = torch.full((T, V), 3.0 - below).to(dtype)
        x[:, V // 3] = 3.0
        tokens = torch.full((T,), 7, dtype=I32)
        got = [t[:2] for t in _run(x.to(DEV), tokens.to(DEV), 3)]
        _compare(x[:2], tokens[:2].tolist(), got, 3, 1.0, L)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_outside_the_plain_range_of_equal_logits_but_one(dtype):
    """The same with logits of 2^100 and a scale that brings their differences back."""
    V, scale = 40000, 2.0 ** -98
    for below in (0.4375, 0.8125, 1.25):
        x = (torch.full((2, V), 4.0 - below, dtype=torch.float64) * 2.0 ** 98).to(dtype)
        x[:, V // 3] = 2.0 ** 100
        got = _run(x.to(DEV), torch.tensor([7, V // 3], dtype=I32, device=DEV), 3, scale=scale)
        _compare(x, [7, V // 3], got, 3, scale, V / 32)
