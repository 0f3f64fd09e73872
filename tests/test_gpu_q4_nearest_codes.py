"""Codes of a cache in 4 bits where x - low has more digits than fp32: the nearest code all the
same, ties to even. The expected codes come from fractions, which round nothing."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _codes(group, step):
    """The nearest codes, ties to even, of a group of bf16 values."""
    x = [Fraction(float(v)) for v in group]
    return [min(round((v - min(x)) / Fraction(step)), 15) for v in x]  # round(): ties to even


def _groups():
    """(32 values, their step): values half way between two codes but for digits far below."""
    half = [k + 0.5 for k in range(15)]
    for e in (-12, -16, -17, -18, -20, -24, -25, -30, -40, -100, -126, -133):
        for tiny in (2.0 ** e, -2.0 ** e):
            # a least value next to 0: x - low lies right above or below half a step
            yield [tiny] + [15.0] * 2 + half + [1.0] * 14, 1.0
            yield [v * 64 for v in [tiny / 64 if e < -120 else tiny] + [15.0] * 2 + half + [1.0] * 14], 64.0
            # values next to 0 above a least one of half steps
            yield [-4.5, 10.5] + [tiny] * 15 + [0.0] * 15, 1.0
            yield [-9.0, 21.0] + [tiny, 0.0, 3 * tiny, -1.0, 2.0] * 6, 2.0
    # the same among the smallest numbers, where quotients go another way
    for e in (-110, -120):
        for low in (2.0 ** -133, -2.0 ** -133):
            yield [v * 2.0 ** e for v in [low * 2.0 ** -e] + [15.0] * 2 + half + [1.0] * 14], 2.0 ** e


@pytest.mark.parametrize("d,group", SHAPES)
def test_codes_where_x_minus_low_does_not_fit_fp32(d, group):
    rows, want = [], []
    for values, step in _groups():
        assert len(values) == 32
        x = torch.tensor(values, dtype=torch.float64).to(torch.bfloat16)
        assert torch.equal(x.double(), torch.tensor(values, dtype=torch.float64))  # bf16 as they are
        y = x.repeat(d // 32)
        rows.append(y)
        want.append(_codes(y.tolist(), step))
    x, want, n = torch.stack(rows).view(-1, 1, d).to(DEV), np.array(want), len(rows)
    pool = torch.zeros(-(-n // 8), 1, 1, 16 * (d // 2 + 4 * d // group), dtype=torch.uint8, device=DEV)
    dm.decomoe_paged_append_q4(x, x, torch.arange(n, dtype=I32, device=DEV), pool)
    _, _, ks, vs = O.q4_values(pool.cpu().numpy(), d, group)  # step * code
    steps = np.array([s for _, s in _groups()])[:, None]
    for got in (ks, vs):
        got = got.reshape(-1, d)[:n] / steps
        assert np.array_equal(got, want), np.argwhere(got != want)[:10]
