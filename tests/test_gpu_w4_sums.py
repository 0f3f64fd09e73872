"""Sums of the products with 4-bit weights against 64 bits, bounded by the formula's own
terms |x (q - 8) scale|: rows near the foot of bf16's range, and large values that
meet the code of zero, which add nothing. Sizes of either kernel."""
import pytest
import torch

import paper_2609_38823_gb300 as dm

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
SMALL, LARGE = (300, 1024), (17000, 2048)  # N, K


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _weights(N, K, group, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randint(0, 256, (N, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    return w, (torch.rand(N, K // group, generator=g, device=DEV) * 0.02 - 0.005).to(BF16)


def _check(x, w, ws, xs=None):
    """A product is exact; a group's at most eight matrix products of 16 terms each lose at most 2^-22
    of the magnitudes added so far (fp32, alignment included), 2^-19 of all terms, the sums over groups and warps
    less than that again at these sizes: 2^-18 of the terms. Below fp32's normal numbers
    each of fewer than K roundings loses at most 2^-149. Then the output's own rounding."""
    T, K = x.shape
    N, groups = ws.shape
    out = torch.full((T, N), 5.0, dtype=F32, device=DEV)
    dm.decomoe_w4_linear(x, w, ws, out, x_scale=xs)
    x64 = x.double() * (1.0 if xs is None else xs.double()[:, None])
    for n in range(0, N, 4096):
        b = w[n:n + 4096].int()
        full = (torch.stack([b % 16, b // 16], -1).flatten(1).double() - 8) * ws[n:n + 4096].double().repeat_interleave(K // groups, 1)
        ref, terms = x64 @ full.t(), x64.abs() @ full.abs().t()
        err = (out[:, n:n + 4096].double() - ref).abs()
        bound = 2.0 ** -23 * ref.abs() + 2.0 ** -18 * terms + K * 2.0 ** -149
        assert (err <= bound).all(), (n, float((err / bound).max()))
    return out


@pytest.mark.parametrize("N,K", [SMALL, LARGE])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 8, 11, 24, 30])
def test_small_rows(N, K, group, T):
    w, ws = _weights(N, K, group, T)
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.randn(T, K, generator=g, device=DEV)
    for e in (-95, -110, -122):
        _check((x * 2.0 ** e).to(BF16), w, ws)


@pytest.mark.parametrize("N,K", [SMALL, LARGE])
def test_rows_of_every_size_side_by_side(N, K):
    w, ws = _weights(N, K, 64, 5)
    e = torch.tensor([0, -60, -95, -110, -122, 60, 100, 115], device=DEV)
    x = torch.randn(8, K, device=DEV) * 2.0 ** e.double()[:, None]
    _check(x.to(BF16), w, ws)
    # and group by group
    f = 2.0 ** e[(torch.arange(K, device=DEV) // 64) % 8].double()
    _check((torch.randn(3, K, device=DEV) * f).to(BF16), w, ws)


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("N,K", [SMALL, LARGE])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T", [1, 12, 20, 32])
def test_large_values_on_the_code_of_zero(kind, N, K, group, T):
    w, ws = _weights(N, K, group, T)
    g = torch.Generator(device=DEV).manual_seed(T + 1)
    x = torch.randn(T, K, generator=g, device=DEV)
    # one value of a group 2^14 times its neighbours (e4m3: 448 beside values of 1/64), its weights all zero
    at = torch.arange(0, K, group, device=DEV) + torch.randint(0, group, (K // group,), generator=g, device=DEV)
    x = x / 64 if kind == E4M3 else x
    x[:, at] = 448.0 if kind == E4M3 else 2.0 ** 14
    low, byte = at % 2 == 0, at // 2
    w[:, byte] = torch.where(low, (w[:, byte] & 0xF0) | 8, (w[:, byte] & 0x0F) | 0x80)
    xs = torch.rand(T, generator=g, device=DEV) + 0.5 if kind == E4M3 else None
    out = _check(x.to(kind), w, ws, xs)
    # without them: not a bit changes
    x[:, at] = 0
    again = torch.empty_like(out)
    dm.decomoe_w4_linear(x.to(kind), w, ws, again, x_scale=xs)
    assert torch.equal(out, again)


@pytest.mark.parametrize("kind", [BF16, E4M3])
@pytest.mark.parametrize("N,K", [SMALL, LARGE])
def test_values_that_are_not_finite(kind, N, K):
    """NaN in a row makes all of it NaN; an infinity (bf16) gives the infinity of its weight's
    sign, NaN on a weight of zero; the other rows keep their bits."""
    w, ws = _weights(N, K, 64, 3)
    ws = ws.abs() + 2.0 ** -10
    x = torch.randn(11, K, device=DEV).to(kind)
    xs = torch.ones(11, device=DEV) if kind == E4M3 else None
    out = [torch.empty(11, N, dtype=F32, device=DEV) for _ in range(2)]
    dm.decomoe_w4_linear(x, w, ws, out[0], x_scale=xs)
    x[2, 70] = float("nan")
    if kind == BF16:
        x[9, 130], x[4, 131] = float("inf"), -float("inf")
    dm.decomoe_w4_linear(x, w, ws, out[1], x_scale=xs)
    assert torch.isnan(out[1][2]).all()
    keep = [0, 1, 3, 5, 6, 7, 8, 10]
    assert torch.equal(out[0][keep], out[1][keep])
    if kind == BF16:
        for t, q, sign in ((9, (w[:, 65] & 15).int() - 8, 1.0), (4, (w[:, 65] >> 4).int() - 8, -1.0)):
            ref = torch.where(q == 0, float("nan"), sign * torch.sign(q.float()) * float("inf"))
            assert torch.equal(torch.nan_to_num(out[1][t], nan=0.5, posinf=2.0, neginf=-2.0),
                               torch.nan_to_num(ref, nan=0.5, posinf=2.0, neginf=-2.0))
    else:
        assert torch.equal(out[0][[4, 9]], out[1][[4, 9]])
