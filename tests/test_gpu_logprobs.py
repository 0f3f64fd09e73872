"""Log probabilities of given tokens, entropies and alternatives against the oracle.

fp32 throughout. With d = scale (x - max) of the elements: each exponential is off by |d| 2^-23 (d
itself, two roundings) + 2^-22 (the exponential) of itself, the sum over V by at most V 2^-24 / 32 more (a
thread's own sum is V / (256 S) long, and trees of 13 additions follow), so ln Z is off by less than
  z = 2^-22 + ln(V + 1) 2^-23 + (V / 256 + 16) 2^-24
absolutely (the terms weigh with their p, and p |d| adds up to at most ln V), a log probability by z + 3
2^-24 (|lp| + |d|) and the entropy by 2 z + (|lnZ| + sum p |d|) (z + 2^-22). Ids are exact."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _run(x, tokens, n, scale=1.0, status=None, fill=-7.0, stream=None):
    T = x.shape[0]
    lp, ent = (torch.full((T,), fill, device=DEV) for _ in range(2))
    ids, top = torch.full((T, n), -7, dtype=I32, device=DEV), torch.full((T, n), fill, device=DEV)
    dm.decomoe_token_logprobs(x, tokens, None if tokens is None else lp, ent, ids if n else None, top if n else None,
                              scale=scale, status=status, stream=stream)
    return lp, ent, ids, top


def _compare(x, tokens, got, n, scale=1.0):
    lp, ent, ids, top = (f64(t) for t in got)
    V = x.shape[1]
    x64 = f64(x)
    rlp, rent, rids, rtop = O.token_logprobs(x64, tokens, n, scale)
    assert np.array_equal(ids.astype(np.int64), rids)
    z = 2.0 ** -22 + np.log(V + 1) * 2.0 ** -23 + (V / 256 + 16) * 2.0 ** -24
    for t in range(x.shape[0]):
        for g, r in [(lp[t], rlp[t])] + list(zip(top[t], rtop[t])):
            if not np.isfinite(r):
                assert np.array_equal(g, r, equal_nan=True), (t, g, r)
            else:
                m = scale * x64[t].max()
                lnz = -(rtop[t, 0] if n else O.token_logprobs(x64[t:t + 1], [0], 1, scale)[3][0, 0])
                assert abs(g - r) <= z + 3 * 2.0 ** -24 * (2 * abs(r) + abs(lnz)), (t, g, r, m)
        if not np.isfinite(rent[t]):
            assert np.array_equal(ent[t], rent[t], equal_nan=True)
        elif np.isfinite(rlp[t]) or not np.isneginf(x64[t]).all():
            y = scale * (x64[t] - x64[t].max())
            p = np.exp(y)
            lnz, mean = np.log(p.sum()), -(p[p > 0] * y[p > 0]).sum() / p.sum()
            assert abs(ent[t] - rent[t]) <= 2 * z + (lnz + mean) * (z + 2.0 ** -22), (t, ent[t], rent[t])


def _logits(T, V, dtype, seed, std=2.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, V, generator=g) * std).to(dtype), torch.randint(0, V, (T,), generator=g).to(I32)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,n", [(1, 1, 1), (1, 2, 2), (3, 7, 5), (2, 31, 31), (5, 33, 32), (1, 257, 1), (4, 1000, 32),
                                   (1, 2048, 5), (1, 4097, 20), (2, 32001, 5), (7, 32000, 0), (150, 5001, 3), (400, 777, 8),
                                   (1, 151001, 32), (3, 260001, 20), (700, 64, 32)])
def test_parity(T, V, n, dtype):
    x, tokens = _logits(T, V, dtype, T + V)
    got = _run(x.to(DEV), tokens.to(DEV), n)
    _compare(x, tokens.tolist(), got, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V,n", [(770, 4201, 32), (1900, 9001, 5), (400, 9003, 20), (1100, 20011, 0), (330, 40003, 32)])
def test_a_block_per_row(T, V, n, dtype):
    """Rows enough for a block of four or eight warps each; some masked in long stretches, some padding, unaligned."""
    x, tokens = _logits(T, V + 3, dtype, T + V)
    x[::3, 100:V // 2] = float("-inf")
    x[5, 1:] = float("-inf")
    tokens = torch.where(torch.arange(T) % 7 == 6, -1, tokens.clamp(max=V - 1)).to(I32)
    x = x[:, 1:V + 1]
    got = [None if t is None else t[tokens >= 0] for t in _run(_shifted(x), tokens.to(DEV), n)]
    _compare(x[tokens >= 0], tokens[tokens >= 0].tolist(), got, n)


def _shifted(x):
    """On the GPU, as a slice of wider rows."""
    wide = torch.zeros(x.shape[0], x.shape[1] + 3, dtype=x.dtype, device=DEV)
    wide[:, 1:-2] = x.to(DEV)
    return wide[:, 1:-2]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("off", range(9))
def test_rows_at_any_alignment(dtype, off):
    """Rows inside wider ones, at every place of a 16-byte vector."""
    T, V, n = 5, 1003, 6
    g = torch.Generator().manual_seed(off)
    wide = (torch.randn(T, V + 21, generator=g) * 3).to(dtype)
    wide[:, :off], wide[:, off + V:] = 1e30, 1e30  # next to the rows: larger than anything in them
    tokens = torch.randint(0, V, (T,), generator=g).to(I32)
    got = _run(wide.to(DEV)[:, off:off + V], tokens.to(DEV), n)
    _compare(wide[:, off:off + V], tokens.tolist(), got, n)


@pytest.mark.parametrize("n", [1, 5, 32])
@pytest.mark.parametrize("T,V", [(2, 40), (3, 5000), (1, 32001), (200, 3001)])
def test_ties_go_to_the_lowest_index(T, V, n):
    # all equal; two values; few values, the largest anywhere
    g = torch.Generator().manual_seed(V + n)
    for x in (torch.full((T, V), 1.5), torch.randint(0, 2, (T, V), generator=g).float(),
              torch.randint(-3, 4, (T, V), generator=g).float() * 0.5, torch.tensor([0.0, -0.0]).repeat(T, V)[:, :V]):
        for dtype in (BF16, F32):
            tokens = [0] * T
            got = _run(x.to(dtype).to(DEV), torch.zeros(T, dtype=I32, device=DEV), n)
            _compare(x.to(dtype), tokens, got, n)


@pytest.mark.parametrize("S", [1, 300])
def test_largest_elements_in_one_thread(S):
    """The largest elements all where one thread reads them (every 2048th of bf16 and more): more
    are collected than the threads' maxima promise, and where hundreds are, than there is room for."""
    V, n = 200_000, 32
    for pattern in (2048, 1024, 256):
        x = torch.linspace(0, 1, V).repeat(S, 1)
        for v in range(8):
            x[:, v::pattern] += 100
        x = x.to(F32)
        got = _run(x.to(DEV), torch.zeros(S, dtype=I32, device=DEV), n)
        ref = torch.sort(x[0].double(), descending=True, stable=True).indices[:n]
        assert (got[2].cpu() == ref.to(I32)).all()
    # rows in falling order: the first elements, all in the first vectors
    x = torch.linspace(100, 0, V).repeat(S, 1)
    got = _run(x.to(DEV), torch.zeros(S, dtype=I32, device=DEV), n)
    assert (got[2].cpu() == torch.arange(n, dtype=I32)).all()


def test_more_collected_than_there_is_room_for():
    """One warp's threads hold thousands of equal largest values, the other warps' none."""
    V, n = 300 * 2048, 32
    x = torch.zeros(1, V)
    x.view(300, 256, 8)[:, :4] = 5.0  # bf16 vectors of four threads
    for dtype in (BF16, F32):
        for rows in (1, 400):
            got = _run(x.to(dtype).to(DEV).expand(rows, V).contiguous() if rows > 1 else x.to(dtype).to(DEV),
                       torch.zeros(rows, dtype=I32, device=DEV), n)
            assert (got[2].cpu() == torch.arange(n, dtype=I32)).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [50, 8193, 40000])
def test_values_that_are_not_finite(dtype, V):
    inf, nan, low = float("inf"), float("nan"), torch.finfo(dtype).min
    x, _ = _logits(10, V, F32, V)
    x[0] = -inf                                  # nothing left
    x[1, 1:] = -inf                              # one token left
    x[2, V // 3:] = -inf                         # masked, as a grammar masks
    x[3] = low                                   # the type's lowest value everywhere: even
    x[4, V // 2:] = low
    x[5, V // 2], x[6, 3], x[7, V - 1] = nan, inf, nan
    x[8, ::2] = -inf
    x[9] = -inf
    x[9, V - 3:] = torch.tensor([1.0, 2.0, 1.0])
    x = x.to(dtype)
    tokens = torch.tensor([1, 0, V - 1, 2, V - 1, 0, 3, 1, 2, V - 2], dtype=I32)
    n = 5
    got = _run(x.to(DEV), tokens.to(DEV), n)
    _compare(x, tokens.tolist(), got, n)
    assert torch.isneginf(got[0][0]) and got[1][0] == 0 and got[2][0].tolist() == [0, 1, 2, 3, 4]
    assert got[1][1] == 0 and got[0][1] == 0
    assert torch.isnan(got[0][[5, 6, 7]]).all() and torch.isnan(got[3][[5, 6, 7]]).all()


def test_padded_rows_are_left_as_they_were():
    x, tokens = _logits(40, 3001, BF16, 1)
    x[7] = float("nan")
    tokens[[7, 20, 39]] = -1
    tokens[25] = 3001
    status = torch.zeros(1, dtype=I32, device=DEV)
    got = _run(x.to(DEV), tokens.to(DEV), 4, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
    pad = [7, 20, 25, 39]
    assert all((t[pad] == -7).all() for t in got)
    keep = [i for i in range(40) if i not in pad]
    _compare(x[keep], tokens[keep].tolist(), [t[keep] for t in got], 4)
    tokens[25] = -5
    _run(x.to(DEV), tokens.to(DEV), 4, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK


@pytest.mark.parametrize("scale", [0.25, 1.7, 50.0])
def test_scale(scale):
    x, tokens = _logits(6, 5003, F32, 3)
    _compare(x, tokens.tolist(), _run(x.to(DEV), tokens.to(DEV), 7, scale=scale), 7, scale)


def test_outputs_that_are_not_wanted():
    x, tokens = _logits(3, 999, BF16, 5)
    xd, td = x.to(DEV), tokens.to(DEV)
    lp, ent, ids, top = _run(xd, td, 6)
    one = lambda t: torch.full_like(t, -7)  # noqa: E731
    a, b, c, d = one(lp), one(ent), one(ids), one(top)
    dm.decomoe_token_logprobs(xd, td, a)
    dm.decomoe_token_logprobs(xd, None, None, b)
    dm.decomoe_token_logprobs(xd, td, top_id=c)
    dm.decomoe_token_logprobs(xd, None, top_logprob=d)
    assert torch.equal(a, lp) and torch.equal(b, ent) and torch.equal(c, ids) and torch.equal(d, top)


def test_same_bits_streams_and_graphs():
    for T, V in ((1, 32001), (30, 50000), (500, 4001)):
        x, tokens = _logits(T, V, BF16, T)
        xd, td = x.to(DEV), tokens.to(DEV)
        first = _run(xd, td, 5)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            second = _run(xd, td, 5)
        side.synchronize()
        outs = [torch.full_like(t, -7) for t in first]
        graph = dm.capture_graph(lambda: dm.decomoe_token_logprobs(xd, td, *outs))
        for t in outs:
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        for a, b, c in zip(first, second, outs):
            assert torch.equal(a, b) and torch.equal(a, c)
        _compare(x[:3], tokens[:3].tolist(), [t[:3] for t in first], 5)


def test_refusals():
    x, tokens = _logits(3, 99, BF16, 5)
    xd, td = x.to(DEV), tokens.to(DEV)
    f = lambda *s: torch.zeros(*s, device=DEV)  # noqa: E731
    ok = dict(logits=xd, tokens=td, logprob=f(3))
    dm.decomoe_token_logprobs(**ok)
    for kw in (dict(logits=xd.half()), dict(tokens=td.long()), dict(tokens=td[:2]), dict(logprob=f(2)), dict(logprob=f(3).double()),
               dict(entropy=f(6)[::2]), dict(top_id=torch.zeros(3, 4, dtype=I32, device=DEV), top_logprob=f(3, 5)),
               dict(logits=xd[:, ::2]), dict(logits=x), dict(top_logprob=f(12))):
        with pytest.raises((ValueError, TypeError)):
            dm.decomoe_token_logprobs(**(ok | kw))
    for kw in (dict(tokens=None), dict(top_logprob=f(3, 33)), dict(scale=0.0), dict(scale=float("nan")), dict(scale=-1.0),
               dict(logits=xd[:, :3], top_logprob=f(3, 4)), dict(logprob=xd.view(F32).view(-1)[:3] if x.numel() % 2 == 0 else td.view(F32))):
        with pytest.raises(dm.DecomoeError):
            dm.decomoe_token_logprobs(**(ok | kw))
    dm.decomoe_token_logprobs(xd[:0], td[:0], f(0))  # no rows: nothing to do
    torch.cuda.synchronize()
