"""The alternatives where few groups of threads see anything: all logits masked but for a range of
neighbours, as a grammar's digits or one script's tokens leave them."""
import pytest
import torch

import paper_2609_38823_gb300 as dm
from tests.test_gpu_logprobs import BF16, DEV, F32, I32, _compare, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V", [(2, 151001), (24, 40007), (3, 2600), (320, 20003)])
def test_a_range_of_neighbours(T, V, dtype):
    g = torch.Generator().manual_seed(V)
    for mask in (float("-inf"), torch.finfo(dtype).min):
        for n in (1, 20, 32):
            x = torch.randn(T, V, generator=g) * 2.5
            keep, allowed = [], torch.zeros(T, V, dtype=torch.bool)
            for t in range(T):  # ranges of every length, over the borders of slices and at the row's ends
                size = min(V, (1, 7, 31, 33, 100, 513, 600, 1500, 5000)[int(torch.randint(0, 9, (1,), generator=g))])
                at = (0, V - size, min(V - size, V // 8 - size // 2), int(torch.randint(0, V - size + 1, (1,), generator=g)))[t % 4]
                allowed[t, max(at, 0):max(at, 0) + size] = True
                keep.append(max(at, 0) + size // 2)
            x = torch.where(allowed, x, mask).to(dtype)
            some = range(T) if T <= 24 else range(0, T, 31)
            got = [t[list(some)] for t in _run(x.to(DEV), torch.tensor(keep, dtype=I32, device=DEV), n)]
            _compare(x[list(some)], [keep[t] for t in some], got, n)


def _us(x, n):
    """A call's time in a graph of ten, the least of several."""
    T = x.shape[0]
    ids, top, tokens = torch.zeros(T, n, dtype=I32, device=DEV), torch.zeros(T, n, device=DEV), torch.zeros(T, dtype=I32, device=DEV)
    graph = dm.capture_graph(lambda: [dm.decomoe_token_logprobs(x, tokens, top_id=ids, top_logprob=top) for _ in range(10)])
    times = []
    for _ in range(12):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        graph.replay()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 100)
    return min(times)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_range_takes_no_longer_than_scattered_logits(dtype):
    """24 rows of 151001: as many logits left next to each other as were left anywhere."""
    T, V, n = 24, 151001, 20
    x = torch.randn(T, V, generator=torch.Generator().manual_seed(1)).to(dtype).to(DEV)
    scattered = torch.randperm(V, generator=torch.Generator().manual_seed(2))
    for size in (600, 1500, 5000):
        us = []
        for at in (scattered[:size], torch.arange(V // 3, V // 3 + size)):
            m = torch.full((V,), float("-inf"))
            m[at] = 0
            us.append(_us(x + m.to(DEV), n))
        assert us[1] <= 2 * us[0] + 2, (size, us)
