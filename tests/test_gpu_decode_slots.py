"""Slots of a decode step's batch that have no request, or whose request waits:
they add no row, take no page and leave the other requests alone, in eager steps
and in captured ones; a new prompt takes a slot up again. A cache that ran out of pages
goes on when it has some again."""
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from paper_2609_38823_gb300.decode import DecodeStep, PagedCache
from tests.helpers import BF16_MAX_ABS, BF16_REL_L2, assert_close_out, f64
from tests.test_gpu_decode_step import D, D_MODEL, DEV, HKV, HQ, K, L, _model, _prompt

pytestmark = pytest.mark.gpu
PS = 8


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _pages(lens):
    return sum(-(-n // PS) for n in lens)


class _Server:
    """Three requests, and their keys and values kept on the host."""

    def __init__(self, lens, seed=1):
        layers, _ = _model()
        self.cache = PagedCache(L, len(lens), pages=60, page_size=PS, max_pages=24, hkv=HKV, d=D)
        self.held = _prompt(self.cache, lens, seed)
        self.step = DecodeStep(layers, self.cache, len(lens), HQ, K)
        self.g = torch.Generator().manual_seed(seed + 1)
        self.live = [True] * len(lens)

    def check(self, l, s, h_in, h_out):
        torch.cuda.synchronize()
        for b in range(len(self.live)):
            if not self.live[b]:
                continue
            self.held[l][b][0].append(s.k_new[b].cpu())
            self.held[l][b][1].append(s.v_new[b].cpu())
            k, v = (f64(torch.stack(self.held[l][b][i])) for i in (0, 1))
            assert_close_out(f64(s.heads[b]), O.attention(f64(s.q[b:b + 1]), k, v)[0], 2 * BF16_REL_L2, 2 * BF16_MAX_ABS,
                             f"layer {l} request {b} of {len(k)} rows")

    def steps(self, n):
        for _ in range(n):
            h0 = torch.randn(len(self.live), D_MODEL, generator=self.g).to(torch.bfloat16).to(DEV)
            self.step(h0, trace=self.check)
            self.cache.advance()

    def rows(self):
        return [len(self.held[0][b][0]) for b in range(len(self.live))]

    def as_planned(self):
        """Lengths and pages are those of the rows kept on the host, slots the pool's places of them."""
        lens = self.rows()
        assert self.cache.cached.tolist() == lens and int(self.cache.head) == _pages(lens)
        assert dm.decomoe_read_status(self.cache.status) == dm.DECOMOE_OK
        for b, n in enumerate(lens):
            for l in range(L):
                for pool, kept in ((self.cache.k(l), self.held[l][b][0]), (self.cache.v(l), self.held[l][b][1])):
                    rows = pool[self.cache.table[b, :-(-n // PS)].long()].reshape(-1, HKV, D)[:n].cpu()
                    assert n == 0 or torch.equal(rows, torch.stack(kept)), (b, l)


def test_steps_go_on_after_a_release_and_a_new_prompt():
    s = _Server([5, 47, 30])
    s.steps(2)
    s.as_planned()
    s.cache.release(1)
    s.live[1] = False
    for l in range(L):
        s.held[l][1] = [[], []]
    s.steps(10)  # over page ends
    s.as_planned()
    # a prompt in the free slot, beside the others' rows
    n = 19
    slots = torch.empty(n, dtype=torch.int32, device=DEV)
    s.cache.plan(torch.tensor([0, n, 0], dtype=torch.int32, device=DEV), slots)
    for l in range(L):
        k, v = (torch.randn(n, HKV, D, generator=s.g).to(torch.bfloat16) for _ in range(2))
        dm.decomoe_paged_append(k.to(DEV), v.to(DEV), slots, s.cache.k(l), s.cache.v(l), status=s.cache.status)
        s.held[l][1] = [list(k), list(v)]
    s.cache.advance()
    s.live[1] = True
    s.as_planned()
    s.steps(7)
    s.as_planned()
    assert s.rows() == [24, 26, 49]


@pytest.mark.parametrize("idle", [(0,), (1,), (2,), (0, 2), (0, 1, 2)])
def test_requests_that_wait_add_no_row(idle):
    s = _Server([7, 16, 23], seed=4)
    s.steps(1)
    for b in idle:
        s.step.fresh[b] = 0
        s.live[b] = False
    s.steps(9)
    s.as_planned()
    assert all(int(s.step.slots[b]) == -1 and int(s.step.positions[b]) == -1 for b in idle)
    for b in idle:
        s.step.fresh[b] = 1
        s.live[b] = True
    s.steps(2)
    s.as_planned()


def test_captured_steps_with_a_slot_released_and_taken_up_again():
    """The captured step needs no new capture when slots come and go."""
    runs = []
    for graph in (False, True):
        s = _Server([9, 20, 14], seed=6)
        h0 = torch.zeros(3, D_MODEL, dtype=torch.bfloat16, device=DEV)
        out = []
        replay = dm.capture_graph(lambda: out.append(s.step(h0))) if graph else None
        got = []

        def steps(n):
            for _ in range(n):
                h0.copy_(torch.randn(3, D_MODEL, generator=s.g).to(torch.bfloat16))
                if graph:
                    replay.replay()
                else:
                    out.append(s.step(h0))
                got.append(out[-1].clone())
                s.cache.advance()

        steps(2)
        s.cache.release(0)
        steps(9)
        slots = torch.empty(11, dtype=torch.int32, device=DEV)
        s.cache.plan(torch.tensor([11, 0, 0], dtype=torch.int32, device=DEV), slots)
        for l in range(L):
            k = torch.randn(11, HKV, D, generator=s.g).to(torch.bfloat16).to(DEV)
            dm.decomoe_paged_append(k, k, slots, s.cache.k(l), s.cache.v(l), status=s.cache.status)
        s.cache.advance()
        steps(4)
        assert s.cache.cached.tolist() == [15, 35, 29] and int(s.cache.head) == _pages([15, 35, 29])
        assert dm.decomoe_read_status(s.cache.status) == dm.DECOMOE_OK
        runs.append(torch.stack(got))
    assert torch.equal(runs[0], runs[1])


def test_a_cache_that_ran_out_of_pages_goes_on():
    """Rows without a page do not count: their request goes on where its rows end."""
    cache = PagedCache(L, 3, pages=9, page_size=PS, max_pages=6, hkv=HKV, d=D)
    layers, _ = _model()
    held = _prompt(cache, [16, 15, 33], 1)  # 2 + 2 + 5 pages: none is left
    step = DecodeStep(layers, cache, 3, HQ, K)
    g = torch.Generator().manual_seed(2)
    h0 = lambda: torch.randn(3, D_MODEL, generator=g).to(torch.bfloat16).to(DEV)  # noqa: E731
    kept = [16, 15, 33]
    for i in range(4):  # request 0 gets no page, request 1 fills its last one
        step(h0())
        slots = step.slots.tolist()
        assert slots[0] == -1 and slots[2] >= 0 and (slots[1] >= 0) == (i == 0)
        assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_ERR_BAD_INPUT
        for l in range(L):
            for b in range(3):
                if slots[b] >= 0:
                    held[l][b][0].append(cache.k(l).reshape(-1, HKV, D)[slots[b]].cpu())
        kept = [n + (x >= 0) for n, x in zip(kept, slots)]
        cache.advance()
        assert cache.cached.tolist() == kept and int(cache.head) == 9
    assert kept == [16, 16, 37]
    cache.release(2)
    cache.status.zero_()
    for i in range(3):
        step(h0())
        assert all(x >= 0 for x in step.slots.tolist()[:2]) and step.positions.tolist() == [16 + i, 16 + i, -1]
        cache.advance()
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK
    assert cache.cached.tolist() == [19, 19, 0] and int(cache.head) == 6
    for l in range(L):
        for b in (0, 1):
            rows = cache.k(l)[cache.table[b, :2].long()].reshape(-1, HKV, D).cpu()
            assert torch.equal(rows, torch.stack(held[l][b][0]))
    cache.release(0)
    cache.release(1)
    assert int(cache.head) == 0 and sorted(cache.free.tolist()) == list(range(9))
