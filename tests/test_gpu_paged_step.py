"""A decode step's plan and the lengths after it against the oracle (exact)."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _i32(v):
    return torch.as_tensor(np.asarray(v, np.int64)).to(I32).to(DEV)


def _step(cached, fresh, ps, width, n_free, head=0, seed=0, drop=()):
    """One call and a repeated one; drop: (request, entry) of held pages that are gone."""
    r = np.random.default_rng(seed)
    B = len(cached)
    pages = r.permutation(100_000)
    free, at = pages[:n_free], n_free
    table = np.full((B, width), -7, np.int64)
    for b in range(B):
        have = min(-(-max(cached[b], 0) // ps), width)
        table[b, :have] = pages[at:at + have]
        at += have
    for b, e in drop:
        table[b, e] = -1
    sizes = {"seq_len": B, "slots": B, "positions": B, "head": 1}
    out = {n: torch.full((m + 5,), -99, dtype=I32, device=DEV) for n, m in sizes.items()}
    view = {n: out[n][:m] for n, m in sizes.items()}
    t, status = _i32(table).view(B, width), torch.zeros(1, dtype=I32, device=DEV)
    args = (_i32(cached), _i32(fresh), ps, _i32(free), t, view["seq_len"], view["slots"], view["positions"])
    kw = dict(free_head=_i32([head]), free_head_out=view["head"], status=status)
    dm.decomoe_paged_plan_step(*args, **kw)
    code = dm.decomoe_read_status(status)
    first = {n: v.clone() for n, v in out.items()} | {"table": t.clone()}
    dm.decomoe_paged_plan_step(*args, **kw)
    torch.cuda.synchronize()
    assert all(torch.equal(first[n], v) for n, v in out.items()) and torch.equal(first["table"], t)
    assert all((out[n][m:] == -99).all() for n, m in sizes.items())
    rows = [min(f, 1) for f in fresh]
    ref = O.paged_plan(cached, rows, ps, free, head, table, B)
    at = ref[2][:-1]
    live = np.array([f > 0 for f in rows], bool)
    by = lambda v: np.where(live, np.append(v, -1)[np.minimum(at, B)], -1) if B else v  # noqa: E731
    for n, x in (("table", ref[0]), ("seq_len", ref[1]), ("slots", by(ref[3])), ("positions", by(ref[4]))):
        got = t if n == "table" else view[n]
        assert np.array_equal(got.cpu().numpy(), x), n
    assert int(view["head"][0]) == ref[5]
    assert code == (dm.DECOMOE_OK if ref[6] and max(fresh, default=0) <= 1 else dm.DECOMOE_ERR_BAD_INPUT)
    return ref


@pytest.mark.parametrize("B,ps,hi,live,seed", [(1, 16, 40, 1.0, 0), (1, 16, 40, 0.0, 1), (24, 16, 4000, 0.5, 2),
                                               (7, 1, 30, 0.7, 3), (300, 8, 900, 0.2, 4), (257, 64, 3000, 0.9, 5),
                                               (4096, 16, 100, 0.5, 6), (3, 1024, 5000, 0.6, 7)])
def test_step_plan_parity(B, ps, hi, live, seed):
    r = np.random.default_rng(seed)
    cached, fresh = r.integers(0, hi, B), (r.random(B) < live).astype(int)
    cached[::3] = cached[::3] // ps * ps  # requests whose row begins a page
    ref = _step(list(cached), list(fresh), ps, -(-hi // ps) + 1, B + 9, head=4, seed=seed)
    assert ref[6]


def test_step_plan_edges():
    _step([], [], 16, 4, 3)
    _step([0] * 5, [0] * 5, 16, 4, 3)
    _step([0, 15, 16, 31, 32], [1, 0, 1, 1, 1], 16, 5, 9)
    assert not _step([16, 5, 32, 48], [1, 1, 1, 1], 16, 5, 2)[6]       # the list runs out
    assert not _step([64, 5], [1, 1], 16, 4, 9)[6]                     # a full table row
    assert not _step([-2, 70, 3], [1, 0, -1], 16, 4, 9)[6]             # lengths that cannot be
    _step([3, 9, 17], [2, 0, 5], 16, 4, 9)                             # more than a row: one, and marked
    assert not _step([20, 5], [1, 1], 16, 4, 9, drop=[(0, 1)])[6]      # a row into a page that is gone


def test_step_plan_refusals():
    B = 3
    ok = dict(cached=_i32([1, 2, 3]), fresh=_i32([1, 1, 1]), ps=16, free=_i32([0, 1]), table=_i32([[5, 6]] * B).view(B, 2),
              seq=_i32([0] * B), slots=_i32([0] * B), pos=_i32([0] * B))

    def call(**kw):
        a = ok | kw
        dm.decomoe_paged_plan_step(a["cached"], a["fresh"], a["ps"], a["free"], a["table"], a["seq"], a["slots"], a["pos"])

    call()
    for kw in (dict(slots=_i32([0] * 4)), dict(pos=_i32([0] * 2)), dict(fresh=_i32([1, 1])), dict(seq=_i32([0] * B).long()),
               dict(table=_i32([5, 6, 7])), dict(cached=torch.zeros(B, dtype=I32))):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(ps=12), dict(seq=ok["cached"]), dict(seq=ok["fresh"])):
        with pytest.raises(dm.DecomoeError) as e:
            call(**kw)
        assert e.value.code == dm.DECOMOE_ERR_INVALID_ARG
    torch.cuda.synchronize()


def _advance(cached, seq_len, table, ps):
    c, head, out = _i32(cached), _i32([3]), _i32([7])
    t = _i32(table).view(len(cached), -1)
    dm.decomoe_paged_advance(c, _i32(seq_len), t, ps, free_head=head, free_head_out=out)
    first = c.clone()
    dm.decomoe_paged_advance(c, _i32(seq_len), t, ps)  # the same plan once more: nothing is left to do
    assert torch.equal(c, first) and int(head) == 7
    return c.tolist()


def test_rows_without_a_page_do_not_count():
    table = [[0, -1, -1, -1],    # a decode row without a page
             [1, -1, -1, -1],    # one row in the last page, one without
             [2, 3, -1, -1],     # a prompt of which two pages were given out
             [4, 5, -1, -1],     # a row in a held page
             [6, 7, -1, -1],     # nothing added
             [-1, -1, 8, 9]]     # a full one, whose first pages (a hidden block) were given back
    assert _advance([4, 3, 0, 6, 8, 16], [5, 5, 9, 7, 8, 16], table, 4) == [4, 4, 8, 7, 8, 16]
    assert _advance([0, -2, 3], [9, 4, -1], [[0, 1], [2, -1], [3, 4]], 4) == [8, 4, 0]  # cut at the table's end


@pytest.mark.parametrize("B,ps,width,seed", [(1, 1, 300, 0), (70, 16, 100, 1), (4096, 8, 5, 2), (9, 64, 33, 3), (5, 4, 64, 4)])
def test_advance_parity(B, ps, width, seed):
    r = np.random.default_rng(seed)
    cached = r.integers(0, width * ps + 1, B)
    seq_len = np.minimum(cached + r.integers(0, width * ps, B), width * ps)
    table, ref = r.integers(0, 1000, (B, width)), []
    for b in range(B):
        have, need = -(-int(cached[b]) // ps), -(-int(seq_len[b]) // ps)
        cut = int(r.integers(have, need + 1))  # the list ran out from this page on
        table[b, cut:] = -1
        ref.append(min(int(seq_len[b]), cut * ps) if cut < need else int(seq_len[b]))
    assert _advance(list(cached), list(seq_len), table, ps) == ref


def test_advance_refusals():
    c, n, t = _i32([1, 2]), _i32([2, 2]), _i32([[0], [1]])
    for args in ((c, n[:1], t, 4), (c, n, t[:1], 4), (c, n.long(), t, 4), (c.cpu(), n, t, 4)):
        with pytest.raises(ValueError):
            dm.decomoe_paged_advance(*args)
    for args, kw in (((c, c, t, 4), {}), ((c, n, t, 5), {}), ((t.view(-1), n, t, 4), {}), ((c, n, t, 4), {"free_head": _i32([0])})):
        with pytest.raises(dm.DecomoeError) as e:
            dm.decomoe_paged_advance(*args, **kw)
        assert e.value.code == dm.DECOMOE_ERR_INVALID_ARG
    assert c.tolist() == [1, 2]
