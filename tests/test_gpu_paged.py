"""The paged key-value cache against the oracle: block tables, slots and
positions (exact), the store of new rows (exact), and the attention of one
token per request over its pages.

Attention outputs are bf16 with fp32 scores, softmax and sums and weights
rounded to bf16, as decomoe_attention: the bf16 output tolerance."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from tests.helpers import BF16_MAX_ABS, BF16_REL_L2, assert_close_out, f64

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


# ------------------------------------------------------------------ plan

def _plan(cached, fresh, ps, width, n_free, head=0, N=None, seed=0, null_head=False):
    r = np.random.default_rng(seed)
    B = len(cached)
    N = int(sum(max(f, 0) for f in fresh)) + 3 if N is None else N
    pages = r.permutation(100_000)
    free = pages[:n_free]
    table = np.full((B, width), -7, np.int64)  # unused entries: anything
    at = n_free
    for b in range(B):
        have = min(-(-max(cached[b], 0) // ps), width)
        table[b, :have] = pages[at:at + have]
        at += have
    t = _i32(table)
    guard = 5
    out = {n: torch.full((m + guard,), -99, dtype=I32, device=DEV)
           for n, m in (("seq_len", B), ("row_start", B + 1), ("slots", N), ("positions", N), ("head", 1))}
    sizes = {"seq_len": B, "row_start": B + 1, "slots": N, "positions": N, "head": 1}
    view = {n: out[n][:sizes[n]] for n in out}
    status = torch.zeros(1, dtype=I32, device=DEV)
    args = (_i32(cached), _i32(fresh), ps, _i32(free), t, view["seq_len"], view["row_start"], view["slots"],
            view["positions"])
    kw = dict(free_head=None if null_head else _i32([head]), free_head_out=view["head"], status=status)
    dm.decomoe_paged_plan(*args, **kw)
    first = {n: v.clone() for n, v in out.items()} | {"table": t.clone()}
    code = dm.decomoe_read_status(status)
    dm.decomoe_paged_plan(*args, **kw)  # a repeated call writes the same values
    torch.cuda.synchronize()
    assert all(torch.equal(first[n], v) for n, v in out.items()) and torch.equal(first["table"], t)
    assert all((out[n][sizes[n]:] == -99).all() for n in out)
    ref = O.paged_plan(cached, fresh, ps, free, head, table, N)
    for n, x in zip(("table", "seq_len", "row_start", "slots", "positions"), ref):
        got = t if n == "table" else view[n]
        assert np.array_equal(got.cpu().numpy(), x), n
    assert int(view["head"][0]) == ref[5]
    assert code == (dm.DECOMOE_OK if ref[6] else dm.DECOMOE_ERR_BAD_INPUT)
    return ref


@pytest.mark.parametrize("B,ps,hi,fresh_hi,seed", [(1, 16, 1, 2, 0), (1, 16, 40, 2, 1), (24, 16, 4000, 2, 2),
                                                   (7, 1, 30, 5, 3), (300, 8, 900, 40, 4), (257, 64, 3000, 2, 5),
                                                   (4096, 128, 2000, 3, 6), (3, 1024, 5000, 4000, 7)])
def test_plan_parity(B, ps, hi, fresh_hi, seed):
    r = np.random.default_rng(seed)
    cached, fresh = r.integers(0, hi, B), r.integers(0, fresh_hi, B)
    width = -(-int((cached + fresh).max()) // ps) + 1
    ref = _plan(cached, fresh, ps, width, 100 + int((-(-fresh // ps) + 1).sum()), head=seed * 3, seed=seed)
    assert ref[6]


def test_plan_from_nothing_and_for_whole_prompts():
    # every table built from the lengths alone: prompts of ragged sizes, no page held
    _plan([0] * 9, [1, 0, 16, 17, 1552, 33, 0, 64, 5], 16, 100, 200, null_head=True)
    # no request, no row, no page
    _plan([], [], 16, 4, 0, N=0)
    _plan([], [], 16, 4, 0, N=6)
    # requests at a page's last row, and just past it
    _plan([15, 16, 17, 31, 32], [1, 1, 1, 1, 1], 16, 5, 9)


def test_plan_marks_what_it_cannot_give():
    assert not _plan([10, 20, 30], [10, 20, 30], 8, 20, 4)[6]         # the list runs out inside a request
    assert not _plan([10, 20], [1, 90], 8, 8, 30)[6]                  # a table row too narrow for its request
    assert not _plan([100, 20], [1, 1], 8, 8, 30)[6]                  # ... and for what it holds
    assert not _plan([-3, 5], [4, -2], 8, 8, 30)[6]                   # negative lengths count as 0
    assert not _plan([3, 5], [4, 9], 8, 8, 30, N=7)[6]                # more rows than the slot map holds
    assert not _plan([3, 5], [4, 9], 8, 8, 5, head=5)[6]              # the list is used up
    assert _plan([3, 5], [4, 3], 8, 8, 0, head=0)[6]                  # ... which is fine if no page is wanted


# ------------------------------------------------------------------ append

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,hkv,d,ps,interleaved", [(1, 4, 128, 16, False), (23, 4, 128, 16, True), (300, 1, 8, 4, False),
                                                    (4097, 2, 64, 64, True), (5, 3, 40, 1, False)])
def test_append_parity(dtype, N, hkv, d, ps, interleaved):
    g = torch.Generator().manual_seed(N)
    P = -(-2 * N // ps) + 1
    both = torch.randn(P, 2, ps, hkv, d, generator=g).to(dtype).to(DEV)
    kp, vp = (both[:, 0], both[:, 1]) if interleaved else (both[:, 0].contiguous(), both[:, 1].contiguous())
    qkv = torch.randn(N, 4 * hkv, d, generator=g).to(dtype).to(DEV)
    k, v = qkv[:, hkv:2 * hkv], qkv[:, 3 * hkv:]
    slots = torch.randperm(P * ps, generator=g)[:N].to(I32)
    if N > 3:
        slots[N // 2] = -1
    ref = [p.clone().reshape(-1, hkv, d) for p in (kp, vp)]
    for r, s in enumerate(slots.tolist()):
        if s >= 0:
            ref[0][s], ref[1][s] = k[r], v[r]
    status = torch.zeros(1, dtype=I32, device=DEV)
    dm.decomoe_paged_append(k, v, slots.to(DEV), kp, vp, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    for p, x in zip((kp, vp), ref):
        assert torch.equal(p.reshape(-1, hkv, d), x)


def test_append_skips_slots_outside_the_pool():
    k = torch.ones(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    kp, vp = (torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    status = torch.zeros(1, dtype=I32, device=DEV)
    dm.decomoe_paged_append(k, k, _i32([11, 12, -5, -1]), kp, vp, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
    for p in (kp, vp):
        assert int(p.float().sum()) == 2 * 64 and (p.view(12, 2, 64)[11] == 1).all()


# ------------------------------------------------------------------ attention

def _case(lens, hq, hkv, d, ps, seed=0, hide=None, width_extra=1, interleaved=False, spare=3, poison=None):
    """Pools whose unused rows hold `poison` (finite noise if None)."""
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    used = [-(-n // ps) for n in lens]
    P, width = sum(used) + spare, max(used + [0]) + width_extra
    pages = torch.randperm(P, generator=g)
    both = torch.randn(P, 2, ps, hkv, d, generator=g).to(torch.bfloat16)
    table = torch.full((B, width), -1, dtype=I32)
    live = torch.zeros(P, ps, dtype=torch.bool)
    at = 0
    for b, n in enumerate(lens):
        h0, h1 = (0, 0) if hide is None else (hide[b][0], hide[b][0] + hide[b][1])
        for i in range(used[b]):
            p = int(pages[at + i])
            rows = [j for j in range(i * ps, min(n, (i + 1) * ps)) if not h0 <= j < h1]
            for j in rows:
                live[p, j - i * ps] = True
            if rows:
                table[b, i] = p  # pages that are hidden altogether have been given back
        at += used[b]
    if poison is not None:
        both[~live[:, None].expand(P, 2, ps)] = poison
    kp, vp = both[:, 0], both[:, 1]
    if interleaved:
        both = both.to(DEV)
        dk, dv = both[:, 0], both[:, 1]
    else:
        dk, dv = kp.contiguous().to(DEV), vp.contiguous().to(DEV)
    q = torch.randn(B, hq + 2 * hkv, d, generator=g).to(torch.bfloat16)
    return q[:, :hq], kp, vp, dk, dv, table, q.to(DEV)[:, :hq]


def _attend(dq, dk, dv, table, lens, hide=None, scale=0.0, status=None, stream=None):
    B, hq, d = dq.shape
    ws = dm.workspace(dm.decomoe_paged_attention_workspace_bytes(B, hq, dk.shape[2], d), DEV)
    ws.fill_(0xAB)
    out = torch.full((B, hq, d), 9.0, dtype=torch.bfloat16, device=DEV)
    h = [None, None] if hide is None else [_i32([x[i] for x in hide]) for i in (0, 1)]
    dm.decomoe_paged_attention(dq, dk, dv, table.to(DEV), _i32(lens), out, ws, hide_begin=h[0], hide_count=h[1],
                               scale=scale, status=status, stream=stream)
    torch.cuda.synchronize()
    return out


def _ref(q, kp, vp, table, lens, hide=None, scale=None):
    h = [None, None] if hide is None else [[x[i] for x in hide] for i in (0, 1)]
    return O.paged_attention(f64(q), kp.double().numpy(), vp.double().numpy(), table.numpy(), lens, h[0], h[1], scale)


def _check(lens, hq, hkv, d, ps, seed=0, hide=None, **kw):
    q, kp, vp, dk, dv, table, dq = _case(lens, hq, hkv, d, ps, seed, hide, **kw)
    status = torch.zeros(1, dtype=I32, device=DEV)
    out = _attend(dq, dk, dv, table, lens, hide, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    ref = _ref(q, kp, vp, table, lens, hide)
    assert_close_out(f64(out), ref, BF16_REL_L2, BF16_MAX_ABS, f"lens {lens[:6]} heads {hq}/{hkv} D {d} page {ps}")
    # requests are also compared one by one: a short one must not hide behind a long one
    for b in range(len(lens)):
        assert_close_out(f64(out[b]), ref[b], 2 * BF16_REL_L2, 2 * BF16_MAX_ABS, f"request {b} of {lens[b]} rows")
    assert torch.equal(out, _attend(dq, dk, dv, table, lens, hide))
    return out, ref


@pytest.mark.parametrize("n", [1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 2049, 5000])
@pytest.mark.parametrize("d,ps", [(128, 16), (64, 32)])
def test_attention_one_request(n, d, ps):
    _check([n], 32, 4, d, ps, seed=n)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 4), (8, 1), (9, 1), (16, 2), (17, 1), (24, 4), (25, 5), (33, 1), (64, 2),
                                    (6, 3), (48, 16)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_head_layouts(hq, hkv, d):
    _check([3, 200, 0, 77, 513], hq, hkv, d, 16, seed=hq)


@pytest.mark.parametrize("ps", [1, 2, 4, 8, 16, 32, 64, 128, 1024])
def test_attention_page_sizes(ps):
    # pages smaller than, equal to and larger than any tile, ends inside one
    _check([1, 50, 129, 300, 47], 16, 2, 128, ps, seed=ps, interleaved=ps % 4 == 0)
    _check([1, 50, 129, 300, 47], 4, 4, 64, ps, seed=ps)


def test_attention_ragged_batches():
    r = np.random.default_rng(5)
    _check([int(x) for x in np.exp(r.uniform(0, np.log(3000), 40))], 32, 4, 128, 64, seed=1)
    _check([0] * 5 + [int(x) for x in r.integers(0, 40, 300)], 2, 2, 64, 16, seed=2)
    _check([20000, 1, 1, 1, 0, 3], 8, 1, 128, 32, seed=3)
    _check([1] * 700, 8, 8, 64, 8, seed=4)


def test_attention_most_requests():
    # as many requests as a call takes: some long, many short, every fifth empty
    r = np.random.default_rng(8)
    lens = [0 if b % 5 == 0 else int(r.integers(1, 30)) for b in range(4096)]
    lens[77], lens[4000] = 3000, 900
    _check(lens, 2, 1, 64, 16, seed=9)


def test_attention_empty_requests():
    for lens in ([0], [0, 0, 0], [0, 5, 0], [0] * 200):
        out, _ = _check(lens, 8, 2, 128, 16, seed=1)
        assert all((out[b] == 0).all() for b, n in enumerate(lens) if n == 0)
    # a table of no columns, a pool of no pages
    q = torch.randn(2, 8, 64, device=DEV).to(torch.bfloat16)
    none = torch.empty(0, 16, 2, 64, dtype=torch.bfloat16, device=DEV)
    assert (_attend(q, none, none, torch.empty(2, 0, dtype=I32), [0, 0]) == 0).all()


@pytest.mark.parametrize("d,ps", [(128, 16), (64, 64), (128, 8)])
def test_attention_hidden_blocks(d, ps):
    lens = [400, 400, 90, 33, 1, 700, 64, 64, 0]
    # inside pages, whole pages, to the end, from the start, everything, nothing
    hide = [(16, 320), (13, 200), (50, 40), (0, 17), (0, 1), (100, 0), (0, 64), (60, 4), (0, 3)]
    out, _ = _check(lens, 16, 4, d, ps, seed=ps, hide=hide, poison=float("nan"))
    assert (out[4] == 0).all() and (out[6] == 0).all()
    # the same rows as compacted caches
    for b in (0, 5):
        q, kp, vp, _, _, table, _ = _case(lens, 16, 4, d, ps, ps, hide, poison=float("nan"))
        rows = [j for j in range(lens[b]) if not hide[b][0] <= j < hide[b][0] + hide[b][1]]
        k = torch.stack([kp[table[b, j // ps], j % ps] for j in rows])
        v = torch.stack([vp[table[b, j // ps], j % ps] for j in rows])
        assert_close_out(f64(out[b]), O.attention(f64(q[b:b + 1]), f64(k), f64(v))[0], BF16_REL_L2, BF16_MAX_ABS)


def test_attention_hidden_blocks_past_the_ends_are_cut():
    lens, hide = [50, 50, 50, 50], [(-5, 10), (40, 100), (60, 10), (10, -4)]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 64, 16, 1)
    same = [(0, 10), (40, 10), (0, 0), (0, 0)]  # a negative begin is 0, a negative count none
    assert torch.equal(_attend(dq, dk, dv, table, lens, hide), _attend(dq, dk, dv, table, lens, same))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_attention_rows_past_the_length_do_not_reach_a_result(value):
    _check([1, 33, 100, 15, 0, 250], 16, 2, 128, 16, poison=value, seed=3)
    _check([1, 33, 100, 15, 0, 250], 4, 4, 64, 64, poison=value, seed=4)


def test_attention_values_that_are_not_finite_stay_in_their_request():
    lens = [40, 40, 40]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 64, 16, 2)
    clean = _attend(dq, dk, dv, table, lens)
    dv[table[1, 0], 3, 1, 5] = float("inf")   # one value of KV head 1: its feature 5 only
    dk[table[2, 1], 2, 0, 0] = float("nan")   # a key of KV head 0: all of its query heads
    out = _attend(dq, dk, dv, table, lens)
    assert torch.equal(out[0], clean[0])
    assert torch.equal(out[1, :4], clean[1, :4]) and torch.isinf(out[1, 4:, 5]).all()
    assert torch.isfinite(out[1, 4:, 6:]).all()
    assert torch.isnan(out[2, :4]).all() and torch.equal(out[2, 4:], clean[2, 4:])


@pytest.mark.parametrize("big", [3e4, -3e4])
def test_attention_large_scores(big):
    # scores around +-1e10: the softmax is decided by differences, and a row whose
    # scores are all far below zero still has its largest one
    lens = [1, 60, 300]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 64, 16, 6)
    dk.fill_(big)
    dq = torch.full_like(dq, abs(big))
    k = torch.full_like(kp, big)
    out = _attend(dq, dk, dv, table, lens)
    ref = _ref(dq.cpu(), k, vp, table, lens)
    assert_close_out(f64(out), ref, BF16_REL_L2, BF16_MAX_ABS, "large scores")


def test_attention_bad_tables_and_lengths_are_marked():
    lens = [100, 40]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 128, 16, 4)
    status = torch.zeros(1, dtype=I32, device=DEV)
    for page in (-1, kp.shape[0], 2 ** 31 - 1):
        bad = table.clone()
        bad[0, 2] = page  # rows 32..47 count as hidden
        out = _attend(dq, dk, dv, bad, lens, status=status)
        assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
        ref = _ref(q, kp, vp, table, lens, [(32, 16), (0, 0)])
        assert_close_out(f64(out), ref, BF16_REL_L2, BF16_MAX_ABS, f"page {page}")
    bad = table.clone()
    bad[1] = -1  # a request without any page: nothing to see
    out = _attend(dq, dk, dv, bad, lens, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT and (out[1] == 0).all()
    # a negative length is 0, one beyond the table ends with it
    wide = table[:, :7]
    out = _attend(dq, dk, dv, wide.contiguous(), [112 + 500, -3], status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
    assert (out[1] == 0).all()
    assert_close_out(f64(out[0]), _ref(q, kp, vp, table, [112, 0])[0], BF16_REL_L2, BF16_MAX_ABS)


def test_attention_pool_beyond_32_bit_offsets():
    # 9000 pages of 64 rows of 8 x 128: 8.8 GiB a pool, page offsets past 2^32 elements
    P, ps, hkv, d = 70000, 64, 8, 128
    k, v = (torch.empty(P, ps, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pages = [P - 1, P - 7, 66000, 33000, 3]
    g = torch.Generator(device=DEV).manual_seed(3)
    lens = [200, 64, 40]
    table = torch.tensor([[pages[0], pages[1], pages[2], pages[3]], [pages[4], -1, -1, -1], [pages[1], -1, -1, -1]],
                         dtype=I32)
    for p in pages:
        for t in (k, v):
            t[p] = torch.randn(ps, hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(3, 16, d, generator=g, device=DEV).to(torch.bfloat16)
    # a new row through the append, at the far end of the pool
    new = torch.randn(1, hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    dm.decomoe_paged_append(new, new, _i32([33000 * ps + 7]), k, v)
    dm.decomoe_paged_append(new, new, _i32([(P - 1) * ps + 63]), k, v)
    out = _attend(q, k, v, table, lens)
    small = {p: i for i, p in enumerate(pages)}
    ks, vs = (torch.stack([t[p] for p in pages]).cpu() for t in (k, v))
    assert torch.equal(ks[0, 63], new[0].cpu()) and torch.equal(vs[3, 7], new[0].cpu())
    tab = torch.tensor([[small.get(int(p), -1) for p in row] for row in table], dtype=I32)
    assert_close_out(f64(out), _ref(q.cpu(), ks, vs, tab, lens), BF16_REL_L2, BF16_MAX_ABS, "far pages")


def test_attention_scale_and_stream():
    lens = [70, 300]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 128, 16, 9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = _attend(dq, dk, dv, table, lens, scale=0.3)
    assert_close_out(f64(out), _ref(q, kp, vp, table, lens, scale=0.3), BF16_REL_L2, BF16_MAX_ABS, "scale")
    torch.cuda.synchronize()
    assert torch.equal(_attend(dq, dk, dv, table, lens, scale=0.3, stream=side), out)


def test_steps_in_a_captured_graph():
    """Plan, append and attention of one step captured once and replayed while
    the requests grow over page ends, against caches kept on the host."""
    hq, hkv, d, ps, B, steps = 8, 2, 64, 8, 3, 20
    g = torch.Generator().manual_seed(1)
    cached = torch.tensor([0, 7, 30], dtype=I32, device=DEV)
    fresh = torch.ones(B, dtype=I32, device=DEV)
    width, P = 8, 40
    free = torch.randperm(P, generator=g).to(I32).to(DEV)
    table = torch.full((B, width), -1, dtype=I32, device=DEV)
    new = lambda n: torch.empty(n, dtype=I32, device=DEV)  # noqa: E731
    head, head_out, seq_len, row_start, slots = torch.zeros(1, dtype=I32, device=DEV), new(1), new(B), new(B + 1), new(40)
    kp, vp = (torch.zeros(P, ps, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    status = torch.zeros(1, dtype=I32, device=DEV)
    # the rows that the requests hold at the start, planned and stored as prompts
    rows = torch.randn(37, 2, hkv, d, generator=g).to(torch.bfloat16).to(DEV)
    dm.decomoe_paged_plan(torch.zeros(B, dtype=I32, device=DEV), cached, ps, free, table, seq_len, row_start, slots[:37],
                          free_head=head, free_head_out=head_out, status=status)
    dm.decomoe_paged_append(rows[:, 0], rows[:, 1], slots[:37], kp, vp, status=status)
    head.copy_(head_out)
    held = [[], list(rows[:7].cpu()), list(rows[7:].cpu())]
    q = torch.empty(B, hq, d, dtype=torch.bfloat16, device=DEV)
    kv = torch.empty(B, 2, hkv, d, dtype=torch.bfloat16, device=DEV)
    out = torch.empty_like(q)
    ws = dm.workspace(dm.decomoe_paged_attention_workspace_bytes(B, hq, hkv, d), DEV)

    def step():
        dm.decomoe_paged_plan(cached, fresh, ps, free, table, seq_len, row_start, slots[:B], free_head=head,
                              free_head_out=head_out, status=status)
        dm.decomoe_paged_append(kv[:, 0], kv[:, 1], slots[:B], kp, vp, status=status)
        dm.decomoe_paged_attention(q, kp, vp, table, seq_len, out, ws, status=status)

    q.zero_(), kv.zero_()
    graph = dm.capture_graph(step)
    for i in range(steps):
        q.copy_(torch.randn(B, hq, d, generator=g).to(torch.bfloat16))
        kv.copy_(torch.randn(B, 2, hkv, d, generator=g).to(torch.bfloat16))
        graph.replay()
        cached.copy_(seq_len), head.copy_(head_out)
        torch.cuda.synchronize()
        for b in range(B):
            held[b].append(kv[b].cpu())
            k, v = (f64(torch.stack([r[j] for r in held[b]])) for j in (0, 1))
            assert_close_out(f64(out[b]), O.attention(f64(q[b:b + 1]), k, v)[0], 2 * BF16_REL_L2, 2 * BF16_MAX_ABS)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK


def test_programmatic_launches_change_no_bits():
    """Plan, append, attention, norm and 4-bit products in a row, with and without
    programmatic launches, several times over changing inputs."""
    lens = [300, 41, 0, 1200]
    q, kp, vp, dk, dv, table, dq = _case(lens, 8, 2, 128, 16, 12)
    g = torch.Generator(device=DEV).manual_seed(4)
    w = torch.randint(0, 256, (8 * 128, 128), generator=g, device=DEV, dtype=torch.uint8)
    w_big = torch.randint(0, 256, (20000, 1024), generator=g, device=DEV, dtype=torch.uint8)
    ws, ws_big = (torch.full((n, k // 128), 0.01, dtype=torch.bfloat16, device=DEV) for n, k in ((8 * 128, 256), (20000, 2048)))
    runs = []
    for on in (True, False, True):
        dm.decomoe_set_pdl(on)
        try:
            k, v = dk.clone(), dv.clone()
            h = torch.randn(4, 256, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(torch.bfloat16)
            x8, sc = torch.empty(4, 256, dtype=torch.float8_e4m3fn, device=DEV), torch.empty(4, device=DEV)
            qq, out = torch.empty(4, 8, 128, dtype=torch.bfloat16, device=DEV), torch.empty(4, 8, 128, dtype=torch.bfloat16, device=DEV)
            big = torch.empty(4, 20000, dtype=torch.bfloat16, device=DEV)
            aws = dm.workspace(dm.decomoe_paged_attention_workspace_bytes(4, 8, 2, 128), DEV)
            cached, fresh = _i32([n - 1 if n else 0 for n in lens]), _i32([1 if n else 0 for n in lens])
            n_len, start, slots = _i32([0] * 4), _i32([0] * 5), _i32([0] * 4)
            t = table.to(DEV)
            got = []
            for i in range(5):
                dm.decomoe_add_rmsnorm_q8(h, None, None, y8=x8, y8_scale=sc)
                dm.decomoe_w4_linear(x8, w, ws, qq.view(4, -1), x_scale=sc)
                dm.decomoe_paged_plan(cached, fresh, 16, _i32([0]), t, n_len, start, slots)
                dm.decomoe_paged_append(qq[:, :2], qq[:, 2:4], slots, k, v)
                dm.decomoe_paged_attention(qq, k, v, t, n_len, out, aws)
                dm.decomoe_w4_linear(out.view(4, -1)[:, :256], w, ws, qq.view(4, -1))
                dm.decomoe_w4_linear(torch.cat([out.view(4, -1)] * 2, 1), w_big, ws_big, big)
                dm.decomoe_add_rmsnorm_q8(qq.view(4, -1)[:, :256].contiguous(), h, None, h)
                got += [out.clone(), big.clone(), h.clone()]
            torch.cuda.synchronize()
            runs.append(got)
        finally:
            dm.decomoe_set_pdl(True)
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
    assert all(torch.isfinite(t.float()).all() for t in runs[0])


def test_refusals():
    q, kp, vp, dk, dv, table, dq = _case([20, 5], 8, 2, 64, 16, 1)
    ok = dict(q=dq, k=dk, v=dv, t=table.to(DEV), n=_i32([20, 5]), out=torch.empty(2, 8, 64, dtype=torch.bfloat16, device=DEV),
              ws=dm.workspace(dm.decomoe_paged_attention_workspace_bytes(2, 8, 2, 64), DEV))

    def call(**kw):
        a = ok | kw
        dm.decomoe_paged_attention(a["q"], a["k"], a["v"], a["t"], a["n"], a["out"], a["ws"],
                                   hide_begin=a.get("hb"), hide_count=a.get("hc"))

    call()
    for kw in (dict(n=_i32([20, 5]).long()), dict(t=ok["t"].long()), dict(n=_i32([20])), dict(t=ok["t"][:, ::2]),
               dict(q=dq[:, :6]), dict(k=dk[:, ::2]), dict(v=dv.cpu()), dict(out=ok["out"].float()),
               dict(k=dk.float(), v=dv.float()), dict(hb=_i32([0]), hc=_i32([0, 0]))):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    for kw in (dict(hb=_i32([0, 0])), dict(ws=ok["ws"][:16]), dict(k=dk[:, :3], v=dv[:, :3])):
        with pytest.raises((dm.DecomoeError, ValueError)):
            call(**kw)
    with pytest.raises(dm.DecomoeError):  # 7 query heads on 2 KV heads
        call(q=dq[:, :7], out=torch.empty(2, 7, 64, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(TypeError):
        dm.decomoe_paged_append(dk[0, :4].float(), dv[0, :4].float(), _i32([0, 1, 2, 3]), dk, dv)
    with pytest.raises(ValueError):
        dm.decomoe_paged_append(dk[0, :4], dv[0, :3], _i32([0, 1, 2, 3]), dk, dv)
    torch.cuda.synchronize()
