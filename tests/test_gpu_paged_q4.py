"""The paged cache in 4 bits against the oracle: stored bytes (exact), rows read back
(exact), and the attention of one token per request over its pages.

Attention: keys and values of the pool are the oracle's inputs, so what differs is the
kernel's arithmetic. With p the softmax weights, per output element:
  2^-8 |ref|                   rounding of the output to bf16 (half a step)
  2^-11 sum p step q           weights times steps rounded to fp16, each by 2^-11 of itself at most, or
  n 2^-26 max step             by half of fp16's last place, 2^-25, times codes up to 15, where the n keys'
                               largest step times the largest weight is 2^5 or more
  2 delta sum p |v|            scores off by delta change a weight by the factor exp(+-delta), and
                               the sum of the weights by as much
with delta = (D + 32) 2^-23 sum |q k| scale: fp32 sums of D products and of the groups' terms, in
tensor-core sums that may cut off instead of rounding (2^-23), and the exponentials' 2^-22, which
the 32 covers where sum |q k| scale is 1 or more; below that 2^-20 stands for it. sum |q k| counts the
kernel's own terms, |q| (step code + |low|). Sums of outputs over n keys in fp32 add n 2^-23 sum p (step code +
|low|)."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from paper_2609_38823_gb300.decode import DecodeHead, DecodeStep, PagedCache, quantize_w4
from tests.helpers import BF16_MAX_ABS, BF16_REL_L2, assert_close_out, f64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _i32(v):
    return torch.as_tensor(np.asarray(v, np.int64)).to(I32).to(DEV)


def _tile(d, group):
    return 16 * (d // 2 + 4 * d // group)


def _pool(pages, ps, hkv, d, group, fill=0xFF):
    """A pool of one byte: 0xFF are codes of 15 and parameters that are NaN."""
    return torch.full((pages, hkv, ps // 8, _tile(d, group)), fill, dtype=torch.uint8, device=DEV)


def _rows(n, hkv, d, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, hkv, d, generator=g) * scale
    x[..., ::13] = x[..., ::13] * 6 - 3
    return x.to(torch.bfloat16)


def _stored(pool, k, v, slots, group):
    """The pool (numpy) after the rows have been stored, byte by byte."""
    d, ps = k.shape[2], 8 * pool.shape[2]
    half = 4 * d + 32 * (d // group)
    for value, x in ((0, k), (1, v)):
        codes, step, low = O.q4_quantise(f64(x), group)
        for i, s in enumerate(slots):
            if not 0 <= s < pool.shape[0] * ps:
                continue
            for h in range(x.shape[1]):
                eight = lambda a: np.tile(a[i, h], (8, 1))  # noqa: E731
                with np.errstate(invalid="ignore"):
                    part = O.q4_rows_to_tile(eight(codes), eight(step), eight(low), bool(value))
                t = pool[s // ps, h, s % ps // 8]
                r = s % 8
                for at, w in ((0, d // 2), (4 * d, 4 * (d // group))):
                    t[value * half + at + r * w:value * half + at + (r + 1) * w] = part[at + r * w:at + (r + 1) * w]
    return pool


# ------------------------------------------------------------------ append and read

@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("n,hkv,ps", [(1, 1, 8), (23, 4, 16), (130, 3, 128)])
def test_append_bytes(d, group, n, hkv, ps):
    pages = 2 * n // ps + 3
    r = np.random.default_rng(n + d + group)
    slots = r.permutation(pages * ps)[:n]
    if n > 3:
        slots[2] = -1
    wide = torch.zeros(n, 3 * hkv + 1, d, dtype=torch.bfloat16)
    wide[:, :hkv], wide[:, hkv:2 * hkv] = _rows(n, hkv, d, 1), _rows(n, hkv, d, 2, 0.01)
    on = wide.to(DEV)
    pool = _pool(pages, ps, hkv, d, group, 0xA5)
    status = torch.zeros(1, dtype=I32, device=DEV)
    dm.decomoe_paged_append_q4(on[:, :hkv], on[:, hkv:2 * hkv], _i32(slots), pool, status=status)
    ref = _stored(np.full(pool.shape, 0xA5, np.uint8), wide[:, :hkv], wide[:, hkv:2 * hkv], slots, group)
    assert np.array_equal(pool.cpu().numpy(), ref)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK


def test_append_values_where_a_code_can_go_wrong():
    """Ties between two codes, equal values, one value that stands out, subnormal numbers,
    ranges near the type's largest, zeros of both signs."""
    d, group = 64, 32
    g = torch.Generator().manual_seed(0)
    lattice = torch.arange(32) * 0.5  # step 15.5 / 15 -> ties of a short mantissa
    rows = [lattice, torch.arange(32) % 16 * 1.0, torch.arange(32) % 31 * 0.5, torch.full((32,), 3.25), torch.zeros(32),
            torch.tensor([-0.0, 0.0] * 16), torch.cat([torch.full((31,), 1e-3), torch.tensor([300.0])]),
            torch.arange(32) * 2.0 ** -133, torch.arange(32) * 2.0 ** -126, torch.randint(0, 2, (32,), generator=g) * 2.0 ** -133,
            torch.linspace(-1.6e38, 1.6e38, 32), torch.linspace(1e38, 3.3e38, 32), torch.linspace(-1e-30, 1e-30, 32),
            100 + torch.arange(32) % 2 * 0.5, torch.randn(32, generator=g) * 1e20, 2.0 ** torch.arange(-16, 16)]
    x = torch.stack(rows).to(torch.bfloat16).view(-1, 1, 64)
    n = x.shape[0]
    slots = list(range(n))
    pool = _pool(2, 8, 1, d, group)
    xd = x.to(DEV)
    dm.decomoe_paged_append_q4(xd, xd, _i32(slots), pool)
    ref = _stored(np.full(pool.shape, 0xFF, np.uint8), x, x, slots, group)
    got, half = pool.cpu().numpy(), 4 * d + 64
    for value in (0, 1):
        at = value * half
        assert np.array_equal(got[..., at:at + 4 * d], ref[..., at:at + 4 * d])
        par = lambda p: np.ascontiguousarray(p[..., at + 4 * d:at + half]).view("<u2").astype(np.int64) % 0x8000  # noqa: E731
        sign = lambda p: np.ascontiguousarray(p[..., at + 4 * d:at + half]).view("<u2") >> 15  # noqa: E731
        assert np.array_equal(par(got), par(ref)) and (sign(got) == sign(ref))[par(ref) != 0].all()  # -0 is 0


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_groups_that_are_not_finite_read_back_as_nan(value):
    d, group = 128, 32
    k, v = _rows(9, 2, d, 3), _rows(9, 2, d, 4)
    k[4, 1, 40], v[0, 0, 127], v[8, 1, 0] = value, value, value
    k[2, 0, 64], k[2, 0, 65] = 3.3e38, -3.3e38  # a range that fp32 cannot hold
    pool = _pool(2, 8, 2, d, group, 0)
    slots = _i32(range(9))
    dm.decomoe_paged_append_q4(k.to(DEV), v.to(DEV), slots, pool)
    ko, vo = torch.zeros(9, 2, d, dtype=torch.bfloat16, device=DEV), torch.zeros(9, 2, d, dtype=torch.bfloat16, device=DEV)
    dm.decomoe_paged_read_q4(slots, pool, ko, vo)
    want_k, want_v = (torch.zeros(9, 2, d, dtype=torch.bool) for _ in range(2))
    want_k[4, 1, 32:64] = want_k[2, 0, 64:96] = want_v[0, 0, 96:] = want_v[8, 1, :32] = True
    assert torch.equal(torch.isnan(ko).cpu(), want_k) and torch.equal(torch.isnan(vo).cpu(), want_v)
    assert torch.isfinite(ko.cpu()[~want_k]).all() and torch.isfinite(vo.cpu()[~want_v]).all()


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("n,hkv,ps", [(1, 1, 16), (57, 5, 8), (300, 2, 64)])
def test_read_values(d, group, n, hkv, ps):
    pages = n // ps + 3
    pool = torch.randint(0, 256, (pages, hkv, ps // 8, _tile(d, group)), generator=torch.Generator().manual_seed(n), dtype=torch.uint8)
    G = d // group
    for at in (4 * d, 8 * d + 32 * G):  # parameters of a sensible size
        par = (torch.rand(pages, hkv, ps // 8, 16 * G, generator=torch.Generator().manual_seed(at)) - 0.3).to(torch.bfloat16)
        pool[..., at:at + 32 * G] = par.view(torch.uint8)
    k, v, *_ = O.q4_values(pool.numpy(), d, group)
    r = np.random.default_rng(n)
    slots = r.permutation(pages * ps)[:n]
    out = torch.full((n, 2 * hkv + 1, d), 7.0, dtype=torch.bfloat16, device=DEV)  # keys and values side by side
    skip = n // 2
    slots[skip] = -1 if n > 1 else slots[skip]
    status = torch.zeros(1, dtype=I32, device=DEV)
    dm.decomoe_paged_read_q4(_i32(slots), pool.to(DEV), out[:, :hkv], out[:, hkv:2 * hkv], status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    got = f64(out)
    for i, x in enumerate((k, v)):
        ref = O.bf16(x.reshape(pages * ps, hkv, d)[slots])
        if n > 1:
            ref[skip] = 7.0
        assert np.array_equal(got[:, i * hkv:(i + 1) * hkv], ref)
    assert (got[:, 2 * hkv] == 7.0).all()


@pytest.mark.parametrize("size", [1e-40, 1e-38, 1e-30, 1e30])
def test_read_values_of_any_size(size):
    """Steps and lows down to subnormal numbers, as low + step * code in fp32 gives them."""
    d, group, n = 128, 32, 24
    k, v = _rows(n, 2, d, 5, size), _rows(n, 2, d, 6, size)
    k[:, :, 64:] *= 100
    pool = _pool(3, 8, 2, d, group, 0)
    slots = _i32(range(n))
    dm.decomoe_paged_append_q4(k.to(DEV), v.to(DEV), slots, pool)
    out = torch.empty(2, n, 2, d, dtype=torch.bfloat16, device=DEV)
    dm.decomoe_paged_read_q4(slots, pool, out[0], out[1])
    for got, ref in zip(out, O.q4_values(pool.cpu().numpy(), d, group)[:2]):
        # low + step * code in one rounding to fp32, then to bf16
        ref = ref.reshape(n, 2, d).astype(np.float32).astype(np.float64)
        assert np.array_equal(f64(got), O.bf16(ref))


def test_slots_outside_the_pool_are_skipped_and_marked():
    d, group, n = 64, 64, 5
    k = _rows(n, 2, d, 5).to(DEV)
    status = torch.zeros(1, dtype=I32, device=DEV)
    for bad in (24, -2, 2 ** 31 - 1, -2 ** 31):
        pool = _pool(3, 8, 2, d, group, 0)
        slots = _i32([0, bad, 9, -1, 23])
        dm.decomoe_paged_append_q4(k, k, slots, pool, status=status)
        assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
        ref = _stored(np.zeros(pool.shape, np.uint8), k.cpu(), k.cpu(), [0, -1, 9, -1, 23], group)
        assert np.array_equal(pool.cpu().numpy(), ref)
        ko, vo = (torch.full((n, 2, d), 5.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        dm.decomoe_paged_read_q4(slots, pool, ko, vo, status=status)
        assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
        assert (ko[1] == 5).all() and (vo[3] == 5).all() and not (ko[0] == 5).all()


def test_rows_read_back_for_a_chunk_of_a_prompt():
    """Two chunks of a prompt: stored, read back, attended; and the same rows by the one-token call."""
    hq, hkv, d, group, ps, n1, n2 = 8, 2, 128, 64, 16, 75, 61
    cache = PagedCache(1, 2, pages=20, page_size=ps, max_pages=12, hkv=hkv, d=d, bits=4, group=group)
    rows = [(_rows(n, hkv, d, i).to(DEV), _rows(n, hkv, d, 9 + i).to(DEV)) for i, n in ((0, n1), (1, n2))]
    for (k, v), n in zip(rows, (n1, n2)):
        slots = torch.empty(n, dtype=I32, device=DEV)
        cache.plan(_i32([0, n]), slots)
        cache.append(0, k, v, slots)
        cache.advance()
    C = n1 + n2
    q = _rows(n2, hq, d, 3).to(DEV)
    out, ko, vo = torch.empty_like(q), *(torch.empty(C, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = dm.workspace(dm.decomoe_attention_workspace_bytes(n2, C, hq, hkv, d), DEV)
    cache.attend_chunk(0, q, cache.slots_of(1, C), ko, vo, out, ws)
    kd, vd, *_ = O.q4_values(cache.pool[0].cpu().numpy(), d, group)
    flat = lambda x: x.reshape(-1, hkv, d)[cache.slots_of(1, C).cpu().numpy()]  # noqa: E731
    assert np.array_equal(f64(ko), O.bf16(flat(kd))) and np.array_equal(f64(vo), O.bf16(flat(vd)))
    assert_close_out(f64(out), O.attention(f64(q), f64(ko), f64(vo)), BF16_REL_L2, BF16_MAX_ABS, "chunk")
    one = torch.empty(2, hq, d, dtype=torch.bfloat16, device=DEV)
    cache.attend(0, torch.stack([q[0], q[-1]]), one, dm.workspace(cache.workspace_bytes(2, hq), DEV))
    assert (one[0] == 0).all()
    assert_close_out(f64(one[1]), O.attention(f64(q[-1:]), flat(kd), flat(vd))[0], BF16_REL_L2, BF16_MAX_ABS, "one token")
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK


# ------------------------------------------------------------------ attention

def _case(lens, hq, hkv, d, group, ps, seed, hide=None, k_scale=1.0):
    """Requests' rows stored in pages of a pool that is NaN where nothing was stored; pages that
    hold only hidden rows are given back."""
    r = np.random.default_rng(seed)
    width = max(1, max(-(-n // ps) for n in lens) + 1)
    P = sum(-(-n // ps) for n in lens) + 3
    ids = r.permutation(P)
    table = r.integers(-5, P + 50, (len(lens), width))  # unused entries: anything
    pool, at = _pool(P, ps, hkv, d, group), 0
    for b, n in enumerate(lens):
        used = -(-n // ps)
        table[b, :used] = ids[at:at + used]
        at += used
        if n == 0:
            continue
        slots = [table[b, j // ps] * ps + j % ps for j in range(n)]
        k, v = _rows(n, hkv, d, 100 * seed + b, k_scale).to(DEV), _rows(n, hkv, d, 100 * seed + 50 + b).to(DEV)
        dm.decomoe_paged_append_q4(k, v, _i32(slots), pool)
        if hide is not None:
            for i in range(used):
                if all(hide[b][0] <= j < hide[b][0] + hide[b][1] for j in range(i * ps, min(n, (i + 1) * ps))):
                    table[b, i] = -1
    q = _rows(len(lens), hq, d, 7 * seed + 1)
    return q, pool, table


def _attend(q, pool, table, lens, hide=None, scale=0.0, status=None, ws=None, stream=None):
    out = torch.full(tuple(q.shape), 77.0, dtype=torch.bfloat16, device=DEV)
    B, hq, d = q.shape
    if ws is None:
        ws = dm.workspace(dm.decomoe_paged_attention_q4_workspace_bytes(B, hq, pool.shape[1], d), DEV)
    hb, hc = (None, None) if hide is None else (_i32([h[i] for h in hide]) for i in (0, 1))
    dm.decomoe_paged_attention_q4(q, pool, _i32(table), _i32(lens), out, ws, hide_begin=hb, hide_count=hc, scale=scale,
                                  status=status, stream=stream)
    return out


def _ref(q, pool, table, lens, group, hide=None, scale=None):
    """(results, bounds) by request from the pool's bytes."""
    q = f64(q)
    B, hq, d = q.shape
    ps, hkv = 8 * pool.shape[2], pool.shape[1]
    kd, vd, span, code = O.q4_values(pool.cpu().numpy(), d, group)
    out, tol = np.zeros(q.shape), np.zeros(q.shape)
    scale = d ** -0.5 if not scale else scale
    for b, n in enumerate(lens):
        j = np.array([i for i in range(n) if hide is None or not max(hide[b][0], 0) <= i < max(hide[b][0], 0) + max(hide[b][1], 0)], int)
        if not len(j):
            continue
        at = (np.asarray(table)[b, j // ps], j % ps)
        for h in range(hq):
            g = h // (hq // hkv)
            k, v = kd[at][:, g], vd[at][:, g]
            s = scale * (k @ q[b, h])
            p = np.exp(s - s.max())
            p /= p.sum()
            ks, vs = span[at][:, g], code[at][:, g]
            size = ((ks + np.abs(k - ks)) @ np.abs(q[b, h])).max() * scale
            delta = (d + 32) * 2.0 ** -23 * size + 2.0 ** -20
            terms = p @ (vs + np.abs(v - vs))
            out[b, h] = p @ v
            tol[b, h] = (2.0 ** -8 * np.abs(out[b, h]) + 2.0 ** -11 * (p @ vs) + len(j) * 2.0 ** -26 * vs.max()
                         + (2 * delta + len(j) * 2.0 ** -23) * terms)
    return out, tol


def _check(lens, hq, hkv, d, group, ps, seed=0, hide=None, **kw):
    q, pool, table = _case(lens, hq, hkv, d, group, ps, seed, hide, **kw)
    status = torch.zeros(1, dtype=I32, device=DEV)
    wide = torch.zeros(len(lens), hq + 3, d, dtype=torch.bfloat16, device=DEV)  # queries inside wider rows
    wide[:, :hq] = q.to(DEV)
    out = _attend(wide[:, :hq], pool, table, lens, hide, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    ref, tol = _ref(q, pool, table, lens, group, hide)
    off = np.abs(f64(out) - ref)
    assert (off <= tol).all(), (off / np.maximum(tol, 1e-30)).max()
    rel = np.linalg.norm(off) / max(np.linalg.norm(ref), 1e-30)
    assert rel <= BF16_REL_L2, rel
    return out, q, pool, table


@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("hq,hkv,ps", [(8, 1, 16), (32, 4, 64), (5, 5, 8), (24, 4, 128), (32, 2, 8), (34, 2, 32)])
def test_attention_parity(d, group, hq, hkv, ps):
    lens = [1, 8, 0, 15, 16, 17, 31, 33, 64, 200, 129]
    out, *_ = _check(lens, hq, hkv, d, group, ps, seed=hq + ps)
    assert (out[2] == 0).all()


@pytest.mark.parametrize("lens,hq,hkv,d,group,ps", [
    ([2049], 32, 4, 128, 64, 16), ([16385], 32, 4, 128, 128, 64), ([3000, 0, 5, 1, 700], 16, 16, 64, 32, 32),
    ([40000], 8, 1, 64, 64, 128), ([1], 1, 1, 128, 32, 8), ([0, 0], 8, 2, 64, 64, 16), ([7] * 300, 8, 2, 128, 64, 8),
    ([513, 512, 511] * 20, 16, 2, 128, 32, 16), ([5000, 4000], 16, 1, 64, 32, 16)])
def test_attention_lengths(lens, hq, hkv, d, group, ps):
    _check(lens, hq, hkv, d, group, ps, seed=len(lens))


@pytest.mark.parametrize("d,group,ps", [(128, 64, 16), (64, 32, 64), (128, 128, 8), (128, 32, 32), (64, 64, 8)])
def test_attention_hidden_blocks(d, group, ps):
    lens = [400, 400, 90, 33, 1, 700, 64, 64, 0, 50, 100, 47]
    # inside pages, whole pages, to the end, from the start, everything, nothing, inside one tile, ends together
    hide = [(16, 320), (13, 200), (50, 40), (0, 17), (0, 1), (100, 0), (0, 64), (60, 4), (0, 3), (18, 5), (31, 2), (8, 39)]
    out, q, pool, table = _check(lens, 16, 4, d, group, ps, seed=ps, hide=hide)
    assert (out[4] == 0).all() and (out[6] == 0).all()


def test_attention_hidden_blocks_past_the_ends_are_cut():
    lens, hide = [50, 50, 50, 50], [(-5, 10), (40, 100), (60, 10), (10, -4)]
    q, pool, table = _case(lens, 8, 2, 64, 32, 16, 1)
    same = [(0, 10), (40, 10), (0, 0), (0, 0)]  # a negative begin is 0, a negative count none
    assert torch.equal(_attend(q.to(DEV), pool, table, lens, hide), _attend(q.to(DEV), pool, table, lens, same))


def test_attention_values_that_are_not_finite_stay_in_their_request():
    lens = [40, 40, 40, 40]
    q, pool, table = _case(lens, 8, 2, 128, 32, 16, 2)
    dq = q.to(DEV)
    clean = _attend(dq, pool, table, lens)
    k, v = _rows(1, 2, 128, 5).to(DEV), _rows(1, 2, 128, 6).to(DEV)
    v[0, 1, 37] = float("inf")  # a value of KV head 1: its group of features
    dm.decomoe_paged_append_q4(k, v, _i32([table[1, 0] * 16 + 3]), pool)
    k[0, 0, 0], v[0, 1, 37] = float("nan"), 0  # a key of KV head 0: all of its query heads
    dm.decomoe_paged_append_q4(k, v, _i32([table[2, 1] * 16 + 2]), pool)
    dq[3, 5, 9] = float("inf")  # a query: its own row
    out = _attend(dq, pool, table, lens)
    assert torch.equal(out[0], clean[0])
    assert torch.isnan(out[1, 4:, 32:64]).all() and torch.isfinite(out[1, :4]).all()
    assert torch.isfinite(out[1, 4:, :32]).all() and torch.isfinite(out[1, 4:, 64:]).all()
    assert torch.isnan(out[2, :4]).all() and torch.isfinite(out[2, 4:]).all()
    assert torch.isnan(out[3, 5]).all() and torch.equal(out[3, :5], clean[3, :5]) and torch.equal(out[3, 6:], clean[3, 6:])


@pytest.mark.parametrize("group", [32, 128])
def test_attention_large_scores(group):
    # scores of some thousands: one key takes almost all of the weight
    _check([1, 60, 300], 8, 2, 128, group, 16, seed=6, k_scale=300.0)


def test_attention_bad_tables_and_lengths_are_marked():
    lens, group = [100, 40], 64
    q, pool, table = _case(lens, 8, 2, 128, group, 16, 4)
    dq, status = q.to(DEV), torch.zeros(1, dtype=I32, device=DEV)
    for page in (-1, pool.shape[0], 2 ** 31 - 1):
        bad = table.copy()
        bad[0, 2] = page  # rows 32..47 count as hidden
        out = _attend(dq, pool, bad, lens, status=status)
        assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
        ref, tol = _ref(q, pool, table, lens, group, [(32, 16), (0, 0)])
        assert (np.abs(f64(out) - ref) <= tol).all()
    bad = table.copy()
    bad[1] = -1  # a request without any page: nothing to see
    out = _attend(dq, pool, bad, lens, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT and (out[1] == 0).all()
    # a negative length is 0, one beyond the table ends with it
    n = 6 * 16
    out = _attend(dq, pool, table[:, :6], [n + 500, -3], status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
    assert (out[1] == 0).all()
    ref, tol = _ref(q, pool, table, [n, 0], group)
    assert (np.abs(f64(out) - ref) <= tol).all()


def test_attention_pages_of_half_a_tile():
    """Eight rows to a page: one half of a tile hidden or without a page, the other not."""
    lens, group = [64, 64], 64
    q, pool, table = _case(lens, 8, 2, 64, group, 8, 8)
    status = torch.zeros(1, dtype=I32, device=DEV)
    bad = table.copy()
    bad[0, 3] = -1
    out = _attend(q.to(DEV), pool, bad, lens, status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_ERR_BAD_INPUT
    ref, tol = _ref(q, pool, table, lens, group, [(24, 8), (0, 0)])
    assert (np.abs(f64(out) - ref) <= tol).all()
    out = _attend(q.to(DEV), pool, bad, lens, [(24, 8), (60, 2)], status=status)
    assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    ref, tol = _ref(q, pool, table, lens, group, [(24, 8), (60, 2)])
    assert (np.abs(f64(out) - ref) <= tol).all()


def test_pool_beyond_32_bit_offsets():
    # 5.2 GB: byte offsets past 2^32; pages far apart, every call
    P, ps, hkv, d, group = 70000, 64, 8, 128, 64
    pool = torch.empty(P, hkv, ps // 8, _tile(d, group), dtype=torch.uint8, device=DEV)
    pages = [P - 1, P - 7, 66000, 33000, 3]
    lens = [200, 64, 40]
    table = np.array([[pages[0], pages[1], pages[2], pages[3]], [pages[4], -1, -1, -1], [pages[1], -1, -1, -1]])
    for i, p in enumerate(pages):
        dm.decomoe_paged_append_q4(_rows(ps, hkv, d, i).to(DEV), _rows(ps, hkv, d, 20 + i).to(DEV),
                                   _i32(p * ps + np.arange(ps)), pool)
    q = _rows(3, 16, d, 50)
    out = _attend(q.to(DEV), pool, table, lens)
    small = torch.stack([pool[p] for p in pages]).cpu()
    tab = np.array([[pages.index(p) if p in pages else -1 for p in row] for row in table])
    ref, tol = _ref(q, small, tab, lens, group)
    assert (np.abs(f64(out) - ref) <= tol).all()
    ko, vo = (torch.empty(1, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    dm.decomoe_paged_read_q4(_i32([(P - 1) * ps + 63]), pool, ko, vo)
    k, v, *_ = O.q4_values(small.numpy(), d, group)
    assert np.array_equal(f64(ko[0]), O.bf16(k[0, 63])) and np.array_equal(f64(vo[0]), O.bf16(v[0, 63]))


def test_pages_apart():
    """Two layers' pages side by side: the pool is a slice, pages lie further apart than they are long."""
    lens, group = [90, 33], 32
    q, pool, table = _case(lens, 8, 2, 64, group, 16, 5)
    both = torch.full((pool.shape[0], 2, *pool.shape[1:]), 0xFF, dtype=torch.uint8, device=DEV)
    both[:, 1] = pool
    assert torch.equal(_attend(q.to(DEV), pool, table, lens), _attend(q.to(DEV), both[:, 1], table, lens))
    k = _rows(2, 2, 64, 1).to(DEV)
    slots = _i32([3, 40])
    dm.decomoe_paged_append_q4(k, k, slots, pool)
    dm.decomoe_paged_append_q4(k, k, slots, both[:, 1])
    assert torch.equal(both[:, 1], pool) and (both[:, 0] == 0xFF).all()


def test_scale_streams_and_the_same_bits_again():
    lens, group = [70, 3000, 0, 555], 64
    q, pool, table = _case(lens, 8, 2, 128, group, 16, 9)
    dq = q.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = _attend(dq, pool, table, lens, scale=0.3)
    torch.cuda.synchronize()
    ref, tol = _ref(q, pool, table, lens, group, scale=0.3)
    assert (np.abs(f64(out) - ref) <= tol).all()
    for i in range(4):
        dm.decomoe_set_pdl(i & 1)
        try:
            again = _attend(dq, pool, table, lens, scale=0.3, stream=side if i < 2 else None)
            torch.cuda.synchronize()
        finally:
            dm.decomoe_set_pdl(True)
        assert torch.equal(again, out)


def _job(lens, seed):
    """run(n, stream): n rounds of all four calls on tensors of the job's own, their results stacked."""
    q, pool, table = _case(lens, 16, 2, 128, 64, 16, seed)
    k, v = _rows(3, 2, 128, seed + 10).to(DEV), _rows(3, 2, 128, seed + 20).to(DEV)
    x = torch.randn(5, 40001, generator=torch.Generator().manual_seed(seed)).to(DEV)
    q, table, seq, where, tokens = q.to(DEV), _i32(table), _i32(lens), _i32([2, 9, 15]), _i32([0, 7, 40000, -1, 3])
    ws = dm.workspace(dm.decomoe_paged_attention_q4_workspace_bytes(len(lens), 16, 2, 128), DEV)
    scratch = _pool(1, 16, 2, 128, 64)

    def outputs(n):
        bf = dict(dtype=torch.bfloat16, device=DEV)
        return torch.zeros(n, len(lens), 16, 128, **bf), torch.zeros(n, 2, 3, 2, 128, **bf), torch.zeros(n, 5, device=DEV)

    def run(to, stream):
        for out, kv, lp in zip(*to):
            dm.decomoe_paged_attention_q4(q, pool, table, seq, out, ws, stream=stream)
            dm.decomoe_paged_append_q4(k, v, where, scratch, stream=stream)
            dm.decomoe_paged_read_q4(where, scratch, kv[0], kv[1], stream=stream)
            dm.decomoe_token_logprobs(x, tokens, lp, stream=stream)

    return outputs, run


def test_calls_at_once_on_two_streams():
    """A workspace and a pool each, many calls under way together: every result as if it were alone."""
    jobs = [_job([4000, 9, 700], 20), _job([2500] * 7, 60)]
    alone, many = [o(1) for o, _ in jobs], [o(40) for o, _ in jobs]
    for (_, run), to in zip(jobs, alone):
        run(to, None)
    torch.cuda.synchronize()
    for (_, run), to, side in zip(jobs, many, [torch.cuda.Stream() for _ in jobs]):
        run(to, side)
    torch.cuda.synchronize()
    for a, b in zip(alone, many):
        for one, got in zip(a, b):
            assert torch.equal(got, one.expand_as(got))


def test_a_wait_that_ends_in_time_leaves_no_mark():
    """The smallest time limit that a call can meet is not taken for a fault: copies arrive."""
    lens = [2000] * 8
    q, pool, table = _case(lens, 8, 2, 128, 64, 16, 3)
    status = torch.zeros(1, dtype=I32, device=DEV)
    dm.decomoe_set_wait_limit_ns(1_000_000_000)
    try:
        _attend(q.to(DEV), pool, table, lens, status=status)
        assert dm.decomoe_read_status(status) == dm.DECOMOE_OK
    finally:
        dm.decomoe_set_wait_limit_ns(2_000_000_000)


# ------------------------------------------------------------------ steps

def test_steps_in_two_captured_graphs():
    """Plan, append and attention of one step captured in two graphs with a workspace each, over two
    caches, replayed in turn while the requests grow over page ends."""
    hq, hkv, d, group, ps, B, steps = 8, 2, 64, 32, 8, 3, 18
    g = torch.Generator().manual_seed(1)
    caches = [PagedCache(1, B, pages=40, page_size=ps, max_pages=8, hkv=hkv, d=d, bits=4, group=group) for _ in range(2)]
    state = []
    for cache in caches:
        prompt = [0, 7, 30]
        slots = torch.empty(37, dtype=I32, device=DEV)
        cache.plan(_i32(prompt), slots)
        rows = torch.randn(37, 2, hkv, d, generator=g).to(torch.bfloat16).to(DEV)
        cache.append(0, rows[:, 0], rows[:, 1], slots)
        cache.advance()
        cache.active.fill_(1)
        e = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        s = dict(cache=cache, q=e(B, hq, d), kv=e(B, 2, hkv, d), out=e(B, hq, d), slots=torch.empty(B, dtype=I32, device=DEV),
                 ws=dm.workspace(cache.workspace_bytes(B, hq), DEV))

        def step(s=s):
            c = s["cache"]
            c.plan_step(c.active, s["slots"])
            c.append(0, s["kv"][:, 0], s["kv"][:, 1], s["slots"])
            c.attend(0, s["q"], s["out"], s["ws"])

        s["graph"] = dm.capture_graph(step)
        state.append(s)
    for i in range(steps):
        for s in state:
            s["q"].copy_(torch.randn(B, hq, d, generator=g).to(torch.bfloat16))
            s["kv"].copy_(torch.randn(B, 2, hkv, d, generator=g).to(torch.bfloat16))
            s["graph"].replay()
        for s in state:
            s["cache"].advance()
        torch.cuda.synchronize()
        for s in state:
            c = s["cache"]
            ref, tol = _ref(s["q"], c.pool[0], c.table.cpu().numpy(), c.seq_len.tolist(), group)
            assert (np.abs(f64(s["out"]) - ref) <= tol).all()
    assert all(dm.decomoe_read_status(c.status) == dm.DECOMOE_OK for c in caches)
    assert caches[0].cached.tolist() == [steps, 7 + steps, 30 + steps]


def test_decode_steps_on_a_cache_in_4_bits():
    """DecodeStep and DecodeHead: every layer's attention on what its own cache holds, and the
    log probabilities of the step's logits."""
    from tests.test_gpu_decode_step import D, HKV, HQ, K, L, D_MODEL, _model

    layers, _ = _model()
    lens, group, V = [5, 47, 130], 32, 333
    cache = PagedCache(L, 3, pages=60, page_size=8, max_pages=24, hkv=HKV, d=D, bits=4, group=group)
    n = sum(lens)
    slots = torch.empty(n, dtype=I32, device=DEV)
    cache.plan(_i32(lens), slots)
    for l in range(L):
        cache.append(l, _rows(n, HKV, D, l).to(DEV), _rows(n, HKV, D, 10 + l).to(DEV), slots)
    cache.advance()
    cache.hide(2, 16, 100, from_layer=1)
    step = DecodeStep(layers, cache, 3, HQ, K)
    head = DecodeHead(None, quantize_w4(torch.randn(V, D_MODEL, generator=torch.Generator().manual_seed(2)).to(DEV)), 3, n=4)
    seen = []

    def check(l, s, h_in, h_out):
        torch.cuda.synchronize()
        hide = [(0, 0), (0, 0), (16, 100) if l >= 1 else (0, 0)]
        ref, tol = _ref(s.q, cache.pool[l], cache.table.cpu().numpy(), cache.seq_len.tolist(), group, hide)
        assert (np.abs(f64(s.heads) - ref) <= tol).all()
        k, *_ = O.q4_values(cache.pool[l].cpu().numpy(), D, group)
        codes, st, low = O.q4_quantise(f64(s.k_new), group)
        assert np.array_equal(k.reshape(-1, HKV, D)[s.slots.cpu().numpy()], np.repeat(low, group, -1) + np.repeat(st, group, -1) * codes)
        seen.append(l)

    h = torch.randn(3, D_MODEL, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    for i in range(4):
        h = step(h, trace=check).clone()
        cache.advance()
        logits = f64(head(h))
        tokens = _i32([i, 100 + i, V - 1 - i])
        head.score(tokens, temperature=0.7)
        lp, ent, ids, top = O.token_logprobs(logits, tokens.tolist(), 4, 1 / 0.7)
        assert np.array_equal(head.top_id.cpu().numpy(), ids)
        for got, ref in ((head.logprob, lp), (head.entropy, ent), (head.top_logprob, top)):
            assert np.abs(f64(got) - ref).max() <= 2e-5 * (1 + np.abs(ref).max())
        kept = head.logprob.clone()
        head.score()  # without tokens: logprob is left alone
        assert torch.equal(kept, head.logprob)
    assert seen == list(range(L)) * 4 and dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK


def test_refusals():
    q, pool, table = _case([20, 5], 8, 2, 64, 32, 16, 1)
    ok = dict(q=q.to(DEV), p=pool, t=_i32(table), n=_i32([20, 5]), out=torch.empty(2, 8, 64, dtype=torch.bfloat16, device=DEV),
              ws=dm.workspace(dm.decomoe_paged_attention_q4_workspace_bytes(2, 8, 2, 64), DEV))

    def call(**kw):
        a = ok | kw
        dm.decomoe_paged_attention_q4(a["q"], a["p"], a["t"], a["n"], a["out"], a["ws"], hide_begin=a.get("hb"),
                                      hide_count=a.get("hc"))

    call()
    for kw in (dict(n=ok["n"].long()), dict(t=ok["t"].long()), dict(n=_i32([20])), dict(t=ok["t"][:, ::2]), dict(q=ok["q"][:, :6]),
               dict(p=pool[:, :, ::2]), dict(p=pool[..., :-16]), dict(p=pool.cpu()), dict(p=pool.to(torch.int8)),
               dict(out=ok["out"].float()), dict(q=ok["q"].half()), dict(hb=_i32([0]), hc=_i32([0, 0]))):
        with pytest.raises((ValueError, TypeError)):
            call(**kw)
    for kw in (dict(hb=_i32([0, 0])), dict(ws=ok["ws"][:16]), dict(q=ok["q"][:, :7], out=ok["out"][:, :7].contiguous())):
        with pytest.raises(dm.DecomoeError):
            call(**kw)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    s = _i32([0, 1, 2, 3])
    for kw in (dict(k=k.float()), dict(v=k[:3]), dict(s=s.long()), dict(p=pool[:, :1]), dict(k=k[:, :, ::2])):
        a = dict(k=k, v=k, s=s, p=pool) | kw
        with pytest.raises((ValueError, TypeError)):
            dm.decomoe_paged_append_q4(a["k"], a["v"], a["s"], a["p"])
        with pytest.raises((ValueError, TypeError)):
            dm.decomoe_paged_read_q4(a["s"], a["p"], a["k"], a["v"])
    with pytest.raises(dm.DecomoeError):
        dm.decomoe_paged_read_q4(s, pool, k, k)  # one output for two
    with pytest.raises(ValueError):
        PagedCache(1, 1, pages=2, page_size=4, max_pages=2, hkv=1, d=64, bits=4)
    torch.cuda.synchronize()


@pytest.mark.parametrize("low,high", [(-30, -30), (-80, -80), (25, 25), (90, 90), (-25, 25), (0, 12)])
def test_attention_values_of_any_size(low, high):
    """Values whose sizes lie far from 1, or far apart from key to key: the weights are scaled with the
    largest step seen so far."""
    lens, hq, hkv, d, group, ps = [300, 77, 1200], 8, 2, 128, 64, 16
    q, pool, table = _case(lens, hq, hkv, d, group, ps, 11)
    r = np.random.default_rng(5)
    for b, n in enumerate(lens):
        k = _rows(n, hkv, d, b)
        v = (_rows(n, hkv, d, 20 + b).double() * torch.from_numpy(2.0 ** r.integers(low, high + 1, (n, 1, 1)))).to(torch.bfloat16)
        slots = [table[b, j // ps] * ps + j % ps for j in range(n)]
        dm.decomoe_paged_append_q4(k.to(DEV), v.to(DEV), _i32(slots), pool)
    ref, tol = _ref(q, pool, table, lens, group)
    off = np.abs(f64(_attend(q.to(DEV), pool, table, lens)) - ref)
    assert (off <= tol + 2.0 ** -133).all(), (off / np.maximum(tol, 1e-300)).max()


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e12, 1e30])
def test_attention_queries_of_any_size(size):
    lens = [300, 77]
    q, pool, table = _case(lens, 8, 2, 128, 32, 16, 12, k_scale=1.0 / size if 1e-13 < size < 1e13 else 1.0)
    q = (q.double() * size).to(torch.bfloat16)
    out = _attend(q.to(DEV), pool, table, lens)
    ref, tol = _ref(q, pool, table, lens, 32)
    assert (np.abs(f64(out) - ref) <= tol).all()


def test_attention_queries_of_zeros():
    lens = [300, 17, 5]
    q, pool, table = _case(lens, 8, 2, 128, 32, 16, 13)
    q[0], q[1, 3], q[2] = 0, 0, 2.0 ** -130
    out = _attend(q.to(DEV), pool, table, lens)
    ref, tol = _ref(q, pool, table, lens, 32)
    assert (np.abs(f64(out) - ref) <= tol).all()
