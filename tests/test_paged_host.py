"""Host-side checks of the paged cache's and the dense steps' calls that need no
GPU (refusals before anything is launched, on the C ABI and on tensors), and pins
of their oracle against other routes."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()
    return dm.lib()


P = ctypes.c_void_p(0x1000)  # never dereferenced: the checks fail first
Q = ctypes.c_void_p(0x2000)


def test_plan_arguments():
    def plan(B=4, ps=16, n_free=8, head_in=None, head_out=None, max_pages=4, seq_len=Q, start=P, N=8, slots=P, cached=P,
             table=P, pages=P):
        return dm.lib().decomoe_paged_plan(cached, P, B, ps, pages, n_free, head_in, head_out, table, max_pages, seq_len,
                                           start, slots, P, N, None, None)

    for kw in (dict(B=-1), dict(B=4097), dict(ps=0), dict(ps=12), dict(ps=-16), dict(n_free=-1), dict(max_pages=-1),
               dict(max_pages=1 << 28), dict(N=-1), dict(N=1 << 31), dict(start=None), dict(slots=None), dict(cached=None),
               dict(table=None), dict(pages=None), dict(seq_len=None), dict(seq_len=P), dict(head_in=P, head_out=P)):
        assert plan(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
        assert b"paged_plan" in dm.lib().decomoe_last_error()


def test_append_arguments():
    def append(k=P, ks=512, v=P, vs=512, N=4, width=512, dtype=0, slots=P, kp=P, pages=8, ps=16, stride=16 * 512):
        return dm.lib().decomoe_paged_append(k, ks, v, vs, N, width, dtype, slots, kp, P, pages, ps, stride, None, None)

    for kw in (dict(dtype=2), dict(N=-1), dict(width=0), dict(ps=24), dict(pages=-1), dict(pages=1 << 28),
               dict(stride=16 * 512 - 8), dict(k=None), dict(slots=None), dict(kp=None), dict(ks=504), dict(vs=511),
               dict(width=508, stride=16 * 512), dict(ks=516), dict(stride=16 * 512 + 4), dict(k=ctypes.c_void_p(0x1008))):
        assert append(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
    assert append(N=0, k=None, v=None, slots=None) == dm.DECOMOE_OK


def test_attention_arguments():
    def attend(q=P, qs=4096, B=2, kp=P, pages=8, ps=16, stride=16 * 512, table=P, max_pages=4, lens=P, hb=None, hc=None,
               hq=32, hkv=4, d=128, out=P, ws=P, ws_bytes=1 << 30):
        return dm.lib().decomoe_paged_attention(q, qs, B, kp, P, pages, ps, stride, table, max_pages, lens, hb, hc, hq, hkv,
                                                d, 0.0, out, ws, ws_bytes, None, None)

    for kw in (dict(B=-1), dict(B=4097), dict(d=96), dict(hq=30), dict(hkv=0), dict(hq=2), dict(hq=1028), dict(ps=10),
               dict(pages=-1), dict(pages=1 << 28), dict(max_pages=-1), dict(max_pages=1 << 28),
               dict(stride=16 * 512 - 8), dict(stride=16 * 512 + 4), dict(qs=4095), dict(qs=4100), dict(hb=P), dict(hc=P),
               dict(q=None), dict(lens=None), dict(out=None), dict(table=None), dict(kp=None),
               dict(out=ctypes.c_void_p(0x1004)), dict(ws=ctypes.c_void_p(0x1008))):
        assert attend(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
    # more tiles than a launch counts
    assert attend(B=4096, max_pages=1 << 22, hq=64, hkv=64, stride=16 * 64 * 128, qs=64 * 128) == dm.DECOMOE_ERR_INVALID_ARG
    assert attend(ws=None) == dm.DECOMOE_ERR_WORKSPACE and attend(ws_bytes=16) == dm.DECOMOE_ERR_WORKSPACE
    assert attend(B=0, q=None, out=None, ws=None, ws_bytes=0) == dm.DECOMOE_OK
    L = dm.lib()
    assert L.decomoe_paged_attention_workspace_bytes(0, 32, 4, 128) == 0
    assert L.decomoe_paged_attention_workspace_bytes(4, 2, 4, 128) == 0
    assert L.decomoe_paged_attention_workspace_bytes(4, 48, 4, 128) > L.decomoe_paged_attention_workspace_bytes(4, 32, 4, 128)


@pytest.mark.parametrize("ps,max_pages", [(16, 2 ** 27 - 1), (1, 2 ** 31 - 1), (1, 2 ** 31 - 31)])
def test_attention_refuses_a_table_whose_last_tile_passes_32_bits(ps, max_pages):
    """A length of max_pages * page_size, rounded up to a tile of 32 keys, has to fit 32 bits."""
    args = (P, 64, 1, P, P, 8, ps, ps * 64, P, max_pages, P, None, None, 1, 1, 64, 0.0, P, P, 1 << 30, None, None)
    assert dm.lib().decomoe_paged_attention(*args) == dm.DECOMOE_ERR_INVALID_ARG
    assert b"max_pages" in dm.lib().decomoe_last_error()


def test_dense_arguments():
    L = dm.lib()

    def norm(x=P, res=None, w=None, T=2, d=64, eps=1e-6, dtype=0, s=Q, y=None, y8=None, sc=None):
        return L.decomoe_add_rmsnorm_q8(x, res, w, T, d, eps, dtype, s, y, y8, sc, None)

    for kw in (dict(T=-1), dict(d=0), dict(eps=-1.0), dict(eps=float("nan")), dict(dtype=2), dict(x=None), dict(s=None),
               dict(y8=P), dict(sc=P), dict(y=Q), dict(d=60), dict(x=ctypes.c_void_p(0x1004)),
               dict(y8=ctypes.c_void_p(0x1004), sc=P)):
        assert norm(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
    assert norm(T=0) == dm.DECOMOE_OK

    def w4(x=P, xt=0, xs_=256, xs=None, T=2, K=256, w=P, ws=P, group=64, N=8, out=P, ot=0):
        return L.decomoe_w4_linear(x, xt, xs_, xs, T, K, w, ws, group, N, out, ot, None)

    for kw in (dict(xt=1), dict(xt=3), dict(ot=2), dict(group=16), dict(group=0), dict(T=-1), dict(K=0), dict(K=224),
               dict(N=0), dict(N=1 << 31), dict(K=1 << 27, xs_=1 << 27), dict(x=None), dict(w=None), dict(ws=None),
               dict(out=None), dict(xs=P), dict(xt=2), dict(xs_=248), dict(xs_=260), dict(x=ctypes.c_void_p(0x1008)),
               dict(w=ctypes.c_void_p(0x1008)), dict(ws=ctypes.c_void_p(0x1001)), dict(out=ctypes.c_void_p(0x1001))):
        assert w4(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
    assert w4(T=0, x=None, w=None, out=None) == dm.DECOMOE_OK


def test_tensors_are_refused_before_the_call():
    """The marshalling of tensors: host tensors, missing ones, other objects."""
    x, i = torch.zeros(2, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    pool = torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: dm.decomoe_add_rmsnorm_q8(x, None, None, x), lambda: dm.decomoe_w4_linear(x, x, x, x),
                 lambda: dm.decomoe_paged_append(pool[0, :2], pool[0, :2], i, pool, pool),
                 lambda: dm.decomoe_paged_plan(i, i, 16, i, i[None], i, i, i),
                 lambda: dm.decomoe_paged_attention(pool[0], pool, pool, i[:, None], i, pool[0], x)):
        with pytest.raises(ValueError, match="device tensors"):
            call()
    for call in (lambda: dm.decomoe_add_rmsnorm_q8(None, None, None, x), lambda: dm.decomoe_w4_linear([1], x, x, x),
                 lambda: dm.decomoe_paged_attention(None, pool, pool, i, i, x, x)):
        with pytest.raises((TypeError, ValueError)):
            call()


# ------------------------------------------------------------------ oracle pins

def test_oracle_plan_is_a_cache_kept_row_by_row():
    """Steps of random growth: every (request, position) keeps one slot for life,
    no slot belongs to two rows, pages are used in the order of the list."""
    r = np.random.default_rng(0)
    B, ps, width = 5, 4, 40
    free = r.permutation(200)
    table, head = np.full((B, width), -1), 3
    cached, where = np.zeros(B, int), {}
    for _ in range(12):
        fresh = r.integers(0, 9, B)
        table, lens, start, slots, pos, head, ok = O.paged_plan(cached, fresh, ps, free, head, table, int(fresh.sum()))
        assert ok and start[-1] == fresh.sum() and np.array_equal(lens, cached + fresh)
        for b in range(B):
            for k in range(fresh[b]):
                at = start[b] + k
                assert pos[at] == cached[b] + k
                where[(b, int(pos[at]))] = int(slots[at])
        cached = lens
    assert len(set(where.values())) == len(where) == cached.sum()
    for (b, p), s in where.items():
        assert s == table[b, p // ps] * ps + p % ps
    used = table[table >= 0]
    assert sorted(used) == sorted(free[3:head]) and len(used) == sum(-(-c // ps) for c in cached)


def test_oracle_paged_attention_is_attention_of_the_gathered_rows():
    r = np.random.default_rng(1)
    lens, ps, hq, hkv, d = [7, 0, 12], 4, 4, 2, 8
    kp, vp = r.standard_normal((2, 9, ps, hkv, d))
    table = r.permutation(9).reshape(3, 3)
    q = r.standard_normal((3, hq, d))
    out = O.paged_attention(q, kp, vp, table, lens, [2, 0, 0], [3, 0, 0])
    assert (out[1] == 0).all()
    for b, keep in ((0, [0, 1, 5, 6]), (2, list(range(12)))):
        k = np.array([kp[table[b, j // ps], j % ps] for j in keep])
        v = np.array([vp[table[b, j // ps], j % ps] for j in keep])
        kk, vv = (torch.from_numpy(np.repeat(t, hq // hkv, axis=1)).permute(1, 0, 2) for t in (k, v))
        ref = torch.softmax(torch.from_numpy(q[b])[:, None] @ kk.transpose(1, 2) / d ** 0.5, -1) @ vv
        assert np.allclose(out[b], ref[:, 0].numpy(), atol=1e-12)


def test_oracle_formats():
    v = O.e4m3_values()
    assert len(v) == 253 and v.max() == 448 and v[v > 0].min() == 2.0 ** -9
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    assert np.array_equal(np.unique(codes[torch.isfinite(codes)].double().numpy()), v)
    w = np.array([[0x80, 0xF7]], np.uint8)
    assert np.array_equal(O.w4_dequant(w, np.array([[0.5, 2.0]])), [[-4.0, 0.0, -2.0, 14.0]])
