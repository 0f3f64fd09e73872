"""A decode step of several requests through layers on a paged cache
(paper_2609_38823_gb300/decode.py): every step's result against the oracle on the
step's own inputs, growth over page ends, a hidden visual block, and the captured
step against the eager one."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from paper_2609_38823_gb300.decode import DecodeLayer, DecodeStep, PagedCache, quantize_w4
from tests.helpers import BF16_MAX_ABS, BF16_REL_L2, assert_close_out, f64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
D_MODEL, E, K, M, HQ, HKV, D, L = 256, 16, 4, 128, 8, 2, 64, 3


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _model(seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).to(DEV)  # noqa: E731
    layers, dense = [], []
    for _ in range(L):
        wg, wu, wd = n(E, M, D_MODEL, std=0.06), n(E, M, D_MODEL, std=0.06), n(E, D_MODEL, M, std=0.06)
        qkv, out = n((HQ + 2 * HKV) * D, D_MODEL, std=0.06), n(D_MODEL, HQ * D, std=0.05)
        # a prefix of k experts: the choice is the whole prefix, so that no near tie decides anything
        layers.append(DecodeLayer(1 + n(D_MODEL, std=0.1), quantize_w4(qkv), quantize_w4(out, 64), None, n(E, D_MODEL, std=0.05),
                                  torch.zeros(E, device=DEV), dm.fuse_gate_up(wg, wu), wd, K))
        dense.append((f64(wg), f64(wu), f64(wd)))
    return layers, dense


def _prompt(cache, lens, seed):
    """Prompts of the given lengths stored in every layer: the rows kept on the host."""
    g = torch.Generator().manual_seed(seed)
    n = sum(lens)
    slots = torch.empty(n, dtype=torch.int32, device=DEV)
    cache.plan(torch.tensor(lens, dtype=torch.int32, device=DEV), slots)
    held = []
    for l in range(L):
        k, v = (torch.randn(n, HKV, D, generator=g).to(torch.bfloat16) for _ in range(2))
        dm.decomoe_paged_append(k.to(DEV), v.to(DEV), slots, cache.k(l), cache.v(l), status=cache.status)
        at = np.cumsum([0] + lens)
        held.append([[list(k[at[b]:at[b + 1]]), list(v[at[b]:at[b + 1]])] for b in range(len(lens))])
    cache.advance()
    return held


def test_decode_steps_against_the_oracle():
    layers, dense = _model()
    lens, hidden = [5, 47, 130], {2: (16, 100)}  # request 2: its visual block hidden from layer 1 on
    cache = PagedCache(L, len(lens), pages=60, page_size=8, max_pages=24, hkv=HKV, d=D)
    held = _prompt(cache, lens, 1)
    cache.hide(2, *hidden[2], from_layer=1)
    step = DecodeStep(layers, cache, len(lens), HQ, K)
    g = torch.Generator().manual_seed(2)

    def check(l, s, h_in, h_out):
        torch.cuda.synchronize()
        w = layers[l]
        x = f64(h_in)
        v = O.rmsnorm(x, 1e-6, f64(w.norm_attn))
        q8 = s.x8.float().double().cpu().numpy() * s.x8_scale.double().cpu().numpy()[:, None]
        # e4m3 keeps 4 bits: at most 2^-4 of a value, and a step of 2^-9 of the row's scale
        assert (np.abs(q8 - v) <= 2.0 ** -4 * 1.01 * np.abs(v) + 2.0 ** -9 * s.x8_scale.double().cpu().numpy()[:, None]).all()
        qkv = q8 @ O.w4_dequant(w.w_qkv[0].cpu().numpy(), f64(w.w_qkv[1])).T
        assert_close_out(f64(s.qkv).reshape(len(lens), -1), qkv, BF16_REL_L2, BF16_MAX_ABS, f"layer {l} qkv")
        for b in range(len(lens)):
            held[l][b][0].append(s.k_new[b].cpu())
            held[l][b][1].append(s.v_new[b].cpu())
            k, vv = (f64(torch.stack(held[l][b][i])) for i in (0, 1))
            if b in hidden and l >= 1:
                h0, n = hidden[b]
                k, vv = np.delete(k, slice(h0, h0 + n), 0), np.delete(vv, slice(h0, h0 + n), 0)
            ref = O.attention(f64(s.q[b:b + 1]), k, vv)[0]
            assert_close_out(f64(s.heads[b]), ref, 2 * BF16_REL_L2, 2 * BF16_MAX_ABS, f"layer {l} request {b} attention")
        proj = f64(s.heads).reshape(len(lens), -1) @ O.w4_dequant(w.w_out[0].cpu().numpy(), f64(w.w_out[1])).T
        assert_close_out(f64(s.proj), proj, BF16_REL_L2, BF16_MAX_ABS, f"layer {l} projection")
        h1 = f64(s.proj) + x
        assert_close_out(f64(s.h1), h1, BF16_REL_L2, BF16_MAX_ABS, f"layer {l} residual")
        assert_close_out(f64(s.xn), O.rmsnorm(h1), BF16_REL_L2, BF16_MAX_ABS, f"layer {l} norm")
        ref = O.moe_layer(f64(s.xn), f64(w.w_r), np.zeros(E), *dense[l], k=K, K=K, residual=f64(s.h1))
        assert_close_out(f64(h_out), ref["out"], BF16_REL_L2, BF16_MAX_ABS, f"layer {l} output")

    for _ in range(10):  # request 0 passes a page's end on the way
        step(torch.randn(len(lens), D_MODEL, generator=g).to(torch.bfloat16).to(DEV), trace=check)
        cache.advance()
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK
    assert cache.cached.tolist() == [n + 10 for n in lens]


def test_captured_step_equals_the_eager_one():
    layers, _ = _model(3)
    lens = [3, 20, 9, 64]
    runs = []
    for graph in (False, True):
        cache = PagedCache(L, len(lens), pages=60, page_size=8, max_pages=24, hkv=HKV, d=D)
        _prompt(cache, lens, 5)
        step = DecodeStep(layers, cache, len(lens), HQ, K)
        g = torch.Generator().manual_seed(7)
        h0 = torch.zeros(len(lens), D_MODEL, dtype=torch.bfloat16, device=DEV)
        out = []
        replay = dm.capture_graph(lambda: out.append(step(h0))) if graph else None
        got = []
        for _ in range(8):
            h0.copy_(torch.randn(len(lens), D_MODEL, generator=g).to(torch.bfloat16))
            if graph:
                replay.replay()
                got.append(out[-1].clone())
            else:
                got.append(step(h0).clone())
            cache.advance()
        torch.cuda.synchronize()
        assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK
        runs.append(torch.stack(got))
    assert torch.equal(runs[0], runs[1])


def test_rotate_sees_the_rows_positions():
    layers, _ = _model(4)
    cache = PagedCache(L, 2, pages=20, page_size=8, max_pages=8, hkv=HKV, d=D)
    _prompt(cache, [6, 11], 1)
    seen = []
    step = DecodeStep(layers, cache, 2, HQ, K, rotate=lambda q, k, pos: seen.append((q.shape, k.shape, pos.tolist())))
    h0 = torch.randn(2, D_MODEL, device=DEV).to(torch.bfloat16)
    step(h0)
    cache.advance()
    step(h0)
    assert [s[2] for s in seen] == [[6, 11]] * L + [[7, 12]] * L and seen[0][:2] == ((2, HQ, D), (2, HKV, D))


def test_quantize_w4():
    g = torch.Generator().manual_seed(0)
    w = torch.randn(10, 256, generator=g) * 0.1
    w[3, :64] = 0
    b, s = quantize_w4(w, 64)
    got = O.w4_dequant(b.numpy(), s.double().numpy())
    # half a step of 1/7 of the group's largest value; the scale itself rounded to 8 bits
    top = w.view(10, 4, 64).abs().amax(-1).repeat_interleave(64, 1).double().numpy()
    assert (np.abs(got - w.double().numpy()) <= top * (0.5 / 7 + 2.0 ** -8) + 1e-12).all() and (got[3, :64] == 0).all()


def test_pages_of_finished_requests_are_given_out_again():
    cache = PagedCache(L, 3, pages=30, page_size=8, max_pages=12, hkv=HKV, d=D)
    lens = [40, 17, 64]
    _prompt(cache, lens, 1)
    first = [set(cache.table[b][cache.table[b] >= 0].tolist()) for b in range(3)]
    assert [len(p) for p in first] == [5, 3, 8]
    cache.hide(2, 4, 10, from_layer=0)
    cache.release(2)
    cache.release(0)
    assert cache.cached.tolist() == [0, 17, 0] and int(cache.head) == 3 and int(cache.hide_count.sum()) == 0
    slots = torch.empty(95, dtype=torch.int32, device=DEV)
    cache.plan(torch.tensor([95, 0, 0], dtype=torch.int32, device=DEV), slots)
    cache.advance()
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK
    again = set(cache.table[0][cache.table[0] >= 0].tolist())
    assert len(again) == 12 and not again & first[1] and first[0] | first[2] > again - set(range(16, 30))
    assert len(set(slots.tolist())) == 95
    with pytest.raises(ValueError):
        cache.head.zero_()
        cache.release(0)
