"""Host-side checks of the calls on a cache in 4 bits and of the token log
probabilities that need no GPU (refusals before anything is launched), and pins of their
oracle against other routes."""
import ctypes
from unittest import mock

import numpy as np
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()
    return dm.lib()


# where there is a GPU, a call that were not refused would be launched
off_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses of nothing stay off a GPU")
BASE, STEP = 1 << 40, 1 << 32
BF16, I32, U8 = torch.bfloat16, torch.int32, torch.uint8


def _places(names):
    return {n: BASE + i * STEP for i, n in enumerate(names.split())}


def _p(a):
    return None if a is None else ctypes.c_void_p(a)


R = _places("k v slots pages status")


def _rows_call(read, N=4, ks=512, vs=512, hkv=4, d=128, group=64, pages=8, ps=16, stride=4 * 2 * 1152, **kw):
    a = R | kw
    if read:
        return dm.lib().decomoe_paged_read_q4(_p(a["slots"]), N, _p(a["pages"]), pages, ps, stride, hkv, d, group, _p(a["k"]), ks,
                                              _p(a["v"]), vs, None, None)
    return dm.lib().decomoe_paged_append_q4(_p(a["k"]), ks, _p(a["v"]), vs, N, hkv, d, group, _p(a["slots"]), _p(a["pages"]), pages,
                                            ps, stride, None, None)


@off_gpu
@pytest.mark.parametrize("read", [False, True])
def test_append_and_read_arguments(read):
    name = b"paged_read_q4" if read else b"paged_append_q4"
    for kw in (dict(N=-1), dict(N=1 << 31), dict(hkv=0), dict(hkv=1025), dict(d=96), dict(d=64, group=128), dict(group=16),
               dict(group=0), dict(ps=4), dict(ps=24), dict(ps=-16), dict(pages=-1), dict(pages=1 << 28), dict(stride=4 * 2 * 1152 - 16),
               dict(stride=4 * 2 * 1152 + 8), dict(ks=504), dict(vs=511), dict(ks=516), dict(k=None), dict(v=None), dict(slots=None),
               dict(pages=8, **{"k": R["k"] + 8}), dict(v=R["v"] + 2)):
        assert _rows_call(read, **kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
        assert name in dm.lib().decomoe_last_error(), kw
    pool = 7 * 4 * 2 * 1152 + 4 * 2 * 1152
    rows = (3 * 512 + 512) * 2
    # (read: the slots and the pool are both inputs)
    for kw in [dict(k=R["pages"]), dict(v=R["pages"] + pool - 16), dict(k=R["pages"] - rows + 16)] + [dict(slots=R["pages"] + 4)] * (not read):
        assert _rows_call(read, **kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
        assert name in dm.lib().decomoe_last_error() and b"overlap" in dm.lib().decomoe_last_error()
    if read:
        # one output over the other, or over the slots; side by side in rows of 1024 they lie apart
        for kw in (dict(v=R["k"]), dict(v=R["k"] + 1024), dict(v=R["k"] + 512, ks=1024, vs=1024), dict(slots=R["k"] + 16),
                   dict(v=R["k"] + 1024, ks=1016, vs=1016), dict(v=R["k"] + 1024, ks=1024, vs=1032)):
            assert _rows_call(read, **kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
            assert b"overlap" in dm.lib().decomoe_last_error()
    assert _rows_call(read, N=0, k=None, v=None, slots=None) == dm.DECOMOE_OK


@off_gpu
def test_attention_arguments():
    p = _places("q pages table lens hb hc out ws")

    def attend(qs=4096, B=2, num=8, ps=16, stride=4 * 2 * 1152, group=64, max_pages=4, hq=32, hkv=4, d=128, ws_bytes=1 << 30,
               hide=False, **kw):
        a = p | kw
        return dm.lib().decomoe_paged_attention_q4(_p(a["q"]), qs, B, _p(a["pages"]), num, ps, stride, group, _p(a["table"]),
                                                   max_pages, _p(a["lens"]), _p(a["hb"]) if hide or "hb" in kw else None,
                                                   _p(a["hc"]) if hide or "hc" in kw else None, hq, hkv, d, 0.0, _p(a["out"]),
                                                   _p(a["ws"]), ws_bytes, None, None)

    for kw in (dict(B=-1), dict(B=4097), dict(d=96), dict(d=64, group=128), dict(group=48), dict(hq=30), dict(hkv=0), dict(hq=2),
               dict(hq=1028), dict(ps=4), dict(ps=10), dict(num=-1), dict(num=1 << 28), dict(max_pages=-1), dict(max_pages=1 << 28),
               dict(stride=4 * 2 * 1152 - 16), dict(stride=4 * 2 * 1152 + 8), dict(qs=4088), dict(qs=4100), dict(hb=BASE), dict(hc=BASE),
               dict(q=None), dict(lens=None), dict(out=None), dict(table=None), dict(pages=None), dict(out=p["out"] + 4),
               dict(ws=p["ws"] + 8), dict(q=p["q"] + 2), dict(B=4000, max_pages=1 << 20)):
        assert attend(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
        assert b"paged_attention_q4" in dm.lib().decomoe_last_error(), kw
    for kw in (dict(ws=None), dict(ws_bytes=100)):
        assert attend(**kw) == dm.DECOMOE_ERR_WORKSPACE, kw
    assert attend(B=0, q=None, lens=None, out=None) == dm.DECOMOE_OK
    need = dm.decomoe_paged_attention_q4_workspace_bytes(2, 32, 4, 128)
    for o in ("out", "ws"):
        for other in ("q", "pages", "table", "lens", "hb", "hc", "out" if o == "ws" else "ws"):
            assert attend(hide=True, **{o: p[other]}) == dm.DECOMOE_ERR_INVALID_ARG, (o, other)
            assert b"overlap" in dm.lib().decomoe_last_error()
    assert attend(ws=p["out"] - need + 16) == dm.DECOMOE_ERR_INVALID_ARG
    assert dm.decomoe_paged_attention_q4_workspace_bytes(0, 32, 4, 128) == 0


@off_gpu
def test_logprobs_arguments():
    p = _places("x tokens lp ent ids top")

    def call(T=3, V=100, ld=104, dtype=0, scale=1.0, n=5, **kw):
        a = p | kw
        return dm.lib().decomoe_token_logprobs(_p(a["x"]), T, V, ld, dtype, _p(a["tokens"]), scale, n, _p(a["lp"]), _p(a["ent"]),
                                               _p(a["ids"]), _p(a["top"]), None, None)

    for kw in (dict(T=-1), dict(T=1 << 27), dict(V=0), dict(V=(1 << 24) + 1, ld=1 << 25), dict(ld=99), dict(dtype=2), dict(scale=0.0),
               dict(scale=-2.0), dict(scale=float("inf")), dict(scale=float("nan")), dict(n=-1), dict(n=33), dict(n=4, V=3),
               dict(n=0), dict(tokens=None), dict(x=None), dict(x=p["x"] + 1), dict(dtype=1, x=p["x"] + 2)):
        assert call(**kw) == dm.DECOMOE_ERR_INVALID_ARG, kw
        assert b"token_logprobs" in dm.lib().decomoe_last_error(), kw
    for o in ("lp", "ent", "ids", "top"):
        for other in ("x", "tokens", "lp", "ent", "ids", "top"):
            if o != other:
                assert call(**{o: p[other]}) == dm.DECOMOE_ERR_INVALID_ARG, (o, other)
                assert b"overlap" in dm.lib().decomoe_last_error()
    assert call(top=p["x"] + (2 * 104 + 100) * 2 - 4) == dm.DECOMOE_ERR_INVALID_ARG
    assert call(T=0, x=None) == dm.DECOMOE_OK


@off_gpu
def test_pages_whose_size_passes_32_bits():
    """1024 heads of 2^27 tiles: 2^37 tiles a page, which no stride given here holds."""
    for ps in (1 << 25, 1 << 30):
        for read in (False, True):
            assert _rows_call(read, hkv=1024, ks=1 << 17, vs=1 << 17, pages=1, ps=ps, stride=1 << 31) == dm.DECOMOE_ERR_INVALID_ARG
            assert b"page_stride" in dm.lib().decomoe_last_error()
        p = [_p(a) for a in _places("q pages table lens out ws").values()]
        assert dm.lib().decomoe_paged_attention_q4(p[0], 1 << 17, 1, p[1], 1, ps, 1 << 31, 64, p[2], 1, p[3], None, None, 1024, 1024,
                                                   128, 0.0, p[4], p[5], 1 << 31, None, None) == dm.DECOMOE_ERR_INVALID_ARG
        assert b"page_stride" in dm.lib().decomoe_last_error()
    assert dm.decomoe_paged_q4_page_bytes(1 << 30, 1024, 128, 64) == 1152 << 37


def test_page_bytes():
    assert dm.decomoe_paged_q4_page_bytes(16, 4, 128, 64) == 4 * 2 * 1152
    assert dm.decomoe_paged_q4_page_bytes(8, 1, 64, 32) == 640
    for bad in ((4, 1, 64, 32), (12, 1, 64, 32), (16, 0, 64, 32), (16, 1, 96, 32), (16, 1, 64, 128), (16, 1, 128, 16)):
        assert dm.decomoe_paged_q4_page_bytes(*bad) == 0


def _fake_calls(dev):
    made = iter(range(100))

    def t(*shape, dtype=I32):
        return torch.empty(*shape, dtype=dtype, device=dev(next(made)))

    with mock.patch.object(torch.cuda, "is_available", lambda: False), FakeTensorMode():
        pool, rows = t(3, 2, 2, 640, dtype=U8), [t(2, 2, 64, dtype=BF16) for _ in range(2)]
        return {
            "append": lambda c=rows + [t(2), pool]: dm.decomoe_paged_append_q4(*c),
            "read": lambda c=[t(2), pool] + rows: dm.decomoe_paged_read_q4(*c),
            "attention": lambda c=[t(2, 4, 64, dtype=BF16), pool, t(2, 3), t(2), t(2, 4, 64, dtype=BF16), t(1 << 24, dtype=U8)]:
                dm.decomoe_paged_attention_q4(*c),
            "logprobs": lambda c=[t(2, 64, dtype=BF16), t(2), t(2, dtype=torch.float32)]: dm.decomoe_token_logprobs(*c),
        }


NAMES = ["append", "read", "attention", "logprobs"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dev", [lambda i: f"cuda:{i % 2}", lambda i: f"cuda:{1 - i % 2}"])
def test_two_devices(name, dev):
    with pytest.raises(ValueError, match="one device"):
        _fake_calls(dev)[name]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_another_device_than_the_current_one(name):
    assert torch.cuda.current_device() == 0
    with pytest.raises(ValueError, match="current device"):
        _fake_calls(lambda i: "cuda:1")[name]()


def test_host_tensors_are_refused():
    x = torch.zeros(2, 2, 64, dtype=BF16)
    with pytest.raises(ValueError):
        dm.decomoe_paged_append_q4(x, x, torch.zeros(2, dtype=I32), torch.zeros(1, 2, 1, 640, dtype=U8))
    with pytest.raises(ValueError):
        dm.decomoe_token_logprobs(torch.zeros(2, 9), None, entropy=torch.zeros(2))


# ------------------------------------------------------------------ the oracle

def test_oracle_bf16_is_torchs_rounding():
    x = torch.randn(4000, generator=torch.Generator().manual_seed(0)) * 2.0 ** torch.arange(-60, 60).repeat_interleave(34)[:4000]
    assert np.array_equal(O.bf16(x.double().numpy()), x.to(BF16).double().numpy())


@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_oracle_codes_are_the_nearest_and_survive_the_layout(d, group):
    x = (torch.randn(8, d, generator=torch.Generator().manual_seed(d + group)) * 3).to(BF16).double().numpy()
    q, step, low = O.q4_quantise(x, group)
    assert q.min() == 0 and q.max() == 15
    s, lo = np.repeat(step, group, 1), np.repeat(low, group, 1)
    mine = np.abs(lo + s * q - x)
    for c in range(16):  # no other code is nearer
        assert (mine <= np.abs(lo + s * c - x) + 1e-12).all()
    k, v = O.q4_rows_to_tile(q, step, low, False), O.q4_rows_to_tile(15 - q, step, low, True)
    keys, values, span, wide = O.q4_values(np.concatenate([k, v])[None, None, None], d, group)
    assert np.array_equal(keys[0, :, 0], lo + s * q) and np.array_equal(values[0, :, 0], lo + s * (15 - q))
    assert np.array_equal(wide[0, :, 0], s * (15 - q)) and np.array_equal(span[0, :, 0], s * q)
    # the places by hand: feature 32 i + 8 c + j of a key, 32 i + 4 r + j of a value
    f = 32 + 8 * 2 + 5
    byte = 4 * (2 * (d // 32) + 1) + 5 // 2
    assert k[byte] >> 4 == q[0, f]
    f = 32 + 4 * 6 + 2
    byte = 2 * (6 * (d // 32) + 1) + 1
    assert v[byte] & 15 == 15 - q[0, f]


def test_oracle_logprobs_against_torch():
    x = torch.randn(5, 300, generator=torch.Generator().manual_seed(4), dtype=torch.float64) * 3
    x[1, 10:] = -torch.inf
    tokens = [3, 5, 299, 0, 17]
    lp, ent, ids, top = O.token_logprobs(x.numpy(), tokens, 7, 0.5)
    ref = torch.log_softmax(0.5 * x, -1)
    assert np.allclose(lp, ref[range(5), tokens].numpy(), rtol=1e-12)
    assert np.allclose(ent, torch.special.entr(ref.exp()).sum(-1).numpy(), rtol=1e-12)
    best, at = torch.sort(ref, descending=True, stable=True)
    assert np.array_equal(ids, at[:, :7].numpy()) and np.allclose(top, best[:, :7].numpy(), rtol=1e-12)
    lp, ent, ids, top = O.token_logprobs(np.array([[-np.inf] * 3, [0.0, np.nan, 1.0], [np.inf, 0.0, 1.0]]), [1, 0, 0], 2)
    assert np.isneginf(lp[0]) and ent[0] == 0 and np.isnan(lp[1:]).all() and ids.tolist() == [[0, 1], [2, 0], [0, 2]]
