"""Outputs over inputs of the paged cache's and the dense steps' calls are refused before
anything is launched, where blocks would read what others have written. No GPU: the
pointers are never followed."""
import ctypes

import pytest
import torch

import paper_2609_38823_gb300 as dm


# where there is a GPU, a call that were not refused would be launched
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="addresses of nothing stay off a GPU")


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()
    return dm.lib()


BASE, STEP = 1 << 40, 1 << 32


def _refused(call, name):
    assert call() == dm.DECOMOE_ERR_INVALID_ARG
    msg = dm.lib().decomoe_last_error()
    assert name.encode() in msg and b"overlap" in msg, msg


def _places(names):
    """A far apart address for each."""
    return {n: BASE + i * STEP for i, n in enumerate(names)}


def _call(f, args):
    return f(*[ctypes.c_void_p(a) if isinstance(a, int) and a >= BASE else a for a in args])


def test_attention():
    p = _places("q k v table lens hb hc out ws".split())
    need = dm.lib().decomoe_paged_attention_workspace_bytes(2, 8, 2, 64)
    kv = (8 * 16 * 2 * 64) * 2  # bytes of a pool
    row = 8 * 64 * 2

    def attend(**kw):
        a = p | kw
        return _call(dm.lib().decomoe_paged_attention,
                     (a["q"], 512, 2, a["k"], a["v"], 8, 16, 2048, a["table"], 4, a["lens"], a["hb"], a["hc"], 8, 2, 64, 0.0,
                      a["out"], a["ws"], need, None, None))

    for at in (p["q"], p["q"] + 2 * row - 16, p["q"] - 2 * row + 16, p["k"], p["k"] + kv - 16, p["v"] + 64, p["table"] + 16,
               p["lens"], p["hb"], p["hc"]):
        _refused(lambda: attend(out=at), "paged_attention")
    for at in (p["q"] + 16, p["q"] - need + 16, p["k"] + kv - 16, p["v"], p["table"], p["lens"], p["hb"], p["hc"], p["out"],
               p["out"] + 2 * row - 16):
        _refused(lambda: attend(ws=at), "paged_attention")


def test_w4_linear():
    p = _places("x xs w ws out".split())

    def w4(xt=0, **kw):
        a = p | kw
        return _call(dm.lib().decomoe_w4_linear, (a["x"], xt, 320, a["xs"] if xt else None, 3, 256, a["w"], a["ws"], 64, 40,
                                                  a["out"], 0, None))

    out = 3 * 40 * 2
    for at in (p["x"], p["x"] + (2 * 320 + 256) * 2 - 2, p["x"] - out + 2, p["w"], p["w"] + 40 * 128 - 2, p["ws"],
               p["ws"] + 40 * 4 * 2 - 2):
        _refused(lambda: w4(out=at), "w4_linear")
    for at in (p["x"] + 2 * 320 + 256 - 2, p["xs"], p["xs"] + 10):
        _refused(lambda: w4(xt=dm.DECOMOE_E4M3, out=at), "w4_linear")


def test_add_rmsnorm():
    p = _places("x res w sum y y8 sc".split())
    rows, d = 5, 64

    def norm(**kw):
        a = p | kw
        return _call(dm.lib().decomoe_add_rmsnorm_q8, (a["x"], a["res"], a["w"], rows, d, 1e-6, 0, a["sum"], a["y"], a["y8"],
                                                       a["sc"], None))

    n = rows * d * 2
    # shifted by a row, or onto the weight: another row's values would be read after they are written
    for out in ("sum", "y"):
        for at in (p["x"] + 2 * d, p["x"] - n + 16, p["res"] + 16, p["w"], p["y8"], p["sc"]):
            _refused(lambda: norm(**{out: at}), "add_rmsnorm_q8")
    for at in (p["x"], p["res"], p["w"], p["sum"], p["y"], p["y"] + n - 8, p["sc"]):
        _refused(lambda: norm(y8=at), "add_rmsnorm_q8")
    for at in (p["x"], p["res"] + 16, p["w"], p["sum"], p["y"]):
        _refused(lambda: norm(sc=at), "add_rmsnorm_q8")
    _refused(lambda: norm(sum=p["y"] + 16), "add_rmsnorm_q8")
    _refused(lambda: norm(sum=p["x"], y=p["x"] + 16), "add_rmsnorm_q8")


@pytest.mark.parametrize("step", [False, True])
def test_plan(step):
    names = "cached fresh free head table lens start slots pos out".split()
    p = _places(names)
    name = "paged_plan_step" if step else "paged_plan"

    def plan(**kw):
        a = p | kw
        tail = [a["lens"]] + ([] if step else [a["start"]]) + [a["slots"], a["pos"]] + ([] if step else [6])
        return _call(getattr(dm.lib(), "decomoe_" + name), [a["cached"], a["fresh"], 6, 16, a["free"], 9, a["head"], a["out"],
                                                            a["table"], 4] + tail + [None, None])

    outs = [n for n in ("table", "lens", "start", "slots", "pos", "out") if not (step and n == "start")]
    for o in outs:
        for other in ["cached", "fresh", "free", "head"] + [n for n in outs if n != o]:
            _refused(lambda: plan(**{o: p[other]}), name)
    _refused(lambda: plan(slots=p["table"] + 4 * (6 * 4 - 1)), name)
    _refused(lambda: plan(free=p["table"] - 4 * 8), name)


def test_advance():
    p = _places("cached lens table head out".split())

    def advance(**kw):
        a = p | kw
        return _call(dm.lib().decomoe_paged_advance, (a["cached"], a["lens"], a["table"], 6, 4, 16, a["head"], a["out"], None))

    for kw in (dict(cached=p["lens"]), dict(cached=p["table"] + 4 * 23), dict(head=p["cached"]), dict(head=p["lens"] + 20),
               dict(head=p["table"])):
        _refused(lambda: advance(**kw), "paged_advance")
