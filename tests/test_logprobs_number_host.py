"""decomoe_token_logprobs: without alternatives their number does not matter (no GPU: what is
refused, and what has nothing to do)."""
import ctypes

import pytest

import paper_2609_38823_gb300 as dm


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()


def _call(n, ids=None, top=None, T=0, V=3):
    p = lambda a: None if a is None else ctypes.c_void_p(a)  # noqa: E731
    return dm.lib().decomoe_token_logprobs(None, T, V, V, dm.DECOMOE_F32, p(1 << 40), 1.0, n, p(2 << 40), None, p(ids), p(top), None, None)


@pytest.mark.parametrize("n", [0, 1, 4, 33, 64, -1, 2 ** 31 - 1])
def test_a_number_of_alternatives_that_nobody_wants(n):
    assert _call(n) == dm.DECOMOE_OK


@pytest.mark.parametrize("n", [0, -1, 4, 33])
def test_a_number_that_is_wanted_is_checked(n):
    for kw in (dict(ids=3 << 40), dict(top=3 << 40), dict(ids=3 << 40, top=4 << 40)):
        assert _call(n, **kw) == dm.DECOMOE_ERR_INVALID_ARG
        assert b"alternatives" in dm.lib().decomoe_last_error()
    assert _call(n, ids=3 << 40, V=100) == (dm.DECOMOE_OK if n == 4 else dm.DECOMOE_ERR_INVALID_ARG)
