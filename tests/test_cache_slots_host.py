"""PagedCache on the host: the slots of a request's rows, without those that a layer hides, and
what has no slot refused."""
import pytest
import torch

from paper_2609_38823_gb300.decode import PagedCache

PS = 8


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()


def _cache(layers=3):
    c = PagedCache(layers, 2, pages=20, page_size=PS, max_pages=5, hkv=2, d=64, bits=4, group=32, device="cpu")
    c.table[0, :4] = torch.tensor([7, 2, 19, 0], dtype=torch.int32)
    c.table[1, :2] = torch.tensor([3, 4], dtype=torch.int32)
    return c


def _slot(c, request, j):
    return int(c.table[request, j // PS]) * PS + j % PS


@pytest.mark.parametrize("rows", [0, 1, 8, 9, 31, 32])
def test_slots_of_a_request_with_nothing_hidden(rows):
    c = _cache()
    for layer in (None, 0, 2):
        s = c.slots_of(0, rows) if layer is None else c.slots_of(0, rows, layer)
        assert s.dtype == torch.int32 and s.is_contiguous() and s.tolist() == [_slot(c, 0, j) for j in range(rows)]


@pytest.mark.parametrize("rows", [5, 12, 20, 30])
def test_hidden_rows_are_left_out_from_their_layer_on(rows):
    c = _cache()
    c.hide(0, 6, 15, from_layer=1)
    c.table[0, 1] = -1  # a page that holds only hidden rows was given back
    for layer in (1, 2):
        assert c.slots_of(0, rows, layer).tolist() == [_slot(c, 0, j) for j in range(rows) if not 6 <= j < 21]
    if rows > 8:  # layer 0 still sees the rows of that page
        with pytest.raises(ValueError, match="page"):
            c.slots_of(0, rows, 0)
    if rows > 6:  # which layer's?
        with pytest.raises(ValueError, match="layer"):
            c.slots_of(0, rows)
    assert c.slots_of(0, 6).tolist() == c.slots_of(0, 6, 2).tolist() == [_slot(c, 0, j) for j in range(6)]
    assert c.slots_of(1, 16, 2).tolist() == [_slot(c, 1, j) for j in range(16)]  # another request


def test_hidden_blocks_past_the_ends_are_cut():
    c = _cache()
    c.hide(0, 25, 100, from_layer=0)
    assert c.slots_of(0, 30, 0).tolist() == [_slot(c, 0, j) for j in range(25)]
    c.hide(0, -3, 5, from_layer=0)  # a negative begin is 0, as the attention reads it
    assert c.slots_of(0, 30, 1).tolist() == [_slot(c, 0, j) for j in range(5, 30)]
    c.hide(0, 4, -2, from_layer=0)
    assert c.slots_of(0, 30, 1).tolist() == [_slot(c, 0, j) for j in range(30)]


def test_rows_without_a_page_are_refused():
    c = _cache()
    for request, rows in ((0, 33), (1, 17), (0, 40)):
        with pytest.raises(ValueError, match="page"):
            c.slots_of(request, rows)
    for rows in (41, 1 << 40, -1):  # more than a request can have
        with pytest.raises(ValueError, match="rows"):
            c.slots_of(0, rows)
    for page in (20, 2 ** 31 - 1, 2 ** 29):  # outside the pool
        c.table[0, 2] = page
        assert c.slots_of(0, 16).tolist() == [_slot(c, 0, j) for j in range(16)]
        with pytest.raises(ValueError, match="page"):
            c.slots_of(0, 17)


def test_a_cache_in_4_bits_has_no_bf16_pools():
    c = _cache()
    for f in (c.k, c.v):
        with pytest.raises(ValueError, match="4 bits"):
            f(0)
    b = PagedCache(2, 1, pages=3, page_size=PS, max_pages=2, hkv=2, d=64, device="cpu")
    assert b.k(1).shape == b.v(1).shape == (3, PS, 2, 64) and b.k(1).data_ptr() != b.v(1).data_ptr()
