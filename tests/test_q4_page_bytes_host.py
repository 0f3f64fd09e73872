"""decomoe_paged_q4_page_bytes: 0 for what no call on such pages takes."""
import pytest

import paper_2609_38823_gb300 as dm
from paper_2609_38823_gb300.decode import PagedCache


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()


@pytest.mark.parametrize("d,group", [(64, 32), (128, 128)])
def test_more_heads_than_any_call_takes(d, group):
    assert dm.decomoe_paged_q4_page_bytes(8, 1024, d, group) == 1024 * 16 * (d // 2 + 4 * d // group)
    for ps in (8, 1 << 30):
        for hkv in (1025, 1 << 20, 2 ** 31 - 1):  # (2^31 heads of 2^27 tiles: above 64 bits)
            assert dm.decomoe_paged_q4_page_bytes(ps, hkv, d, group) == 0
    with pytest.raises(ValueError, match="heads"):
        PagedCache(1, 1, pages=1, page_size=8, max_pages=1, hkv=1025, d=d, bits=4, group=group, device="cpu")
