"""A prompt's chunk on a cache in 4 bits whose request hides a block: what one token's attention
leaves out, the chunk's does too; rows without a slot are marked."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from paper_2609_38823_gb300.decode import PagedCache
from tests.helpers import BF16_MAX_ABS, BF16_REL_L2, assert_close_out, f64
from tests.test_gpu_paged_q4 import DEV, I32, _i32, _rows

pytestmark = pytest.mark.gpu
HQ, HKV, D, GROUP, PS, N1, N2 = 8, 2, 128, 64, 16, 90, 37


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _cache():
    """Two layers, the request 1 of 127 rows in two chunks."""
    cache = PagedCache(2, 2, pages=20, page_size=PS, max_pages=12, hkv=HKV, d=D, bits=4, group=GROUP)
    for i, n in enumerate((N1, N2)):
        slots = torch.empty(n, dtype=I32, device=DEV)
        cache.plan(_i32([0, n]), slots)
        for layer in range(2):
            cache.append(layer, _rows(n, HKV, D, 10 * layer + i).to(DEV), _rows(n, HKV, D, 50 + 10 * layer + i).to(DEV), slots)
        cache.advance()
    return cache


@pytest.mark.parametrize("begin,count", [(10, 60), (0, 33), (16, 64), (89, 1)])
def test_chunk_leaves_the_hidden_block_out(begin, count):
    cache = _cache()
    flat = [x.reshape(-1, HKV, D) for x in O.q4_values(cache.pool[1].cpu().numpy(), D, GROUP)[:2]]
    at = cache.slots_of(1, N1 + N2, 1).cpu().numpy()
    keep = [j for j in range(N1 + N2) if not begin <= j < begin + count]
    cache.hide(1, begin, count, from_layer=1)
    for page in range(12):  # pages that hold only hidden rows are given back
        if begin <= page * PS and (page + 1) * PS <= begin + count:
            cache.table[1, page] = -1
    slots = cache.slots_of(1, N1 + N2, 1)
    assert np.array_equal(slots.cpu().numpy(), at[keep])
    C = len(keep)
    q = _rows(N2, HQ, D, 3).to(DEV)
    out = torch.empty_like(q)
    k, v = (torch.full((C, HKV, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    cache.attend_chunk(1, q, slots, k, v, out, dm.workspace(dm.decomoe_attention_workspace_bytes(N2, C, HQ, HKV, D), DEV))
    assert np.array_equal(f64(k), O.bf16(flat[0][at[keep]])) and np.array_equal(f64(v), O.bf16(flat[1][at[keep]]))
    ref = O.attention(f64(q), f64(k), f64(v))
    assert_close_out(f64(out), ref, BF16_REL_L2, BF16_MAX_ABS, "chunk")
    # the last row by the call of a single token
    one = torch.empty(2, HQ, D, dtype=torch.bfloat16, device=DEV)
    cache.attend(1, torch.stack([q[0], q[-1]]), one, dm.workspace(cache.workspace_bytes(2, HQ), DEV))
    assert_close_out(f64(one[1]), O.attention(f64(q[-1:]), flat[0][at[keep]], flat[1][at[keep]])[0], BF16_REL_L2, BF16_MAX_ABS, "one")
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_OK


@pytest.mark.parametrize("bad", [-1, -2, 20 * PS])
def test_chunk_marks_rows_without_a_slot(bad):
    cache = _cache()
    C = N1 + N2
    slots = cache.slots_of(1, C)
    slots[40] = bad
    q = _rows(N2, HQ, D, 3).to(DEV)
    k, v = (torch.zeros(C, HKV, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = dm.workspace(dm.decomoe_attention_workspace_bytes(N2, C, HQ, HKV, D), DEV)
    cache.attend_chunk(0, q, slots, k, v, torch.empty_like(q), ws)
    assert dm.decomoe_read_status(cache.status) == dm.DECOMOE_ERR_BAD_INPUT
    assert slots[40] == bad  # the caller's slots are left as they were
