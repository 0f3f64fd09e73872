"""The attentions over paged caches called by several host threads at once, with batches of
different sizes: what one call sets for its launch is enough for the other's."""
import ctypes
import threading
import time

import pytest
import torch

import paper_2609_38823_gb300 as dm

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


@pytest.mark.parametrize("bits", [4, 16])
def test_threads_with_batches_of_different_sizes(bits):
    """Requests without rows, so that a call is little more than its launch; a foreign call lets other threads run."""
    hq, hkv, d, ps = 8, 2, 64, 16
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    pool = torch.zeros(2, hkv, ps // 8, 576, dtype=torch.uint8, device=DEV)
    kv = torch.zeros(2, 2, ps, hkv, d, dtype=torch.bfloat16, device=DEV)
    size = dm.decomoe_paged_attention_q4_workspace_bytes if bits == 4 else dm.decomoe_paged_attention_workspace_bytes
    batches = (4096, 1, 1, 4096, 1, 1)
    seen, start = {}, threading.Barrier(len(batches))

    def work(i, B):
        q = torch.zeros(B, hq, d, dtype=torch.bfloat16, device=DEV)
        out, table = torch.full_like(q, 7.0), torch.zeros(B, 1, dtype=I32, device=DEV)
        lens, need = torch.zeros(B, dtype=I32, device=DEV), size(B, hq, hkv, d)
        ws = dm.workspace(need, DEV)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        rest = [hq, hkv, d, 0.0, p(out), p(ws), need, None, stream.cuda_stream]
        if bits == 4:
            call, args = dm.lib().decomoe_paged_attention_q4, [p(q), hq * d, B, p(pool), 2, ps, pool[0].numel(), 64]
        else:
            call, args = dm.lib().decomoe_paged_attention, [p(q), hq * d, B, p(kv[0]), p(kv[1]), 2, ps, kv[0, 0].numel()]
        args += [p(table), 1, p(lens), None, None] + rest
        codes = set()
        start.wait()
        end = time.monotonic() + 3
        while time.monotonic() < end:
            for _ in range(50):
                codes.add(call(*args))
        stream.synchronize()
        seen[i] = codes, bool((out == 0).all())

    threads = [threading.Thread(target=work, args=a) for a in enumerate(batches)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert seen == {i: ({dm.DECOMOE_OK}, True) for i in range(len(batches))}, seen
