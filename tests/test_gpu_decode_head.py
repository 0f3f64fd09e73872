"""DecodeHead: tokens outside the vocabulary are marked in its status word."""
import numpy as np
import pytest
import torch

import paper_2609_38823_gb300 as dm
from oracle import decomoe_oracle as O
from paper_2609_38823_gb300.decode import DecodeHead, quantize_w4
from tests.helpers import f64

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
I32 = torch.int32
V, C, B = 333, 256, 4


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__

    __graft_entry__.build()
    dm.lib()


def _head(**kw):
    g = torch.Generator().manual_seed(2)
    head = DecodeHead(None, quantize_w4(torch.randn(V, C, generator=g).to(DEV)), B, n=3, **kw)
    return head, torch.randn(B, C, generator=g).to(torch.bfloat16).to(DEV)


@pytest.mark.parametrize("own", [True, False])
def test_a_token_outside_the_vocabulary_is_marked(own):
    status = torch.zeros(1, dtype=I32, device=DEV)
    head, h = _head() if own else _head(status=status)
    assert own or head.status is status
    logits = f64(head(h))
    head.score(torch.tensor([1, 2, 3, V - 1], dtype=I32, device=DEV))
    assert dm.decomoe_read_status(head.status) == dm.DECOMOE_OK
    kept = [t[2].clone() for t in (head.logprob, head.entropy, head.top_id, head.top_logprob)]
    tokens = [5, -1, V, 7]
    head.score(torch.tensor(tokens, dtype=I32, device=DEV))
    assert dm.decomoe_read_status(head.status) == dm.DECOMOE_ERR_BAD_INPUT
    for t, was in zip((head.logprob, head.entropy, head.top_id, head.top_logprob), kept):
        assert torch.equal(t[2], was)
    lp, _, ids, _ = O.token_logprobs(logits[[0, 3]], [5, 7], 3)
    assert np.array_equal(head.top_id.cpu().numpy()[[0, 3]], ids)
    # fp32: sums of 333 exponentials (4e-6 is ample), and roundings of numbers as large as lp and ln 333 < 6
    assert (np.abs(f64(head.logprob)[[0, 3]] - lp) <= 4e-6 + 3 * 2.0 ** -24 * (2 * np.abs(lp) + 6)).all()
    head.score(torch.tensor([0, 0, 0, -1], dtype=I32, device=DEV))  # the mark was read
    assert dm.decomoe_read_status(head.status) == dm.DECOMOE_OK
