"""Tensors of several devices, or of another device than the current one, are refused
before anything is called. The tensors are fake ones, without memory."""
from unittest import mock

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2609_38823_gb300 as dm

BF16, I32 = torch.bfloat16, torch.int32


@pytest.fixture(scope="module", autouse=True)
def built_lib():
    import __graft_entry__

    __graft_entry__.build()
    return dm.lib()


def _calls(dev):
    """Each call's arguments, tensor by tensor on the device dev(i)."""
    made = iter(range(100))

    def t(*shape, dtype=I32):
        return torch.empty(*shape, dtype=dtype, device=dev(next(made)))

    # a fake tensor of a device that is not there is made only where torch sees no GPU at all
    with mock.patch.object(torch.cuda, "is_available", lambda: False), FakeTensorMode():
        pool = [t(3, 16, 2, 64, dtype=BF16) for _ in range(2)]
        return {
            "plan": lambda c=[t(2), t(2), 16, t(4), t(2, 3), t(2), t(3), t(2)]: dm.decomoe_paged_plan(*c),
            "plan_step": lambda c=[t(2), t(2), 16, t(4), t(2, 3), t(2), t(2)]: dm.decomoe_paged_plan_step(*c),
            "advance": lambda c=[t(2), t(2), t(2, 3), 16]: dm.decomoe_paged_advance(*c),
            "append": lambda c=[t(2, 2, 64, dtype=BF16), t(2, 2, 64, dtype=BF16), t(2)] + pool: dm.decomoe_paged_append(*c),
            "attention": lambda c=[t(2, 4, 64, dtype=BF16)] + pool + [t(2, 3), t(2), t(2, 4, 64, dtype=BF16),
                                                                     t(1 << 24, dtype=torch.uint8)]:
                dm.decomoe_paged_attention(*c),
            "norm": lambda c=[t(2, 64, dtype=BF16), t(2, 64, dtype=BF16), t(64, dtype=BF16), t(2, 64, dtype=BF16)]:
                dm.decomoe_add_rmsnorm_q8(*c),
            "w4": lambda c=[t(2, 64, dtype=BF16), t(8, 32, dtype=torch.uint8), t(8, 1, dtype=BF16), t(2, 8, dtype=BF16)]:
                dm.decomoe_w4_linear(*c),
        }


NAMES = ["plan", "plan_step", "advance", "append", "attention", "norm", "w4"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("dev", [lambda i: f"cuda:{i % 2}", lambda i: f"cuda:{1 - i % 2}"])
def test_two_devices(name, dev):
    with pytest.raises(ValueError, match="one device"):
        _calls(dev)[name]()


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_another_device_than_the_current_one(name):
    assert torch.cuda.current_device() == 0
    with pytest.raises(ValueError, match="current device"):
        _calls(lambda i: "cuda:1")[name]()
