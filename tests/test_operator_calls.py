"""The short way of the 8-bit operators' calls: what it takes, what it leaves to binding.py.  Stand-ins with null addresses for the
tensors, so that the library answers without a GPU."""
import pytest
import torch

import __graft_entry__ as entry
from paper_2211_17192_b200 import binding

F, B, H, E, I8, I, U = torch.float32, torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8, torch.int32, torch.uint8


class StandIn:
    is_cuda = True

    def __init__(self, dtype, *shape, contiguous=True, device=0, stride=None):
        self.shape, self.dtype, self.contiguous, self.device, self.strides = torch.Size(shape), dtype, contiguous, device, stride

    def is_contiguous(self):
        return self.contiguous

    def get_device(self):
        return self.device

    def stride(self):
        return self.strides or torch.empty(self.shape, device="meta").stride()

    def data_ptr(self):
        return 0


def plain():
    cache = [StandIn(I8, 9, 2, 2, 64, 128), StandIn(F, 9, 2, 2, 64), StandIn(I, 3, 5)]
    return {
        "quantize": [StandIn(B, 4, 64), StandIn(E, 4, 64), StandIn(F, 4)],
        "norm": [StandIn(B, 4, 64), StandIn(F, 64), 1e-6, StandIn(F, 4, 64), StandIn(F, 4, 64), StandIn(E, 4, 64), StandIn(F, 4)],
        "linear": [StandIn(E, 4, 64), StandIn(F, 4), StandIn(E, 96, 64), StandIn(F, 96), StandIn(F, 96), 4, StandIn(B, 4, 48), StandIn(B, 4, 48)],
        "append": [StandIn(B, 3, 7, 2, 128), StandIn(B, 3, 7, 2, 128), *cache, StandIn(I, 3), StandIn(I, 3), StandIn(F, 99, 64, 2), StandIn(B, 3, 7, 4, 128),
                   StandIn(B, 3, 7, 4, 128)],
        "read": [*cache, StandIn(I, 3), 7, StandIn(I, 3), StandIn(B, 3, 7, 2, 128), StandIn(B, 3, 7, 2, 128)],
        "attention": [StandIn(B, 3, 7, 4, 128), *cache, StandIn(I, 3), 0.1, StandIn(B, 3, 7, 4, 128), StandIn(U, 1 << 20)],
    }


@pytest.fixture(scope="module")
def calls():
    entry.build()
    binding.lib()
    if binding._calls is None:
        pytest.skip("the module of csrc/calls.c is not built")
    return binding._calls


@pytest.mark.parametrize("name", list(plain()))
def test_plain_calls_reach_the_library(calls, name):
    assert getattr(calls, name)(*plain()[name], 0, 0) == -1 and b"null pointer" in binding.lib().spec_last_error()


@pytest.mark.parametrize("name", list(plain()))
def test_every_tensor_is_looked_at(calls, name):
    call = getattr(calls, name)
    for i, a in enumerate(plain()[name]):
        if not isinstance(a, StandIn):
            continue
        shape = tuple(a.shape)
        bad = [None, torch.zeros(shape, dtype=a.dtype), StandIn(torch.int64, *shape), StandIn(a.dtype, *shape, 1), StandIn(a.dtype, *shape, device=1),
               StandIn(a.dtype, *shape[:-1], 0), StandIn(a.dtype, *shape, contiguous=False, stride=(1,) * len(shape))]
        if a.dtype != U and not (a.dtype == I and len(shape) == 2):  # (any size of workspace is the library's to judge, and any width is a table's)
            bad.append(StandIn(a.dtype, *shape[:-1], shape[-1] + 1))
        for change in bad:
            args = plain()[name]
            args[i] = change
            optional = {"norm": (3,), "linear": (4, 6), "append": (6, 7), "read": (5,)}.get(name, ())
            status = call(*args, 0, 0)
            if change is None and i in optional:
                assert status == -1  # (one that may be missing)
            else:
                assert status is None, (i, change and (change.dtype, change.shape))


def test_types_and_strides(calls):
    args = plain()["attention"]
    args[0] = StandIn(B, 3, 7, 4, 128, contiguous=False, stride=(7 * 1024, 1024, 128, 1))  # part of a fused projection
    assert calls.attention(*args, 0, 0) == -1
    for stride in ((7 * 1024 + 8, 1024, 128, 1), (7 * 1024, 1024, 256, 1), (7 * 1024, 1024, 128, 2)):
        args[0] = StandIn(B, 3, 7, 4, 128, contiguous=False, stride=stride)
        assert calls.attention(*args, 0, 0) is None
    args = plain()["attention"]
    args[1], args[2] = StandIn(B, 9, 2, 2, 64, 128), None  # 16-bit pools have no scales
    assert calls.attention(*args, 0, 0) == -1
    args[2] = StandIn(F, 9, 2, 2, 64)
    assert calls.attention(*args, 0, 0) is None
    args = plain()["norm"]
    args[4] = StandIn(B, 4, 64)
    assert calls.norm(*args, 0, 0) is None  # residual and sum of different types
    args = plain()["linear"]
    for act in (0, 1, 5, -1, 2.0):
        args[5] = act
        assert calls.linear(*args, 0, 0) is None
    assert calls.quantize() is None and calls.linear(1, 2) is None
