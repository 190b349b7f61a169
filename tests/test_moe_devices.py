"""A routing whose arrays are on another device than the current one is refused, as other tensors are, before the library is called."""
import pytest
import torch

import paper_2207_04606_amd as sptir
from paper_2207_04606_amd import moe


class Elsewhere(torch.Tensor):
    """Host memory that says it is on a GPU: no call gets as far as to read it."""
    is_cuda = property(lambda self: True)

    def get_device(self):
        return getattr(self, "number", 0)


def on(number, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Elsewhere)
    t.number = number
    return t


@pytest.fixture
def current_device_0(monkeypatch):
    def called(*_):
        raise AssertionError("the library was called")

    class Library:
        sptir_moe_product_int8 = sptir_moe_product_dx_packed = sptir_moe_product_dw_packed = staticmethod(called)
        sptir_moe_product_dw_packed_workspace = staticmethod(lambda *_: 0)

    monkeypatch.setattr(moe, "_ready", Library)
    monkeypatch.setattr(moe, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def routing(number, T=4, k=1, E=2):
    return sptir.MoeRouting(T, k, E, on(number, E + 1, dtype=torch.int32), on(number, T * k, dtype=torch.int32), on(number, T * k, dtype=torch.int32))


def calls(r, number):
    i8, u8 = torch.int8, torch.uint8
    X, W, Q, X_e = on(number, 4, 32, dtype=i8), on(0, 2, 16, 32, dtype=i8), on(0, 4, 32, dtype=i8), on(0, 4, 1, dtype=u8)
    yield lambda: sptir.sptir_moe_product_int8(r, X, on(0, 4), W, on(0, 2, 16), on(0, 4, 16))
    yield lambda: sptir.sptir_moe_product_dx_packed(r, on(number, 4, 16), on(0, 2, 16, 32), on(0, 4, 32), Q, X_e, activation="relu")
    yield lambda: sptir.sptir_moe_product_dw_packed(r, on(number, 4, 16), Q, X_e, on(0, 2, 16, 32))


def test_routing_elsewhere(current_device_0):
    for call in calls(routing(0), 0):
        with pytest.raises(AssertionError, match="the library was called"):  # (everything where it has to be)
            call()
    for call in calls(routing(0), 1):
        with pytest.raises(ValueError, match="current device"):
            call()
    for call in calls(routing(1), 0):
        with pytest.raises(ValueError, match="current device"):
            call()
