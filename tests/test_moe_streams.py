"""Memory that the mixture-of-experts binding allocates for a call on a given stream: taken under that stream, so that the caching
allocator orders it behind what the stream has yet to do.  A block taken under the current stream may still be read or written
there, by kernels that the call's own do not wait for.  (Host logic: torch's streams are stood in for, no GPU is touched.)"""
import contextlib
import types

import pytest
import torch

from paper_2207_04606_amd import moe


class Stream:
    def __init__(self, number):
        self.cuda_stream = number

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream


class Allocator:
    """torch.empty that notes the stream it was called under and the streams a block was recorded on."""

    def __init__(self, monkeypatch):
        self.now, self.taken = Stream(11), []
        cuda = types.SimpleNamespace(Stream=Stream, ExternalStream=self.external, stream=self.stream, current_stream=lambda: self.now,
                                     default_stream=lambda: Stream(0))
        names = {name: getattr(torch, name) for name in ("uint8", "int32", "Tensor")}
        monkeypatch.setattr(moe, "torch", types.SimpleNamespace(cuda=cuda, empty=self.empty, **names))

    def external(self, number):
        assert number != 0  # (torch would make a new stream of it)
        return Stream(number)

    @contextlib.contextmanager
    def stream(self, s):
        before, self.now = self.now, s
        yield
        self.now = before

    def empty(self, n, dtype, device):
        block = types.SimpleNamespace(under=self.now, on=[], numel=lambda: n, data_ptr=lambda: 4096)
        block.record_stream = block.on.append
        self.taken.append(block)
        return block


GIVEN = [(Stream(77), 77), (78, 78), (0, 0)]


@pytest.mark.parametrize("given,number", GIVEN)
def test_workspace_is_taken_under_the_stream_of_the_call(monkeypatch, given, number):
    a = Allocator(monkeypatch)
    moe._workspace(64, given)
    assert [b.under.cuda_stream for b in a.taken] == [number] and a.now == Stream(11)
    moe._workspace(64, None)
    assert a.taken[-1].under == Stream(11)
    assert moe._workspace(0, given) is None


@pytest.mark.parametrize("given,number", GIVEN)
def test_a_new_routing_is_taken_under_the_stream_of_the_call(monkeypatch, given, number):
    a = Allocator(monkeypatch)
    calls = []
    lib = types.SimpleNamespace(sptir_moe_sort_workspace=lambda n, e: 256, sptir_moe_sort=lambda *args: calls.append(args) or 0)
    monkeypatch.setattr(moe, "_ready", lib)
    monkeypatch.setattr(moe, "_dev", lambda t, dtype, what: t)
    monkeypatch.setattr(moe, "_stream_ptr", lambda s: number)
    experts = torch.zeros(5, 2, dtype=torch.int32)
    moe.sptir_moe_sort(experts, 3, stream=given)
    assert len(calls) == 1 and [b.under.cuda_stream for b in a.taken] == [number] * 4
    # the three arrays go to the caller, who uses them under the current stream
    assert all(Stream(11) in b.on for b in a.taken[:3])
    del a.taken[:]
    moe.sptir_moe_sort(experts, 3)
    assert [b.under.cuda_stream for b in a.taken] == [11] * 4 and not any(b.on for b in a.taken)
