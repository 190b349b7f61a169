"""Calls on a stream that is not the current one, without a wait of the host between them: workspaces and new routings come from that
stream's memory, and calls on two streams at once do not meet in it."""
import pytest
import torch

import moe_reference as ref
from paper_2207_04606_amd import moe
from test_gpu_moe import BF16, choices, randn, say

pytestmark = pytest.mark.gpu


def test_memory_of_the_stream_of_the_call(gpu_lib):
    """A block that was freed under the current stream is not handed to a call on another one."""
    side, nbytes = torch.cuda.Stream(), 12 << 20
    torch.cuda.synchronize()
    for given in (side, side.cuda_stream):
        block = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        freed = block.data_ptr()
        del block
        on_side = moe._workspace(nbytes, given)
        assert on_side.data_ptr() != freed
        here = moe._workspace(nbytes, None)
        assert here.data_ptr() == freed
        del here
        assert moe._workspace(nbytes, 0).data_ptr() == freed  # (the default stream, which is the current one)
        del on_side


@pytest.mark.parametrize("T,k,E", [(9000, 1, 3), (30000, 2, 40)])
def test_two_streams_at_once(gpu_lib, T, k, E):
    """Sorts and weight gradients in parts, alternating between two streams: the results of calls one after another."""
    say("two streams", T, k, E)
    gen = torch.Generator().manual_seed(T)
    chosen = [choices(gen, T, k, E, 0.1) for _ in range(2)]
    dev = [e.cuda() for e in chosen]
    dense = [(randn(gen, 9000, 24 + i, dtype=BF16).cuda(), randn(gen, 9000, 40, dtype=BF16).cuda()) for i in range(2)]
    want = []
    for dZ, X in dense:
        dW = torch.empty(dZ.shape[1], 40, dtype=BF16, device="cuda")
        gpu_lib.sptir_moe_product_dw(None, dZ, X, dW)
        want.append(dW)
    assert moe._library().sptir_moe_product_dw_workspace(9000, 1, 40, 24) > 0 and moe._library().sptir_moe_sort_workspace(T * k, E) > 0
    outs = [[torch.empty_like(w) for _ in range(20)] for w in want]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    routings = [[], []]
    for n in range(20):
        for which, stream in ((0, None), (1, side)):
            gpu_lib.sptir_moe_product_dw(None, *dense[which], outs[which][n], stream=stream)
            routings[which].append(gpu_lib.sptir_moe_sort(dev[which], E, stream=stream))
            del routings[which][:-3]
    torch.cuda.synchronize()
    for which in range(2):
        for dW in outs[which]:
            assert torch.equal(dW, want[which])
        order = ref.sort(chosen[which], E)
        for r in routings[which]:
            assert all(torch.equal(got.cpu(), w) for got, w in zip((r.expert_ptr, r.entry_of, r.slot_of), order))
