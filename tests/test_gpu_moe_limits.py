"""As many tokens and rows as the entry points promise: more workgroups than a launch can have, counts that pass 31 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def same(a, b, at_once=1 << 27):
    """a equals b, a piece at a time"""
    return a.shape == b.shape and all(torch.equal(a[i:i + at_once], b[i:i + at_once]) for i in range(0, a.shape[0], at_once))


def repeats(t, few):
    """whether the rows of t are those of `few` over and over"""
    n = t.shape[0] // few.shape[0]
    whole = t[:n * few.shape[0]].view(n, -1)
    some = max(1, (1 << 27) // whole.shape[1])
    return (all(bool((whole[i:i + some] == few.reshape(1, -1)).all()) for i in range(0, n, some))
            and torch.equal(t[n * few.shape[0]:], few[:t.shape[0] - n * few.shape[0]]))


# 16 lanes a token, and 64: 2^32 threads and more in one launch
@pytest.mark.parametrize("T,E,k", [(2 ** 28 + 3, 1, 1), (2 ** 26 + 3, 17, 17)])
def test_router_of_many_tokens(gpu_lib, T, E, k):
    print("[moe limits] router", T, E, k, flush=True)
    gen = torch.Generator().manual_seed(1)
    few = torch.randn(64, E, generator=gen).to(BF16).cuda()
    few_dw = torch.randn(64, k, generator=gen).cuda()

    def route(logits, dw):
        n = logits.shape[0]
        experts, weights = torch.full((n, k), -7, dtype=torch.int32, device="cuda"), torch.full((n, k), -7.0, device="cuda")
        d = torch.full((n, E), -7.0, dtype=BF16, device="cuda")
        gpu_lib.sptir_moe_route(logits, experts, weights, normalise=False)
        gpu_lib.sptir_moe_route_backward(logits, experts, weights, dw, d, normalise=False)
        return experts, weights, d

    want = route(few, few_dw)
    times = -(-T // 64)
    got = route(few.repeat(times, 1)[:T], few_dw.repeat(times, 1)[:T])
    torch.cuda.synchronize()
    for g, w, what in zip(got, want, ("experts", "weights", "d_logits")):
        assert repeats(g, w), what


# (where the kernel for few rows would take 2^32 threads and more)
@pytest.mark.parametrize("rows", [2 ** 29 + 5])
def test_product_of_many_rows(gpu_lib, rows):
    print("[moe limits] product", rows, flush=True)
    X = torch.randn(1009, 1, generator=torch.Generator().manual_seed(2)).to(BF16).cuda().repeat(-(-rows // 1009), 1)[:rows]
    W, Y = torch.full((1, 1), -1.75, dtype=BF16, device="cuda"), torch.zeros(rows, 1, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_product(None, X, W, Y)
    assert repeats(Y, (X[:1009].float() * -1.75).to(BF16))  # (a product of two is rounded once)


# all but five rows of the last expert, and of no expert
@pytest.mark.parametrize("E", [2, 1])
def test_experts_of_as_many_rows_as_there_may_be(gpu_lib, E):
    n = 2 ** 31 - 2
    print("[moe limits] rows", n, E, flush=True)
    ptr = torch.tensor([0, 5, n][:E + 1], dtype=torch.int32, device="cuda")
    unread = torch.empty(n, dtype=torch.int32, device="cuda")
    r = gpu_lib.MoeRouting(n, 1, E, ptr, unread, unread)
    few = torch.randn(1009, 1, generator=torch.Generator().manual_seed(3)).to(BF16).cuda()
    X = few.repeat(-(-n // 1009), 1)[:n]
    W = torch.tensor([[[0.5]], [[-3.0]]][:E], dtype=BF16, device="cuda")
    Y = torch.full((n, 1), 7.0, dtype=BF16, device="cuda")
    last = -3.0 if E == 2 else 0.0
    for call in (gpu_lib.sptir_moe_product, gpu_lib.sptir_moe_product_dx):
        Y.fill_(7.0)
        call(r, X, W, Y)
        assert torch.equal(Y[:5], (few[:5].float() * 0.5).to(BF16))
        assert repeats(Y[1009:], (few.float() * last).to(BF16))
        assert torch.equal(Y[5:1009], (few[5:].float() * last).to(BF16))


def test_entries_of_as_many_tokens_as_there_may_be(gpu_lib):
    """Sorted, there and back, a column wide: token t goes to expert t % 2."""
    n = 2 ** 31 - 2
    print("[moe limits] entries", n, flush=True)
    half = n // 2
    experts = torch.tensor([[0], [1]], dtype=torch.int32, device="cuda").repeat(half, 1)
    r = gpu_lib.sptir_moe_sort(experts, 2)
    assert r.expert_ptr.tolist() == [0, half, n]
    for which in range(2):
        places, entries = r.slot_of.view(half, 2)[:, which], r.entry_of[which * half:(which + 1) * half]
        for i in range(0, half, 1 << 28):
            want = torch.arange(i, min(i + (1 << 28), half), dtype=torch.int32, device="cuda")
            assert torch.equal(places[i:i + (1 << 28)], want + which * half) and torch.equal(entries[i:i + (1 << 28)], want * 2 + which)
    X = torch.randn(1009, 1, generator=torch.Generator().manual_seed(4)).to(BF16).cuda().repeat(-(-n // 1009), 1)[:n]
    Xs, Y = torch.zeros_like(X), torch.zeros_like(X)
    gpu_lib.sptir_moe_gather(r, X, Xs)
    assert same(Xs[:half], X[::2]) and same(Xs[half:], X[1::2])
    gpu_lib.sptir_moe_combine(r, Xs, Y)
    assert same(Y, X)
