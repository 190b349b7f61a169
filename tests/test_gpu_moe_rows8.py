"""Rows in 8 bits: quantised with a scale each, packed with an exponent for every 32 columns and read back; codes, scales and exponents
have to be those of the definition exactly (tests/moe8_reference.py)."""
import math

import pytest
import torch

import moe8_reference as ref8
import moe_reference as ref
from test_gpu_moe import ACTS, BF16, F16, F32, TYPES, out_like, randn, say, strided

pytestmark = pytest.mark.gpu
SHAPES = [(1, 1, 0), (1, 8, 0), (3, 7, 2), (5, 31, 1), (5, 32, 0), (4, 33, 3), (70, 64, 0), (9, 100, 4), (33, 256, 8), (12, 777, 5), (7, 2048, 0),
          (5, 2056, 0), (3, 4099, 1), (2, 20000, 0), (600, 40, 0), (20000, 16, 0)]


def rows_of(gen, n, width, dtype):
    """Rows of many sizes, some with values that are ties, zeros, or all alike."""
    X = randn(gen, n, width) * torch.exp(2.0 * randn(gen, n, 1))
    if n > 2:
        X[1] = 0.0
        X[2] = torch.randint(-254, 255, (width,), generator=gen).float() / 2   # halves: ties
        X[2, 0] = 127.0
    if n > 4:
        X[3] = -0.0
        X[4] = 3.0
    return X.to(dtype)


def codes_like(rows, cols, extra):
    whole = torch.full((rows, cols + extra), 99, dtype=torch.int8, device="cuda")
    return whole[:, :cols], whole[:, cols:]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,width,extra", SHAPES)
def test_quantise(gpu_lib, dtype, n, width, extra):
    say("quantise", dtype, n, width, extra)
    X = rows_of(torch.Generator().manual_seed(n + width), n, width, dtype)
    Q, rest = codes_like(n, width, extra)
    scales = torch.full((n,), math.nan, device="cuda")
    gpu_lib.sptir_moe_quantise(strided(X, extra), Q, scales)
    want, s_want = ref8.quantise(X)
    assert torch.equal(scales.cpu(), s_want)
    assert torch.equal(Q.cpu(), want)
    assert (rest == 99).all()


def test_quantise_at_the_ends(gpu_lib):
    tiny = 2.0 ** -149
    X = torch.tensor([[3.4e38, -1.7e38, 1.0, 0.0], [tiny * 100, tiny * 99, -tiny, 0.0], [tiny * 60, tiny, 0.0, -tiny * 60],
                      [tiny * 190, tiny * 100, -tiny * 190, 0.0], [2.0 ** -126, 2.0 ** -127, -(2.0 ** -130), 0.0],
                      [math.inf, 1.0, 0.0, 0.0], [1.0, math.nan, 0.0, 0.0], [-math.inf, math.nan, 0.0, 0.0], [2.0 ** -60, 2.0 ** -61, -(2.0 ** -62), 0.0]])
    Q, scales = torch.empty(9, 4, dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda")
    gpu_lib.sptir_moe_quantise(X.cuda(), Q, scales)
    want, s_want = ref8.quantise(X)
    assert torch.equal(torch.nan_to_num(scales.cpu(), nan=-1.0), torch.nan_to_num(s_want, nan=-1.0))
    assert torch.equal(Q.cpu(), want)


@pytest.mark.parametrize("seed", range(4))
def test_quantise_next_to_the_middle(gpu_lib, seed):
    """Values one unit of float32 above and below the middle between two codes, of scales with many digits."""
    gen = torch.Generator().manual_seed(seed)
    n, width = 64, 255
    most = torch.exp(3.0 * randn(gen, n, 1))
    s = (most / torch.tensor(127.0)).double()
    X = (s * (torch.arange(width).double() - 127.0 + 0.5)).float()
    X[:, 0] = most[:, 0]
    for shifted in (X, torch.nextafter(X, torch.full_like(X, math.inf)), torch.nextafter(X, torch.full_like(X, -math.inf))):
        x = torch.where(shifted.abs() > most, most, shifted)
        Q, scales = torch.empty(n, width, dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        gpu_lib.sptir_moe_quantise(x.cuda(), Q, scales)
        want, s_want = ref8.quantise(x)
        assert torch.equal(scales.cpu(), s_want) and torch.equal(Q.cpu(), want)


def test_quantise_weights_of_experts(gpu_lib):
    gen = torch.Generator().manual_seed(7)
    W = randn(gen, 5, 24, 72, dtype=BF16)
    Q, scales = torch.empty(5, 24, 72, dtype=torch.int8, device="cuda"), torch.empty(5, 24, device="cuda")
    gpu_lib.sptir_moe_quantise(W.cuda(), Q, scales)
    want, s_want = ref8.quantise(W.view(-1, 72))
    assert torch.equal(Q.cpu().view(-1, 72), want) and torch.equal(scales.cpu().view(-1), s_want)


def packed(lib, X, extra=0):
    n, width = X.shape
    Q, rest = codes_like(n, width, extra)
    blocks = -(-width // ref8.BLOCK)
    E = torch.full((n, blocks + extra), 9, dtype=torch.uint8, device="cuda")
    lib.sptir_moe_pack(strided(X, extra), Q, E[:, :blocks])
    assert (rest == 99).all() and (E[:, blocks:] == 9).all()
    return Q, E[:, :blocks]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,width,extra", SHAPES)
def test_pack_and_unpack(gpu_lib, dtype, n, width, extra):
    say("pack", dtype, n, width, extra)
    X = rows_of(torch.Generator().manual_seed(n + width), n, width, dtype)
    Q, E = packed(gpu_lib, X, extra)
    want, e_want = ref8.pack(X)
    assert torch.equal(E.cpu(), e_want)
    assert torch.equal(Q.cpu(), want)
    values = ref8.kept(want, e_want, dtype)
    # (the exponent e is the smallest with largest < 127.5 * 2^e, so largest >= 127.5 * 2^(e - 1), and half a unit is 2^(e - 1))
    largest = X.double().abs().amax(1, keepdim=True)
    off = float(((values.double() - X.double()).abs() / largest.clamp(min=1e-300)).max())
    assert off <= 1.0 / 127.5
    for act in ACTS:
        if act == "swiglu" and width % 2:
            continue
        y, limit = ref8.unpacked(values, act)
        out, rest = out_like(n, y.shape[1], dtype, extra)
        gpu_lib.sptir_moe_unpack(Q, E, out, activation=act)
        # (the product of two large halves of a float16 row is past its range: rounded to an infinity)
        past = torch.isinf(y.to(dtype))
        assert torch.equal(out.cpu()[past], y.to(dtype)[past])
        ref.check(torch.where(past, torch.zeros_like(y), out.cpu().double()), torch.where(past, 0.0, y), torch.where(past, 0.0, limit), "unpack " + act)
        assert torch.isnan(rest).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_pack_at_the_ends(gpu_lib, dtype):
    """The largest and the smallest numbers of a type, the borders between exponents, infinities and NaN."""
    info = torch.finfo(dtype)
    least = 2.0 ** -149 if dtype is F32 else 2.0 ** -24 if dtype is F16 else 2.0 ** -133
    rows = [[info.max, -info.max, 1.0, 0.0], [info.max / 2, 1.0, -1.0, 0.0], [least, -least, 0.0, least * 2], [least * 127, least * 128, 0.0, least],
            [info.tiny, -info.tiny, least, 0.0], [127.0, 127.5, -1.5, 2.5], [127.5, 64.0, 0.5, 1.5], [128.0, 63.5, 1.0, -3.0], [255.0, 254.0, 1.0, 3.0],
            [math.inf, 1.0, 2.0, 3.0], [1.0, math.nan, 2.0, 3.0], [1.0, -math.inf, math.nan, 0.0]]
    X = torch.zeros(len(rows), 64)
    X[:, :4] = torch.tensor(rows, dtype=torch.float64).float()
    X[:, 32:] = 5.0                                        # the other block of the row keeps its values
    X = X.to(dtype)
    Q, E = packed(gpu_lib, X)
    want, e_want = ref8.pack(X)
    assert torch.equal(E.cpu(), e_want)
    live = e_want != 255
    assert torch.equal(Q.cpu().view(-1, 2, 32)[live], want.view(-1, 2, 32)[live])
    out = torch.empty(len(rows), 64, dtype=dtype, device="cuda")
    gpu_lib.sptir_moe_unpack(Q, E, out)
    got = out.cpu()
    assert torch.isnan(got[9:, :32]).all() and torch.isfinite(got[:9]).all()
    assert (got[:, 32:] == 5.0).all()
    values = ref8.kept(want, e_want, dtype)
    assert torch.equal(got[:9], values[:9])


@pytest.mark.parametrize("n,width", [(700001, 8), (70001, 300)])
def test_more_rows_than_workgroups(gpu_lib, n, width):
    X = randn(torch.Generator().manual_seed(n), n, width, dtype=BF16)
    Q, E = packed(gpu_lib, X)
    want, e_want = ref8.pack(X)
    assert torch.equal(E.cpu(), e_want) and torch.equal(Q.cpu(), want)
    out, s = torch.empty(n, width, dtype=BF16, device="cuda"), torch.empty(n, device="cuda")
    gpu_lib.sptir_moe_unpack(Q, E, out)
    assert torch.equal(out.cpu(), ref8.kept(want, e_want, BF16))
    gpu_lib.sptir_moe_quantise(X.cuda(), Q, s)
    want, s_want = ref8.quantise(X)
    assert torch.equal(Q.cpu(), want) and torch.equal(s.cpu(), s_want)


def test_large_strides(gpu_lib):
    """Rows whose places pass 2^32 bytes."""
    n, width, ld = 3, 40, 1 << 31
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    big = torch.empty(2 * ld + width, dtype=torch.int8, device="cuda")
    Q = big.as_strided((n, width), (ld, 1))
    gen = torch.Generator().manual_seed(1)
    X = randn(gen, n, width, dtype=BF16)
    E = torch.empty(n, 2, dtype=torch.uint8, device="cuda")
    gpu_lib.sptir_moe_pack(X.cuda(), Q, E)
    want, e_want = ref8.pack(X)
    assert torch.equal(Q.cpu(), want) and torch.equal(E.cpu(), e_want)
    out = torch.empty(n, width, dtype=BF16, device="cuda")
    gpu_lib.sptir_moe_unpack(Q, E, out)
    assert torch.equal(out.cpu(), ref8.kept(want, e_want, BF16))
    s = torch.empty(n, device="cuda")
    gpu_lib.sptir_moe_quantise(X.cuda(), Q, s)
    want, s_want = ref8.quantise(X)
    assert torch.equal(Q.cpu(), want) and torch.equal(s.cpu(), s_want)


def test_nothing_to_do(gpu_lib):
    for n, width in ((0, 8), (4, 0), (0, 0)):
        X, Q = torch.empty(n, width, device="cuda"), torch.empty(n, width, dtype=torch.int8, device="cuda")
        E, s = torch.empty(n, -(-width // 32), dtype=torch.uint8, device="cuda"), torch.full((n,), math.nan, device="cuda")
        gpu_lib.sptir_moe_quantise(X, Q, s)
        assert (s == 0).all()
        gpu_lib.sptir_moe_pack(X, Q, E)
        gpu_lib.sptir_moe_unpack(Q, E, X)


def test_weights_without_columns_and_strided_scales(gpu_lib):
    for E, n, width in ((3, 5, 0), (0, 5, 8), (3, 0, 8)):
        s = torch.full((E, n), math.nan, device="cuda")
        gpu_lib.sptir_moe_quantise(torch.empty(E, n, width, device="cuda"), torch.empty(E, n, width, dtype=torch.int8, device="cuda"), s)
        assert (s == 0).all()
    W, Q = torch.zeros(3, 5, 8, device="cuda"), torch.zeros(3, 5, 8, dtype=torch.int8, device="cuda")
    with pytest.raises(ValueError):
        gpu_lib.sptir_moe_quantise(W, Q, torch.zeros(3, 6, device="cuda")[:, :5])
    with pytest.raises(ValueError):
        gpu_lib.sptir_moe_quantise(W.mT, Q.mT, torch.zeros(3, 8, device="cuda"))


def test_refusals(gpu_lib):
    X = torch.zeros(4, 64, device="cuda")
    Q, E, s = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(4, 2, dtype=torch.uint8, device="cuda"), torch.zeros(4, device="cuda")
    for call in (lambda: gpu_lib.sptir_moe_quantise(X, Q[:, :63], s), lambda: gpu_lib.sptir_moe_quantise(X, Q, s[:3]), lambda: gpu_lib.sptir_moe_pack(X, Q, E[:, :1]),
                 lambda: gpu_lib.sptir_moe_pack(X, Q.t().contiguous().t(), E), lambda: gpu_lib.sptir_moe_unpack(Q, E, X, activation="tanh"),
                 lambda: gpu_lib.sptir_moe_unpack(Q[:, :63], E, X, activation="swiglu"), lambda: gpu_lib.sptir_moe_unpack(Q, E, X, activation="swiglu")):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gpu_lib.sptir_moe_quantise(X.double(), Q, s), lambda: gpu_lib.sptir_moe_quantise(X, Q.float(), s), lambda: gpu_lib.sptir_moe_pack(X.cpu(), Q, E),
                 lambda: gpu_lib.sptir_moe_pack(X, Q, E.to(torch.int8)), lambda: gpu_lib.sptir_moe_unpack(Q, E, X.double())):
        with pytest.raises(TypeError):
            call()
