"""Which kernel takes a product of an expert layer (csrc/moe_choice.h, compiled alone): the sizes of test_gpu_moe_wide.py take more large
tiles than the card has CUs, and every kernel takes some."""
import os
import subprocess

import pytest

import moe_wide_shapes as wide
from paper_2207_04606_amd import build as sptir_build
from paper_2207_04606_amd import moe

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def choice(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("choice") / "choice")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused-function", "-I", sptir_build.CSRC,
                           "-o", exe, os.path.join(HERE, "moe_choice_main.cpp")])

    def ask(op, *sizes):  # (few, wide, fragments, parts)
        out = subprocess.run([exe], input=" ".join(str(int(v)) if v is not op else v for v in (op, *sizes)), check=True, capture_output=True, text=True)
        return tuple(int(v) for v in out.stdout.split())

    return ask


@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.FORWARD)
def test_large_tiles_of_the_product(choice, T, k, E, d_in, d_out, act, dropped):
    few, is_wide, _, _ = choice("forward", T * k, max(E, 1), E > 0, wide.columns(d_out, act), d_in, 0, 1, act == "swiglu")
    assert not few and is_wide
    assert wide.tiles(T * k * (1 - dropped), wide.columns(d_out, act)) > 256


@pytest.mark.parametrize("T,k,E,d_in,d_out,act,dropped", wide.DX)
def test_large_tiles_of_the_inputs_gradient(choice, T, k, E, d_in, d_out, act, dropped):
    assert choice("dx", T * k, max(E, 1), E > 0, d_in, d_out, 0, 1, 0)[:2] == (0, 1)
    assert wide.tiles(T * k * (1 - dropped), d_in) > 256


@pytest.mark.parametrize("T,k,E,d_in,d_out,dropped", wide.DW)
def test_large_tiles_of_the_weights_gradient(choice, T, k, E, d_in, d_out, dropped):
    assert choice("dw", T * k, max(E, 1), d_in, d_out, 0, 1) == (0, 1, 1, 1)
    assert max(E, 1) * wide.tiles(d_out, d_in) > 256


def test_no_large_tiles_of_float32_or_odd_operands(choice):
    for f32, words in ((1, 1), (0, 0), (1, 0)):
        assert choice("forward", 8192, 1, 0, 8192, 8192, f32, words, 0)[:2] == (0, 0)
        assert choice("dx", 8192, 1, 0, 8192, 8192, f32, words, 0)[:2] == (0, 0)
        assert choice("dw", 8192, 1, 8192, 8192, f32, words)[1] == 0


def test_single_tokens_take_the_kernel_for_few_rows(choice):
    for E, k, d_in, n_j in ((64, 8, 2048, 2048), (8, 2, 256, 128)):
        assert choice("forward", k, E, 1, n_j, d_in, 0, 1, 0)[::2] == (1, 1)
    assert choice("forward", 128, 1, 0, 4096, 4096, 0, 1, 0)[0] == 1
    assert choice("forward", 1024, 1, 0, 4096, 4096, 0, 1, 0)[0] == 0


def test_few_weights_and_many_rows_are_summed_in_parts(choice):
    assert choice("dw", 32768, 1, 1024, 2048, 0, 1)[3] > 1
    assert choice("dw", 32768, 32, 4096, 4096, 0, 1)[3] == 1


def test_the_kernel_for_few_rows_fits_one_launch(choice):
    """A launch of 2^32 threads and more runs only a part of them: other kernels take such calls."""
    for rows, E, routed in ((2 ** 29 + 5, 1, 0), (2 ** 29 + 5, 3, 1), (2 ** 31 - 2, 1, 0), (2 ** 31 - 2, 1024, 1), (3 * 10 ** 8, 1, 0), (2 ** 27 + 1, 1, 0)):
        for n_j, n_r, gated in ((1, 1, 0), (8, 8, 0), (64, 8, 0), (64, 8, 1), (2 ** 28, 1, 0)):
            few, _, fragments, _ = choice("forward", rows, E, routed, n_j, n_r, 0, 0, gated)
            out, cols = (n_j // 2, 16) if gated else (n_j, 16 if fragments == 1 else 32)
            assert not few or -(-rows // (16 * fragments)) * -(-out // cols) * 512 < 2 ** 32


@pytest.mark.parametrize("rows", [16, 32, 64, 128, 256])
def test_tiles_of_as_many_rows_as_there_may_be(choice, rows):
    most = 2 ** 31 - 2
    for lo, hi in ((0, most), (1, most), (0, most - rows), (5, most), (7, 7), (most, most), (0, 1), (3, 3 + rows), (3, 4 + rows)):
        assert choice("tiles", lo, hi, rows) == (-(-(hi - lo) // rows),)


def test_no_workspace_for_sizes_that_are_refused():
    need = moe._library().sptir_moe_product_dw_workspace
    most = 2 ** 31 - 1
    for sizes in ((10 ** 6, 1, 64, most), (10 ** 6, 1, most, 64), (10 ** 6, 1, most, most), (10 ** 6, 1, 64, most // 4 + 1), (2 ** 62, most, 64, 64), (10 ** 6, 1025, 1, 1)):
        assert need(*sizes) == 0
    assert need(10 ** 6, 1, 64, 64) > 0
