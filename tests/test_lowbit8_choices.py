"""Which kernels the sizes of the GPU tests reach (csrc/w8_choice.h and gradient_choice.h, compiled for the host): all of them, whatever the fitted times become (no GPU)."""
import ctypes
import os
import subprocess

import pytest

from tests import test_gradient_kernels_gpu as gradients
from tests import test_gradient_scales_gpu as scales
from tests import test_lowbit8_routes_gpu as routes
from tests import test_w8_kernels_gpu as products

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = {"f32": 0, "bf16": 1, "f16": 2}


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    src, so = d / "choice.cpp", str(d / "choice.so")
    src.write_text('#include "w8_choice.h"\n#include "gradient_choice.h"\n'
                   'extern "C" int product(int rows, int in, int out)\n'
                   '{ const auto c = xnor::w8_choice(rows, in, out);\n'
                   '  return c.tiles ? c.tiles : 10 * c.side + 2 * (c.shares > 1) + (c.side == xnor::W8_SMALL && xnor::w8_alone(rows, in, out, c.shares)) + 4 * (in % 16 == 0); }\n'
                   'extern "C" int gradient(int rows, int in, int out, int group, int type, int w_type)\n'
                   '{ const xnor::GradientParts p(rows, group, type, w_type);\n'
                   '  const auto c = xnor::gradient_choice(p, rows, in, out, w_type == XNOR_F32 ? 4 : 2);\n'
                   '  return c.direct ? 0 : 100 * c.side + 10 * p.parts_x + p.parts_g; }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_1603_05279_amd", "csrc"), "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", so], check=True)
    return ctypes.CDLL(so)


SHARED, ALONE, ALIGNED = 2, 1, 4
# 16, 32 and 64 rows; tiles of 128: aligned alone, beside another, unaligned, each whole and in shares; tiles of 256 aligned and not
PRODUCTS = {1, 2, 4} | {1280 + s + k for s in (0, SHARED) for k in (ALIGNED | ALONE, ALIGNED, 0)} | {2560 + ALIGNED, 2560}
# few products; tiles of 64, 128 and 256 by the parts of rows and gradients (both in two: not with tiles of 256)
GRADIENTS = {0} | {100 * side + parts for side in (64, 128, 256) for parts in (11, 12, 21, 22)} - {25622}


def test_products_with_bias_and_special_scales_reach_every_kernel(lib):
    assert {lib.product(*s) for s in products.SIZES} == PRODUCTS


def test_products_reach_all_kernels_but_that_of_64_rows(lib):
    assert {lib.product(*s) for s in routes.PRODUCTS} | {4} == PRODUCTS


def test_special_gradients_reach_every_kernel(lib):
    assert {lib.gradient(*s, group, CODE[t], CODE[w]) for s in gradients.SIZES for t, w, group in gradients.KINDS} == GRADIENTS


def test_gradients_with_extreme_scales_reach_both_ways(lib):
    reached = {lib.gradient(*s, group, 0, 0) for s in scales.SIZES for group in (0, 32)}
    assert reached == {0, 6412, 6422, 12812, 12822}


def test_sizes_that_the_kernel_of_few_products_cannot_take(lib):
    for rows in (1, 64, 5000):
        assert lib.gradient(rows, 1, 100, 0, 0, 0) and lib.gradient(rows, 100, 1, 32, 1, 1)      # (it takes pairs of columns)
    for size in (1, 2 ** 24):
        assert lib.product(65535 * 64, 131071, size) > 0 and lib.gradient(65535 * 64, size, 2 ** 11, 0, 0, 0) >= 0      # (no overflow)


def test_the_largest_products_fit_a_launch(lib):
    """Outputs up to the memory's size (288 GB of 16 bits: 2^37 results and some) never need more tiles than one launch holds: those of 128 give way to those of 256."""
    most = 0xffffff00 // 512
    for rows, out in ((65535 * 64, 32768), (65535 * 64, 36000), (2 ** 20, 140000), (2 ** 14, 2 ** 23 + 5), (9000, 2 ** 24)):
        for cin in (1, 16, 64, 100, 128, 256, 1000, 1024, 9216, 131071):
            route = lib.product(rows, cin, out)
            if route >= 1280:
                side = 256 if route >= 2560 else 128
                assert -(-rows // side) * -(-out // side) <= most, (rows, cin, out, route)
