"""The options of the 8-bit linear layers' context, without a GPU."""

import ctypes
import os

import pytest

from paper_2510_16981_amd import muonbp as mb


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mb.LIB_PATH):
        from paper_2510_16981_amd import build
        build.build()
    return mb.load_library()


def test_sums_are_the_8_bit_instructions_unless_asked(lib):
    o = mb.LinearOptions()
    lib.muonbp_linear_options_default(ctypes.byref(o))
    assert o.fp32_sums == 0


@pytest.mark.parametrize("value", [2, -1])
def test_fp32_sums_is_0_or_1(lib, value):
    o = mb.LinearOptions(1 << 20, value)
    ctx = ctypes.c_void_p()
    assert lib.muonbp_linear_create(ctypes.byref(o), None, ctypes.byref(ctx)) == 1
    assert not ctx.value
