"""The 8-bit linear-layer operators without a GPU: the oracle's own pins, the
C structs, and what the library refuses before it touches a device."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import linear_oracle as O
from paper_2510_16981_amd import muonbp as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TORCH8 = {0: torch.float8_e4m3fn, 1: torch.float8_e5m2}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(mb.LIB_PATH):
        from paper_2510_16981_amd import build
        build.build()
    return mb.load_library()


@pytest.mark.parametrize("fmt", [0, 1])
def test_oracle_codes_are_the_types(fmt):
    codes = torch.arange(256, dtype=torch.uint8)
    want = codes.view(TORCH8[fmt]).double().numpy()
    np.testing.assert_array_equal(O.code_values(fmt), want)


@pytest.mark.parametrize("fmt", [0, 1])
def test_oracle_rounds_to_nearest_even(fmt):
    g = torch.Generator().manual_seed(fmt)
    x = torch.cat([torch.randn(20000, generator=g) * s for s in (1e-3, 0.1, 1, 50)])
    top = 448.0 if fmt == 0 else 57344.0
    v = O.code_values(fmt)
    ties = torch.from_numpy(((v[:126] + v[1:127]) / 2)[np.isfinite(v[1:127])]).float()
    x = torch.cat([x, ties, -ties, torch.tensor([0.0, -0.0, top, -top])]).clamp(-top, top)
    want = x.to(TORCH8[fmt]).view(torch.uint8).numpy()
    np.testing.assert_array_equal(O.nearest(x.double().numpy(), fmt), want)


@pytest.mark.parametrize("fmt", [0, 1])
def test_oracle_scale_is_the_smallest_that_fits(fmt):
    top = 448.0 if fmt == 0 else 57344.0
    for a in (1e-20, 0.3, 1.0, 1.75, np.nextafter(1.75, 2), 447.9, 448.0, 448.1, 3e38):
        e = O.scale_exponent(a, fmt)
        assert a <= top * 2.0 ** e and a > top * 2.0 ** (e - 1)
    assert O.scale_exponent(0.0, fmt) == O.scale_exponent(1e-40, fmt) == -110


def test_oracle_gradient_against_differences():
    rng = np.random.default_rng(0)
    g, u, d = rng.standard_normal((3, 4, 50)) * 2
    h = 1e-6
    dg, du = O.gated_backward(d, g, u)
    num_g = d * (O.gated_forward(g + h, u) - O.gated_forward(g - h, u)) / (2 * h)
    num_u = d * (O.gated_forward(g, u + h) - O.gated_forward(g, u - h)) / (2 * h)
    np.testing.assert_allclose(dg, num_g, rtol=1e-7, atol=1e-8)
    np.testing.assert_allclose(du, num_u, rtol=1e-7, atol=1e-8)


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a host C compiler")
def test_ctypes_structs_match_header(tmp_path):
    structs = {"muonbp_dense": mb.Dense, "muonbp_blocks": mb.BlocksRef, "muonbp_linear_options": mb.LinearOptions}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "muonbp.h"', "int main(void) {"]
    want = []
    for name, cls in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        want.append(ctypes.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run(["gcc", "-std=c11", "-I", f"{ROOT}/include", str(src), "-o", str(tmp_path / "layout")],
                   check=True, capture_output=True)
    got = subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True, text=True).stdout
    assert [int(v) for v in got.split()] == want


def test_defaults_and_null_context(lib):
    o = mb.LinearOptions()
    lib.muonbp_linear_options_default(ctypes.byref(o))
    assert o.workspace_bytes == 64 << 20
    lib.muonbp_linear_options_default(None)
    assert lib.muonbp_linear_quantize(None, None, None) == 1
    assert lib.muonbp_linear_quantize_weight(None, None, None, None) == 1
    assert lib.muonbp_linear_restore(None, None, None) == 1
    assert lib.muonbp_linear_product(None, None, None, None, 0) == 1
    assert lib.muonbp_linear_weight_grad(None, None, None, None, 0) == 1
    assert lib.muonbp_linear_gated_forward(*[None] * 7) == 1
    assert lib.muonbp_linear_gated_backward(*[None] * 8) == 1
    assert lib.muonbp_linear_set_stream(None, None) == 1
    assert lib.muonbp_linear_synchronize(None) == 1
    assert lib.muonbp_linear_last_error(None) == b"NULL context"
    lib.muonbp_linear_destroy(None)


def test_create_refuses_before_gpu(lib):
    assert lib.muonbp_linear_create(None, None, None) == 1
    ctx = ctypes.c_void_p()
    o = mb.LinearOptions(-1)
    assert lib.muonbp_linear_create(ctypes.byref(o), None, ctypes.byref(ctx)) == 1
    assert not ctx.value


def test_blocks_refuse_host_and_ill_shaped_tensors():
    with pytest.raises(ValueError, match="data"):
        mb.Blocks(torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(1, 4, dtype=torch.int32), 100)
