"""Every kernel of the 8-bit products and weight gradients, at sizes that are no
multiples of its tile, with tiles not divided, all in parts, and those of the last
round in parts (tests/linear_shapes.py), against 64 bits.

Operands lie inside larger buffers, results in rows that are not aligned, with
NaN around them; then the result is added to itself.  An fp32 sum of n steps is
off by at most n 2^-24 sum |a b|: n = K / 8 + 32.  What the 8-bit instructions
drop: tests/test_gpu_linear_sums.py.
"""

import pytest

from tests import linear_shapes as S
from tests.gpu_harness import announce
from tests.test_gpu_linear_sums import U16, U32, _dropped

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def contexts():
    import torch
    from paper_2510_16981_amd import muonbp as mb
    assert torch.cuda.get_device_properties(0).multi_processor_count == 256  # what the sizes are planned for
    made = {False: mb.Linear(), True: mb.Linear(fp32_sums=True)}
    yield made
    for c in made.values():
        c.synchronize()
        c.close()


def _ids(size):
    return "%dx%dx%d" % size


def _random(rows, cols, seed):
    """Columns of different sizes, a few rows of zeros."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    x *= torch.randn(cols, generator=g, device="cuda").exp()
    x[3::17] = 0
    return x


def _blocks(lin, x, fmt):
    """x in 8 bits inside larger buffers, and its values."""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    rows, cols = x.shape
    wide = -(-cols // 128) * 128
    data = torch.full((rows + 2, wide + 16), 0x77, dtype=torch.uint8, device="cuda")
    scales = torch.full((-(-cols // 512), rows + 2), 0x7f7f7f7f, dtype=torch.int32, device="cuda")
    b = lin.quantize(x, out=mb.Blocks(data[2:, :wide], scales[:, 2:], cols, fmt))
    return b, lin.restore(b, dtype=torch.float32).double()


def _strided(rows, cols, dtype):
    """(A matrix of rows cols + 9 apart, one element into its buffer; the buffer.)"""
    import torch
    buf = torch.full((rows * (cols + 9) + 1,), float("nan"), dtype=dtype, device="cuda")
    return buf[1:].view(rows, cols + 9)[:, :cols], buf


def _check(call, a, b, dtype, fp32):
    """call(out, accumulate) against a b^T, then added to itself."""
    import torch
    rows, cols, k = a.shape[0], b.shape[0], a.shape[1]
    out, buf = _strided(rows, cols, dtype)
    call(out, False)
    ref, s1 = a @ b.T, a.abs() @ b.abs().T
    off = (k / 8 + 32) * U32 * s1
    if not fp32:
        off = off + _dropped(a, b)
    last = U16 if dtype == torch.bfloat16 else U32
    worst = float(((out.double() - ref).abs() / (off + last * (ref.abs() + off) + 1e-37)).max())
    plain = torch.empty(rows, cols, dtype=dtype, device="cuda")
    assert torch.equal(call(plain, False), out)
    call(out, True)
    want = ref + plain.double()
    again = float(((out.double() - want).abs() / (off + (last + U32) * (want.abs() + off) + 1e-37)).max())
    announce(f"error over tolerance {worst:.3f}, added {again:.3f}")
    assert worst <= 1 and again <= 1  # false for NaN too
    around = torch.isnan(buf)
    assert int((~around).sum()) == rows * cols


@pytest.mark.parametrize("size", list(S.PRODUCT), ids=_ids)
@pytest.mark.parametrize("fmt", [0, 1], ids=["e4m3", "e5m2"])
def test_product(contexts, size, fmt):
    import torch
    announce(f"product tiles {size} {fmt} {S.PRODUCT[size]}")
    lin, (m, n, k) = contexts[False], size
    a, a64 = _blocks(lin, _random(m, k, 1), fmt)
    b, b64 = _blocks(lin, _random(n, k, 2), 0)
    _check(lambda out, add: lin.product(a, b, out=out, accumulate=add), a64, b64, torch.bfloat16, False)


@pytest.mark.parametrize("size", list(S.EXACT), ids=_ids)
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [0, 1], ids=["e4m3", "e5m2"])
def test_product_of_fp32_sums(contexts, size, out, fmt):
    import torch
    announce(f"product tiles, fp32 sums {size} {out} {fmt} {S.EXACT[size]}")
    lin, (m, n, k) = contexts[out == "bf16"], size
    a, a64 = _blocks(lin, _random(m, k, 3), fmt)
    b, b64 = _blocks(lin, _random(n, k, 4), 0)
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    _check(lambda c, add: lin.product(a, b, out=c, accumulate=add), a64, b64, dtype, True)


@pytest.mark.parametrize("size", list(S.GRAD), ids=_ids)
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", [0, 1], ids=["e4m3", "e5m2"])
def test_weight_grad(contexts, size, out, fmt):
    import torch
    announce(f"weight gradient tiles {size} {out} {fmt} {S.GRAD[size]}")
    lin, (i, o, t) = contexts[False], size
    x, x64 = _blocks(lin, _random(t, i, 5), fmt)
    dy, _ = _strided(t, o, torch.bfloat16)
    dy.copy_(_random(t, o, 6))
    dtype = torch.bfloat16 if out == "bf16" else torch.float32
    _check(lambda dw, add: lin.weight_grad(x, dy, out=dw, accumulate=add), x64.T.contiguous(),
           dy.double().T.contiguous(), dtype, True)
