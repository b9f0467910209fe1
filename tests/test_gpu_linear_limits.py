"""The largest matrices of the 8-bit operators: what is past them is refused
before anything is launched, and the last that is accepted runs."""

import pytest

from tests.gpu_harness import announce

pytestmark = pytest.mark.gpu

MOST = 2 ** 26 - 4  # rows times groups of 512 columns


@pytest.fixture(scope="module")
def lin():
    from paper_2510_16981_amd import muonbp as mb
    ctx = mb.Linear()
    yield ctx
    ctx.synchronize()
    ctx.close()


@pytest.mark.parametrize("rows,cols", [(2 ** 26, 1), (2 ** 26, 512), (MOST + 1, 200), (2 ** 25, 513), (2 ** 13, 2 ** 22)])
def test_larger_ones_are_refused(lin, rows, cols):
    """E_SHAPE, and the context stays usable.  (The descriptions name more
    memory than there is behind them: nothing may read it.)"""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lib, ctx = lin.lib, lin.ctx
    mem = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    wide = -(-cols // 128) * 128
    at = mem.data_ptr()
    ref = [mb._BLOCKS.pack(at + 4096 * k, at + 4096 * k + 2048, rows, cols, wide, rows, mb.E4M3) for k in range(6)]
    d = [mb._DENSE.pack(at + 4096 * (k + 8), rows, cols, cols, mb.BF16) for k in range(4)]
    w = mb._DENSE.pack(at, 8, 8, 8, mb.BF16)
    assert lib.muonbp_linear_quantize(ctx, d[0], ref[0]) == 2
    assert lib.muonbp_linear_restore(ctx, ref[0], d[0]) == 2
    assert lib.muonbp_linear_quantize_weight(ctx, d[0], ref[0], None) == 2
    assert lib.muonbp_linear_product(ctx, ref[0], ref[1], w, 0) == 2
    assert lib.muonbp_linear_weight_grad(ctx, ref[0], d[0], w, 0) == 2
    assert lib.muonbp_linear_gated_forward(ctx, d[0], d[1], d[2], None, ref[0], ref[1]) == 2
    assert lib.muonbp_linear_gated_backward(ctx, d[0], ref[0], ref[1], d[1], d[2], None, None) == 2
    assert b"rows" in lib.muonbp_linear_last_error(ctx) or b"large" in lib.muonbp_linear_last_error(ctx)
    x = torch.randint(-8, 9, (3, 200), device="cuda").float()
    assert torch.equal(lin.restore(lin.quantize(x), dtype=torch.float32), x)
    lin.synchronize()
    assert not bool(mem.any())


def test_the_largest_runs(lin):
    """2^32 - 256 threads, 8.6 GB of bytes."""
    import torch
    announce("largest quantize and restore")
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randint(-8, 9, (MOST, 1), generator=g, device="cuda", dtype=torch.int8).bfloat16()
    b = lin.quantize(x)
    assert torch.equal(lin.restore(b), x)
    assert not bool(b.data[::4099, 1:].any()) and not bool(b.data[-300:, 1:].any())
