"""Errors around the 8-bit operators: whose they are, and what they leave."""

import pytest

pytestmark = pytest.mark.gpu


def test_an_error_of_an_earlier_call_is_not_the_launches():
    """A refused call of the program's own leaves an error on the thread; the
    operators run, and leave it there."""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lin = mb.Linear()
    x, w = torch.randn(40, 256, device="cuda"), torch.randn(256, 48, device="cuda")
    dy = torch.randn(40, 48, device="cuda", dtype=torch.bfloat16)
    x8 = lin.quantize(x)
    w8, wt8 = lin.quantize_weight(w)
    g, g8, u8 = lin.gated_forward(x, x)
    calls = {"quantize": lambda: lin.quantize(x, out=x8), "quantize_weight": lambda: lin.quantize_weight(w),
             "restore": lambda: lin.restore(x8), "product": lambda: lin.product(x8, wt8),
             "product of few rows": lambda: lin.product(x8[:1], wt8), "weight_grad": lambda: lin.weight_grad(x8, dy),
             "gated_forward": lambda: lin.gated_forward(x, x), "gated_backward": lambda: lin.gated_backward(x, g8, u8)}
    for name, call in calls.items():
        call()  # what it allocates is in the allocator's cache from here on
        torch.cuda.synchronize()
        assert lin.lib.hipSetDevice(1 << 20) == 101  # no such device
        try:
            call()
        finally:
            left = lin.lib.hipGetLastError()
        assert left == 101, name
    lin.synchronize()
    assert torch.equal(lin.gated_forward(x, x)[0], g)
    lin.close()
