"""Results in memory that the caller gives: of its own type and format, and
refused where another was asked for."""

import pytest

pytestmark = pytest.mark.gpu


def test_out_of_another_type_than_asked_for():
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lin = mb.Linear()
    x, w = torch.randn(20, 256, device="cuda"), torch.randn(256, 48, device="cuda")
    dy = torch.randn(20, 48, device="cuda", dtype=torch.bfloat16)
    e4, e5 = lin.empty_blocks(20, 256), lin.empty_blocks(20, 256, mb.E5M2)
    with pytest.raises(ValueError, match="format"):
        lin.quantize(x, mb.E5M2, out=e4)
    with pytest.raises(ValueError, match="format"):
        lin.quantize(x, mb.E4M3, out=e5)
    w4, w5t = lin.empty_blocks(256, 48), lin.empty_blocks(48, 256, mb.E5M2)
    for args in ({"out": w4, "out_t": w5t}, {"out": w4, "format": mb.E5M2}, {"out_t": w5t, "format": mb.E4M3}):
        with pytest.raises(ValueError, match="format"):
            lin.quantize_weight(w, **args)
    # No format asked for: the given one's, for both layouts.
    assert torch.equal(lin.quantize(x, out=e5).data, lin.quantize(x, mb.E5M2).data)
    both, want = lin.quantize_weight(w, out_t=w5t), lin.quantize_weight(w, mb.E5M2)
    for got, ref in zip(both, want):
        assert got.format == mb.E5M2 and torch.equal(got.data, ref.data) and torch.equal(got.scales, ref.scales)
    x8, (_, wt8) = lin.quantize(x), lin.quantize_weight(w)
    for call, shape in ((lambda **k: lin.restore(x8, **k), (20, 256)), (lambda **k: lin.product(x8, wt8, **k), (20, 48)),
                        (lambda **k: lin.weight_grad(x8, dy, **k), (256, 48))):
        for have, asked in ((torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)):
            out = torch.full(shape, 7.0, device="cuda", dtype=have)
            with pytest.raises(ValueError, match="not torch"):
                call(out=out, dtype=asked)
            assert bool((out == 7).all())
            assert torch.equal(call(out=out), call(dtype=have))
            assert torch.equal(call(out=out, dtype=have), out)
    lin.close()
