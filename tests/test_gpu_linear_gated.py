"""The gated activation's gradients in 8 bits alone, through the C entry point."""

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 1), (1, 4096), (3, 1000), (77, 1554), (130, 512)], ids=lambda s: "%dx%d" % s)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kept", [0, 1], ids=["e4m3", "e5m2"])
@pytest.mark.parametrize("fmt", [0, 1], ids=["to e4m3", "to e5m2"])
def test_gradients_in_8_bits_alone(shape, dtype, kept, fmt):
    """The bytes and scales that a call gives beside the dense gradients."""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lin = mb.Linear()
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator(device="cuda").manual_seed(shape[1])
    gate, up, dh = (torch.randn(shape, generator=g, device="cuda").to(t) for _ in range(3))
    _, gate8, up8 = lin.gated_forward(gate, up, format=kept)
    _, _, want_gate, want_up = lin.gated_backward(dh, gate8, up8, blocks=True, format=fmt)
    got_gate, got_up = lin.empty_blocks(*shape, fmt), lin.empty_blocks(*shape, fmt)
    for b in (got_gate, got_up):
        b.data.fill_(0x55)
        b.scales.fill_(-1)
    assert lin.lib.muonbp_linear_gated_backward(lin.ctx, lin._dense(dh, "dh"), gate8.ref, up8.ref, None, None,
                                                got_gate.ref, got_up.ref) == 0
    for got, want in ((got_gate, want_gate), (got_up, want_up)):
        assert torch.equal(got.data, want.data) and torch.equal(got.scales, want.scales)
    lin.close()
