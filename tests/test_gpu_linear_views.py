"""Blocks over parts of larger buffers."""

import pytest

from oracle import linear_oracle as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("width", [256, 257, 264, 271])
def test_rows_of_a_buffer_wider_than_its_blocks(width):
    """Rows 272 bytes apart, of which a view takes some: one row of it is taken
    as several are."""
    import numpy as np
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lin = mb.Linear()
    rng = np.random.default_rng(width)
    x = rng.standard_normal((6, 200))
    codes, e = O.quantize(x)
    data = torch.full((6, 272), 0x77, dtype=torch.uint8, device="cuda")
    data[:, :256] = torch.from_numpy(codes)
    scales = torch.from_numpy(O.words(e).view(np.int32)).cuda()
    b = mb.Blocks(data[:, :width], scales, 200)
    want = O.values(codes, e, 200)
    for rows in (slice(0, 6), slice(2, 4), slice(3, 4), slice(5, 6), slice(4, 4)):
        got = lin.restore(b[rows], dtype=torch.float32).double().cpu().numpy()
        np.testing.assert_array_equal(got, want[rows])
    w = lin.quantize(torch.from_numpy(rng.standard_normal((40, 200))).float().cuda())
    whole = lin.product(b, w, dtype=torch.float32)
    assert torch.equal(lin.product(b[3:4], w, dtype=torch.float32), whole[3:4])
    before = data.clone()
    one = b[2:3]
    lin.quantize(torch.from_numpy(x[2:3]).float().cuda(), out=one)
    assert torch.equal(data, before)
    lin.close()
