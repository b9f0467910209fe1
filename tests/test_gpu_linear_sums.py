"""How products add, on the GPU against 64 bits.

A bf16 result hides its sum's error below 2^-8 of itself.  Here ``out`` starts
as the exact product rounded and negated, so that what accumulates in it is the
sum's error and that rounding's: the result c is fp32(sum) + c0 rounded to bf16.

* fp32 sums: n = K / 8 + 32 additions of exact products (eights of a matrix
  instruction, partial sums) are off by at most n 2^-24 S1, S1 = sum |a b|.
* The 8-bit matrix instructions drop, toward zero, the bits of a product below
  2^-13 of the power of two of the largest of its 8 consecutive ones.  A product of two
  values of at most 4 significant bits has none there if it is 2^-6 of the
  largest P or more (its last bit is 2^-6 of its power of two or more, which
  is above 2^-2 of it); otherwise it loses at most itself, and less than
  2^-13 P.
"""

import pytest

from tests.gpu_harness import announce

pytestmark = pytest.mark.gpu

U32, U16 = 2.0 ** -24, 2.0 ** -8


@pytest.fixture(scope="module")
def contexts():
    from paper_2510_16981_amd import muonbp as mb
    made = {False: mb.Linear(), True: mb.Linear(fp32_sums=True)}
    yield made
    for c in made.values():
        c.synchronize()
        c.close()


def _inputs(kind, m, n, k, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(m, k, generator=g, device="cuda")
    w = 0.02 * torch.randn(n, k, generator=g, device="cuda")
    if kind == "outliers":
        x *= torch.randn(k, generator=g, device="cuda").exp()
        x[:, ::97] *= 100
    if kind == "positive":
        x, w = x.abs(), w.abs()
    if kind == "cancelling":  # of every eight, three pairs cancel and two are small
        full = k // 8 * 8
        xv, wv = x[:, :full].view(m, -1, 8), w[:, :full].view(n, -1, 8)
        xv[..., 1:6:2] = -xv[..., 0:6:2]
        wv[..., 1:6:2] = wv[..., 0:6:2]
        xv[..., 6:] *= 2.0 ** -7
        wv[..., 6:] *= 2.0 ** -7
    return x, w


def _values(lin, b):
    import torch
    return lin.restore(b, dtype=torch.float32).double()


def _dropped(a, b):
    """The most that the 8-bit instructions drop of each element of a b^T."""
    import torch
    out = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device="cuda")
    for k in range(0, a.shape[1], 8):
        p = (a[:, None, k:k + 8] * b[None, :, k:k + 8]).abs()
        top = p.amax(2, keepdim=True)
        out += torch.where(p < top * 2.0 ** -6, torch.minimum(p, top * 2.0 ** -13), torch.zeros_like(p)).sum(2)
    return out


@pytest.mark.parametrize("size", [(5, 200, 1030), (40, 200, 1030), (300, 520, 1100)], ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("kind", ["normal", "positive", "outliers", "cancelling"])
@pytest.mark.parametrize("fmt", [0, 1], ids=["e4m3", "e5m2"])
@pytest.mark.parametrize("fp32", [False, True], ids=["8-bit", "fp32"])
def test_bf16_sums(contexts, size, kind, fmt, fp32):
    import torch
    announce(f"sums {size} {kind} {fmt} {fp32}")
    lin = contexts[fp32]
    m, n, k = size
    x, w = _inputs(kind, m, n, k, seed=m + fmt)
    a, b = lin.quantize(x, fmt), lin.quantize(w)
    a64, b64 = _values(lin, a), _values(lin, b)
    ref, s1 = a64 @ b64.T, a64.abs() @ b64.abs().T
    c = -ref.to(torch.bfloat16)
    want = ref + c.double()
    lin.product(a, b, out=c, accumulate=True)
    tol = (k / 8 + 32) * U32 * s1
    if not fp32:
        tol = tol + _dropped(a64, b64)
    tol = tol + U16 * (want.abs() + tol) + 1e-37
    worst = float(((c.double() - want).abs() / tol).max())
    announce(f"error over tolerance {worst:.3f}")
    assert worst <= 1


@pytest.mark.parametrize("m", [1, 16, 17, 130])
def test_products_that_cancel(contexts, m):
    """2^16 - 2^16 + 2^s in one eight: whole in fp32 sums down to s = -7 (24 bits
    below), and to s = 3 in the 8-bit instructions' 13."""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    powers = list(range(16, -8, -1))
    for s in powers:
        x = max(-9, min(8, s // 2))
        a, b = torch.zeros(m, 128, device="cuda"), torch.zeros(20, 128, device="cuda")
        a[:, 40:42], b[:, 40], b[:, 41] = 256.0, 256.0, -256.0
        a[:, 45], b[:, 45] = 2.0 ** x, 2.0 ** (s - x)

        def blocks(v):
            return mb.Blocks(v.to(torch.float8_e4m3fn).view(torch.uint8),
                             torch.full((1, v.shape[0]), 127, dtype=torch.int32, device="cuda"), 128)

        whole = contexts[True].product(blocks(a), blocks(b))
        assert bool((whole == 2.0 ** s).all()), s
        part = contexts[False].product(blocks(a), blocks(b))
        assert bool((part == (2.0 ** s if s >= 3 else part)).all()) and bool((part.abs() <= 2.0 ** s).all()), s


@pytest.mark.parametrize("size", [(1, 100, 700), (16, 333, 1030), (64, 1024, 4096), (777, 999, 1333)],
                         ids=lambda s: "%dx%dx%d" % s)
@pytest.mark.parametrize("fmt", [0, 1], ids=["e4m3", "e5m2"])
def test_fp32_sums_are_the_fp32_result_rounded(contexts, size, fmt):
    import torch
    m, n, k = size
    x, w = _inputs("outliers", m, n, k, seed=3)
    lin = contexts[True]
    a, b = lin.quantize(x, fmt), lin.quantize(w)
    assert torch.equal(lin.product(a, b), lin.product(a, b, dtype=torch.float32).bfloat16())
    c = torch.randn(m, n, device="cuda").bfloat16()
    wide = c.float()
    lin.product(a, b, out=c, accumulate=True)
    lin.product(a, b, out=wide, accumulate=True)
    assert torch.equal(c, wide.bfloat16())
