"""The 8-bit operators called while another stream than their context's is
current: ordered with it on both sides."""

import pytest

from tests.gpu_harness import announce

pytestmark = pytest.mark.gpu


@pytest.fixture()
def own():
    """A context on a stream of its own."""
    import torch
    from paper_2510_16981_amd import muonbp as mb
    ctx = mb.Linear(stream=torch.cuda.Stream())
    yield ctx
    torch.cuda.synchronize()
    ctx.close()


def _busy():
    """Some milliseconds of work on the current stream."""
    import torch
    a = torch.full((4096, 4096), 1e-3, device="cuda")
    for _ in range(20):
        a = a @ a
    return a


def test_operands_and_results_of_the_current_stream(own):
    import torch
    n = 1024
    x = torch.zeros(n, n, device="cuda")
    w = torch.eye(n, device="cuda")
    _, wt = own.quantize_weight(w)
    torch.cuda.synchronize()
    for value in (3.0, 5.0):
        _busy()
        x.fill_(value)
        y = own.product(own.quantize(x), wt, dtype=torch.float32)
        total = y.sum()  # on the current stream, which has waited for y
        assert float(total) == value * n * n


def test_memory_freed_on_the_current_stream(own):
    """An operand that is dropped as soon as the call returns, its memory taken
    by the next tensor of the current stream; a result likewise."""
    import torch
    n = 2048
    torch.cuda.synchronize()
    for k in range(4):
        a = torch.full((n, n), float(k + 1), device="cuda")
        kept = own.quantize(a)
        del a
        torch.full((n, n), -1.0, device="cuda")  # may take a's memory
        out = own.restore(kept, dtype=torch.float32)
        low, high = out.amin(), out.amax()
        del out
        own.restore(own.quantize(torch.zeros(n, n, device="cuda")), dtype=torch.float32)  # may take out's
        assert float(low) == float(high) == k + 1


def test_a_result_belongs_to_the_current_stream(own):
    """Dropped while the current stream has yet to read it, its memory is not
    taken by what the context's stream makes next."""
    import torch
    n = 2048
    kept = own.quantize(torch.full((n, n), 3.0, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(3):
        y = own.restore(kept, dtype=torch.float32)
        _busy()
        low = y.amin()
        del y
        with torch.cuda.stream(own._stream):
            taken = [torch.full((n, n), -1.0, device="cuda") for _ in range(3)]
            taken.append(own.restore(kept, dtype=torch.float32))
        assert float(low) == 3.0
        torch.cuda.synchronize()
        del taken


def test_capture_on_the_current_stream(own):
    """A graph captured on a stream that is not the context's holds the calls;
    every replay gives the eager result on the inputs of the moment."""
    import torch
    announce("capture on another stream than the context's")
    x = torch.randn(40, 1000, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(40, 300, device="cuda", dtype=torch.bfloat16)
    w8, wt8 = own.quantize_weight(torch.randn(1000, 300, device="cuda"))

    def chain():
        x8 = own.quantize(x)
        y = own.product(x8, wt8, dtype=torch.float32)
        return y + 1, own.weight_grad(x8, dy, dtype=torch.float32)

    chain()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dw = chain()
    for _ in range(4):
        x.copy_(torch.randn(40, 1000, device="cuda"))
        want_y, want_dw = chain()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(dw, want_dw)


def test_the_default_stream_is_not_captured():
    import torch
    from paper_2510_16981_amd import muonbp as mb
    lin = mb.Linear(stream=torch.cuda.default_stream())
    x, out = torch.randn(8, 256, device="cuda"), lin.empty_blocks(8, 256)
    lin.quantize(x, out=out)
    torch.cuda.synchronize()
    graph, y = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph):
        y += 1
        with pytest.raises(ValueError, match="set_stream"):
            lin.quantize(x, out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert bool((y == 1).all())
    lin.quantize(x, out=out)  # still usable
    lin.synchronize()
    lin.close()
