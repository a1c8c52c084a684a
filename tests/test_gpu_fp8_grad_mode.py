"""The layer without gradients: under torch.no_grad(), or of inputs that require none."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def inputs(M=70, N=500, K=384):
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn((N, K), generator=g, device="cuda")
    return x, w


@pytest.mark.parametrize("M", [0, 1, 70, 300])
@pytest.mark.parametrize("dtype", [None, torch.float32])
def test_same_result(sbw, M, dtype):
    x, w = inputs(M)
    leaf = w.clone().requires_grad_()
    want = sbw.linear_fp8(x, leaf, dtype)
    assert want.requires_grad
    with torch.no_grad():
        got = sbw.linear_fp8(x, leaf, dtype)
    plain = sbw.linear_fp8(x, w, dtype)
    with torch.inference_mode():
        inference = sbw.linear_fp8(x, w, dtype)
    for y in (got, plain, inference):
        assert not y.requires_grad and y.dtype == want.dtype and torch.equal(y, want)


def test_nothing_is_made_for_a_backward_pass(sbw, monkeypatch):
    from paper_2609_03844_amd import fp8
    x, w = inputs()
    w.requires_grad_()
    orientations = []
    quantized = fp8._quantized

    def spy(x, block_rows, scale_dtype, straight, transposed, *rest):
        orientations.append((straight, transposed))
        return quantized(x, block_rows, scale_dtype, straight, transposed, *rest)
    monkeypatch.setattr(fp8, "_quantized", spy)
    with torch.no_grad():
        sbw.linear_fp8(x, w)
    assert orientations and all(transposed is None for _, transposed in orientations)


def test_captured_while_an_eager_graph_is_alive(sbw):
    """A forward pass alone has no backward pass that would wait for the eager one's stream."""
    x, w = inputs()
    w.requires_grad_()
    eager = sbw.linear_fp8(x, w)
    with torch.no_grad():
        want = sbw.linear_fp8(x, w)
    torch.cuda.synchronize()
    graph, refused, held = torch.cuda.CUDAGraph(), None, None
    marker = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph):
        marker.add_(1.0)                     # a graph of something, were the call refused
        with torch.no_grad():
            try:
                held = sbw.linear_fp8(x, w)
            except RuntimeError as error:
                refused = str(error)
    assert refused is None
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, want)
        with torch.no_grad():
            x.add_(0.25)
            want = sbw.linear_fp8(x, w)
    assert torch.equal(torch.autograd.grad(eager, w, torch.zeros_like(eager))[0], torch.zeros_like(w))
