"""Captures of the layer whose inputs are no leaves."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def inputs():
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((70, 384), generator=g, device="cuda").requires_grad_()
    w = torch.randn((500, 384), generator=g, device="cuda").requires_grad_()
    return x, w, torch.randn((70, 500), generator=g, device="cuda")


@pytest.mark.parametrize("which", ["x", "weight"])
def test_inputs_of_an_eager_call_are_refused(sbw, which):
    """Their gradients would be taken on the stream of that call."""
    x, w, _ = inputs()
    eager = (x if which == "x" else w) * 2.0
    other = (w if which == "x" else x).detach()
    torch.cuda.synchronize()
    graph, refused = torch.cuda.CUDAGraph(), None
    marker = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph):
        marker.add_(1.0)                     # a graph of something
        try:
            sbw.linear_fp8(*((eager, other) if which == "x" else (other, eager)))
        except RuntimeError as error:
            refused = str(error)
    assert refused is not None and "eager graph" in refused
    graph = torch.cuda.CUDAGraph()
    want = sbw.linear_fp8(*((eager, other) if which == "x" else (other, eager))).detach()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = sbw.linear_fp8(*((eager.detach(), other) if which == "x" else (other, eager.detach())))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want)


def test_inputs_of_a_captured_call(sbw):
    """What the capture itself made is taken, with the gradients of what it was made from."""
    x, w, dy = inputs()

    def step():
        y = sbw.linear_fp8(x * 2.0, w + 1.0)
        return [y.detach(), *torch.autograd.grad(y, (x, w), dy)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        with torch.no_grad():
            x.add_(0.5), w.mul_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))
