"""A step of the layer only enqueues kernels: it can be captured, and its replays follow new inputs."""
import pytest
import torch

from paper_1503_05032_amd.layer import Layer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def captured(work):
    """A graph of work(), and the outputs that its replays write."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = work()
    return graph, outs


@pytest.mark.parametrize("tokens", [1, 5, 70])
@pytest.mark.parametrize("kind", ["serve", "train"])
def test_replays_of_a_captured_step(kind, tokens):
    g = torch.Generator().manual_seed(tokens)
    layer = Layer(width=256, inner=136, experts=6, k=2, generator=g)
    eight = layer.for_serving()
    draw = lambda: torch.randn(tokens, layer.width, generator=g).to(DEV, layer.dtype)  # noqa: E731
    x, residual, dy = draw(), draw(), draw()

    def work():
        if kind == "serve":
            return [layer.serve(x, eight, residual)]
        y, saved = layer.forward(x, residual)
        dx, grads = layer.backward(dy, saved)
        return [y, dx, *grads.values()]

    graph, outs = captured(work)
    for turn in range(3):
        for t in (x, residual, dy):
            t.copy_(draw())
        want = [t.clone() for t in work()]
        for t in outs:
            t.fill_(9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), turn
