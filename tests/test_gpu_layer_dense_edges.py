"""Edges of the layer's products and norm that go with what surrounds them: autograd's bookkeeping, empty streams, kernels launched early."""
import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


@pytest.mark.parametrize("rows,dim", [(5, 1000), (5, 4096), (2000, 2048)])
def test_norm_by_weights_that_the_kernel_before_wrote(rows, dim):
    """A conditional norm: weight and bias are what a product has just written in float32.  Replayed, so that launches follow at once."""
    gen = torch.Generator(device=DEV).manual_seed(dim)
    c, w, wb = rand(gen, 1, 64).bfloat16(), rand(gen, dim, 64).bfloat16(), rand(gen, dim, 64).bfloat16()
    x, dy = rand(gen, rows, dim), rand(gen, rows, dim)
    scale, shift = torch.zeros(1, dim, device=DEV), torch.zeros(1, dim, device=DEV)
    graph = torch.cuda.CUDAGraph()

    def step():
        fb.linear(c, wb, out=shift)
        fb.linear(c, w, out=scale)
        y = fb.layer_norm(x, scale[0], shift[0])
        return y, *fb.layer_norm_backward(x, scale[0], dy)[:2]
    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(20):
        c.mul_(-1 if i % 3 else 0.5)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        s, b = scale[0].clone(), shift[0].clone()
        assert s.any()
        torch.cuda.synchronize()
        assert torch.equal(kept[0], fb.layer_norm(x, s, b)) and all(torch.equal(p, q) for p, q in zip(kept[1:], fb.layer_norm_backward(x, s, dy)))
