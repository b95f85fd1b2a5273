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


@pytest.mark.parametrize("tokens", [3, 700])
def test_preact_of_a_stream_without_rows(tokens):
    """preact is written for every real token, whatever its row: with out of no rows as with rows outside of it."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, w, bias = rand(gen, tokens, 64).bfloat16(), rand(gen, 128, 64).bfloat16(), rand(gen, 128)
    want = torch.empty(tokens, 128, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, activation="silu", preact=want)
    rows = torch.zeros(tokens, dtype=torch.int32, device=DEV)
    count = torch.tensor([tokens - 1], dtype=torch.int32, device=DEV)
    for out in (torch.empty(0, 128, device=DEV), torch.full((1, 128), 5.0, device=DEV)):
        got = torch.full_like(want, 7.0)
        where = rows if out.size(0) == 0 else rows + 1
        fb.linear(x, w, bias, activation="silu", rows=where, out=out, residual=out, preact=got, count=count)
        assert torch.equal(got[:-1], want[:-1]) and (got[-1] == 7).all() and (out == 5).all()
        fb.linear(x, w, bias, rows=where, out=out)
    fb.linear_poll_status()
