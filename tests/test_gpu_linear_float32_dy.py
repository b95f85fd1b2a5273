"""Gradients of a float32 result taken in float32: only what the products read is rounded, the bias's gradient is the sum of what dy holds.

Bounds as in the bfloat16 case: a slope is off by 16 units of 2^-23 of its parts (at most 1.5), dz for the products by 2^-8 of itself, a tensor
core's sum by (K / 16 + 4) 2^-23 of the sum of sizes, a float32 sum by 2^-24 of it for each addition, results are rounded once.
"""
import math

import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    z = z.clone().requires_grad_(True)
    y = {"none": lambda: z, "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2)), "silu": lambda: z * torch.sigmoid(z),
         "gelu_tanh": lambda: 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))}[act]()
    return torch.autograd.grad(y.sum(), z)[0].detach()


def within(got, want, bound):
    far = (got.double() - want).abs()
    assert (far <= bound).all(), (far / bound).max()


def check(x, w, dy, preact, act, got):
    g = dy.double() * (1.0 if act == "none" else slope64(preact.double(), act))
    off = (0.0 if act == "none" else 16 * 1.5 * 2.0 ** -23) * dy.double().abs()
    each, (tokens, n_out) = off + 2.0 ** -8 * (g.abs() + off), dy.shape
    dx, dw, db = got
    for result, left, err, right, k in ((dx, g, each, w.double(), n_out), (dw, g.t(), each.t(), x.double(), tokens)):
        if result is not None:
            want = left @ right
            bound = err @ right.abs() + (k / 16 + 4) * 2.0 ** -23 * ((left.abs() + err) @ right.abs())
            within(result, want, (1 + 2.0 ** -8) * bound + 2.0 ** -8 * want.abs() + 1e-37)
    if db is not None:
        within(db, g.sum(0), off.sum(0) + (tokens + 1) * 2.0 ** -24 * (g.abs() + off).sum(0) + 1e-37)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 8, 8), (3, 72, 136), (65, 200, 72), (777, 520, 1400), (1500, 136, 328), (4095, 1024, 2048)])
def test_against_the_formulas(tokens, n_in, n_out, act):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w = rand(gen, tokens, n_in).bfloat16(), (rand(gen, n_out, n_in) * n_in ** -0.5).bfloat16()
    dy, preact = rand(gen, tokens, n_out), (3 * rand(gen, tokens, n_out)).bfloat16()
    kw = dict(preact=None if act == "none" else preact, activation=act, dy_dtype=torch.float32)
    got = fb.linear_backward(x, w, dy, with_bias=True, **kw)
    assert [t.dtype for t in got] == [torch.bfloat16, torch.bfloat16, torch.float32]
    check(x, w, dy, preact, act, got)
    for a, b, bias in ((None, w, False), (x, None, True), (None, None, True)):           # each alone
        part = fb.linear_backward(a, b, dy, with_bias=bias, **kw)
        check(x, w, dy, preact, act, part)
        assert [t is None for t in part] == [b is None, a is None, not bias]
    # rows apart from one another
    wide = torch.full((tokens, n_out + 12), math.nan, device=DEV)
    wide[:, 8:8 + n_out] = dy
    again = fb.linear_backward(x, w, wide[:, 8:8 + n_out], with_bias=True, **kw)
    assert all(torch.equal(s, t) for s, t in zip(got, again))
    fb.linear_poll_status()


@pytest.mark.parametrize("act", ["none", "silu"])
def test_autograd_takes_it_where_it_is_asked_for(act):
    gen = torch.Generator(device=DEV).manual_seed(9)
    x, w = rand(gen, 300, 136).bfloat16(), rand(gen, 264, 136).bfloat16()
    bias, r, dy = rand(gen, 264), rand(gen, 300, 264), rand(gen, 300, 264)
    z = torch.empty(300, 264, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, preact=z)
    for given in (dy, dy.t().contiguous().t(), dy[:1].expand(300, 264)):
        leaves = [t.clone().requires_grad_(True) for t in (x, w, bias, r)]
        fb.linear(leaves[0], leaves[1], leaves[2], activation=act, residual=leaves[3], grad_dtype=torch.float32).backward(given)
        want = fb.linear_backward(x, w, given.contiguous(), preact=z, activation=act, with_bias=True, dy_dtype=torch.float32)
        assert all(torch.equal(leaf.grad, g) for leaf, g in zip(leaves, (*want, given)))
    # a bfloat16 result has a bfloat16 gradient
    leaf = w.clone().requires_grad_(True)
    fb.linear(x, leaf, activation=act, grad_dtype=torch.float32).sum().backward()
    fb.linear(x, w, preact=z)
    assert torch.equal(leaf.grad, fb.linear_backward(x, None, torch.ones(300, 264, device=DEV).bfloat16(), preact=z, activation=act)[1])


def test_captured_and_empty_and_refused():
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, w, dy = rand(gen, 200, 64).bfloat16(), rand(gen, 72, 64).bfloat16(), rand(gen, 200, 72)
    z, wide = rand(gen, 200, 72).bfloat16(), dict(with_bias=True, dy_dtype=torch.float32)
    want = fb.linear_backward(x, w, dy, **wide)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = fb.linear_backward(x, w, dy, **wide)
    dy.mul_(2)                                              # exact
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(s, 2 * t) for s, t in zip(got, want))
    dx, dw, db = fb.linear_backward(x[:0], w, dy[:0], preact=z[:0], activation="silu", **wide)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    off = torch.zeros(200 * 72 + 1, device=DEV)[1:].view(200, 72)
    for call in (lambda: fb.linear_backward(x, w, off, **wide), lambda: fb.linear_backward(x, w, torch.zeros(200, 73, device=DEV)[:, :72], **wide)):
        with pytest.raises(fb.FiError, match="INVALID"):
            call()
    for call in (lambda: fb.linear_backward(x, w, dy), lambda: fb.linear_backward(x, w, dy.bfloat16(), **wide), lambda: fb.linear(x, w, grad_dtype=torch.float16),
                 lambda: fb.linear_backward(x, w, dy.half(), dy_dtype=torch.float16)):
        with pytest.raises(ValueError):
            call()
