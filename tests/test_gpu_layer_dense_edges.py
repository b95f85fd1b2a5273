"""Edges of the layer's products and norm that go with what surrounds them: autograd's bookkeeping, empty streams, kernels launched early."""
import math
import os
import subprocess
import sys

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


def test_first_calls_of_many_threads_at_once():
    """In a process of its own: facts of the device and set-up of the kernels are found by whoever comes first."""
    code = '''
import threading, torch
from paper_2002_02645_b200 import binding as fb
fb.load_library()
gen = torch.Generator(device="cuda").manual_seed(0)
rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
jobs = [(rand(t, k).bfloat16(), rand(n, k).bfloat16(), rand(3000, d)) for t, k, n, d in ((1, 2048, 256, 2048), (300, 1024, 1024, 4104), (50, 4096, 512, 9000), (2000, 512, 768, 1500))]
torch.cuda.synchronize()
start, got = threading.Barrier(16), [None] * 16
def work(i):
    x, w, rows = jobs[i % 4]
    start.wait()
    with torch.cuda.stream(torch.cuda.Stream()):
        got[i] = (fb.linear(x, w), *fb.linear_backward(x, w, x @ w.t())[:2], fb.layer_norm(rows), fb.layer_norm_backward(rows, None, rows)[0])
        torch.cuda.current_stream().synchronize()
threads = [threading.Thread(target=work, args=(i,)) for i in range(16)]
[t.start() for t in threads]; [t.join() for t in threads]
for i in range(16):
    x, w, rows = jobs[i % 4]
    want = (fb.linear(x, w), *fb.linear_backward(x, w, x @ w.t())[:2], fb.layer_norm(rows), fb.layer_norm_backward(rows, None, rows)[0])
    assert all(torch.equal(s, t) for s, t in zip(got[i], want)), i
print("right")
'''
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), stdout=subprocess.PIPE,
                          stderr=subprocess.STDOUT, text=True, timeout=300)
    assert done.returncode == 0 and "right" in done.stdout, done.stdout


def test_results_written_in_place_count_as_changes():
    """What a gradient still needs cannot be overwritten unnoticed, and a tensor that asks for a gradient is no place for a result."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, a = rand(gen, 64, 64).bfloat16(), rand(gen, 64, 32).bfloat16()
    w, b = rand(gen, 64, 64).bfloat16(), rand(gen, 64, 32).bfloat16()
    heads = lambda t: t.view(64, 1, 64)
    writes = [lambda t: fb.linear(a, b, out=t), lambda t: fb.linear(a, b, preact=t), lambda t: fb.layer_norm(w, out=t),
              lambda t: fb.linear_backward(None, w, x.clone(), dx=t), lambda t: fb.linear_backward(w, None, w, dweight=t),
              lambda t: fb.layer_norm_backward(w, None, w, dx=t), lambda t: fb.head_norm_rope(heads(w), None, None, None, None, None, q_out=heads(t))]
    for write in writes:
        saved, leaf = x.clone(), w.clone().requires_grad_(True)
        y = fb.linear(saved, leaf)
        write(saved)
        with pytest.raises(RuntimeError, match="inplace"):
            y.sum().backward()
        asked = x.clone().requires_grad_(True)
        with pytest.raises(ValueError, match="gradient"):
            write(asked)
        with torch.no_grad():
            write(asked)
    with torch.inference_mode():
        for write in writes:
            write(torch.empty(64, 64, device=DEV, dtype=torch.bfloat16))


def test_squares_that_float32_does_not_hold():
    """1 / sqrt(infinity) is 0: such a row comes out as the bias, in short and in long rows."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    for dim in (64, 1000, 4096):
        x, w, b = rand(gen, 1300, dim), rand(gen, dim), rand(gen, dim)
        x[3] = 1e25 * rand(gen, dim)
        y = fb.layer_norm(x, w, b)
        assert torch.equal(y[3], b) and not torch.equal(y[4], b) and not y.isnan().any()
        assert math.isfinite(fb.layer_norm_backward(x, w, torch.ones_like(x))[0][3].abs().max().item())
