"""Blocks behind freeze caches run together: norm out of the residual stream, products with their epilogues, page tables, 4-bit store and
attention, branching requests; and the gradients of a block's dense half."""
import importlib.util
import os

import pytest
import torch

from paper_2002_02645_b200 import binding as fb
from test_gpu_kv_ops import plain_pack
from test_gpu_linear import act64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("freeze_decoder", os.path.join(ROOT, "examples", "freeze_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_blocks_add_to_the_survivors_rows_only_and_branches_go_on_from_their_parent():
    """Each layer against the block in 64 bits from the stream it was given and the keys and values that its store holds.  bfloat16
    roundings on the way (norm's result, qkv, q and k, attention's result, the wide product's): each off by 2^-8 of its value, which the next product
    averages; so the sums are off by 2^-8 of the size of what they add up, several times: bound 8 x 2^-8 of the root mean square of what is
    added, five times that for a single value."""
    ex = load_example()
    model = ex.FreezeDecoder(layers=2, hidden=256, q_heads=6, kv_heads=2, head_dim=64, requests=9, max_keys=64, seed=1, feed=512)
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(9, 256, generator=gen, device="cuda")
    model.calibrate(h, 0.2)
    stored = [[[] for _ in range(9)] for _ in model.layers]
    given = []

    def block64(layer, i, stream, rows, seen):
        rms = lambda t, w: t / (t.pow(2).mean(-1, keepdim=True) + 1e-5).sqrt() * w.double()
        q, k, v, a = seen
        n = len(rows)
        packed = [plain_pack(t[:n].float().cpu().numpy()) for t in (k, v)]
        kv = [torch.tensor(p[3], device="cuda").double() for p in packed]
        out = stream.double().clone()
        x = rms(out[rows], layer.attn_norm)
        qkv = (x @ layer.w_qkv.double().t()).view(n, 10, 64)
        # the values that were stored are those of this product
        assert ((v[:n].double() - qkv[:, 8:]).abs() <= 3 * 2.0 ** -8 * qkv[:, 8:].square().mean().sqrt() + 2.0 ** -8 * qkv[:, 8:].abs()).all()
        att = []
        for s, row in enumerate(rows):
            stored[i][row].append((kv[0][s], kv[1][s]))
            ks, vs = (torch.stack([t[j] for t in stored[i][row]]) for j in (0, 1))
            p = torch.softmax(torch.einsum("kgd,tkd->kgt", q[s].double().view(2, 3, 64), ks) / 8.0, -1)
            att.append(torch.einsum("kgt,tkd->kgd", p, vs).reshape(-1))
        first = torch.stack(att) @ layer.w_out.double().t()
        out[rows] += first
        u = act64(rms(out[rows], layer.feed_norm) @ layer.w_up.double().t() + layer.b_up.double(), "gelu")
        second = u @ layer.w_down.double().t() + layer.b_down.double()
        out[rows] += second
        return out, (first.square().mean() + second.square().mean()).sqrt()

    def step(h):
        streams = []
        original = [layer.run_in_place for layer in model.layers]

        def watched(i):
            def run(stream, rope, positions, rows, count):
                before = stream.clone()
                seen = original[i](stream, rope, positions, rows, count)
                live = rows[:int(count)].tolist()
                if live:
                    want, size = block64(model.layers[i], i, before, live, seen)
                    off = (stream.double() - want)[live]
                    assert off.square().mean().sqrt() <= 8 * 2.0 ** -8 * size and off.abs().max() <= 40 * 2.0 ** -8 * size
                dead = [r for r in range(9) if r not in live]
                assert torch.equal(stream[dead], before[dead])
                streams.append(len(live))
                return seen
            return run

        for i, layer in enumerate(model.layers):
            layer.run_in_place = watched(i)
        out = model.step(h)
        for layer, run in zip(model.layers, original):
            layer.run_in_place = run
        given.append(streams)
        return out

    for t in range(24):
        if t == 20:                                          # (past the first page, inside of the second)
            ended = torch.tensor([3, 7], dtype=torch.int32, device="cuda")
            for layer in model.layers:
                layer.release(ended)
                layer.gather_pages()
            granted = model.branch([0, 1], [3, 7])
            assert all(g.tolist() == [1, 1] for g in granted)
            for i, layer in enumerate(model.layers):
                for src, dst in ((0, 3), (1, 7)):
                    stored[i][dst] = list(stored[i][src])
                    full = len(stored[i][src]) // 16
                    assert torch.equal(layer.block_table[src, :full], layer.block_table[dst, :full])
                used = sorted({p for r, n in enumerate(layer.out.lens.tolist()) for p in layer.block_table[r, :-(-n // 16)].tolist()})
                free = layer.free_pages[:int(layer.out.free_count)].tolist()
                assert sorted(used + free) == list(range(36))
            h = h.clone()
            h[[3, 7]] = h[[0, 1]]
        h, _ = step(h)
        if t == 20:                                          # the same past and the same input: the same step
            assert torch.equal(h[3], h[0]) and torch.equal(h[7], h[1])
        h = 0.7 * (h + torch.randn(h.shape, generator=gen, device="cuda"))
    assert len({tuple(g) for g in given}) > 1                # some steps froze more than others
    for i, layer in enumerate(model.layers):
        layer.kv.poll_status()
        assert layer.out.lens.tolist() == [len(r) for r in stored[i]]
    fb.linear_poll_status()


def test_gradients_of_a_feed_forward_part():
    """Norm, product with activation, product with residual: backward through all of them against the formula in 64 bits.  Every tensor between
    them is rounded to bfloat16 (2^-8 of a value at most, of random sign), in both directions, five on the longest way: gradients are off by a few
    times 2^-8 of their root mean square, a single one by more: 8 and 40 of them."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, g, b = rand(300, 256), 1 + 0.1 * rand(256), 0.1 * rand(256)
    up, b_up = (rand(640, 256) / 16).bfloat16(), 0.1 * rand(640)
    down, b_down = (rand(256, 640) / 640 ** 0.5).bfloat16(), 0.1 * rand(256)
    dy = rand(300, 256)

    def loss(leaves, own):
        x, g, b, up, b_up, down, b_down = leaves
        if own:
            n = fb.layer_norm(x, g, b, out_dtype=torch.bfloat16)
            return (fb.linear(fb.linear(n, up, b_up, activation="gelu"), down, b_down, residual=x) * dy).sum()
        c = x - x.mean(-1, keepdim=True)
        n = c / (c.square().mean(-1, keepdim=True) + 1e-5).sqrt() * g + b
        return ((act64(n @ up.t() + b_up, "gelu") @ down.t() + b_down + x) * dy.double()).sum()

    tensors = (x, g, b, up, b_up, down, b_down)
    got = [t.clone().requires_grad_(True) for t in tensors]
    loss(got, True).backward()
    want = [t.double().clone().requires_grad_(True) for t in tensors]
    loss(want, False).backward()
    for a, w in zip(got, want):
        assert a.grad.dtype is a.dtype
        off, size = a.grad.double() - w.grad, w.grad.square().mean().sqrt()
        assert off.square().mean().sqrt() <= 8 * 2.0 ** -8 * size and off.abs().max() <= 40 * 2.0 ** -8 * size
    # twice the same, and captured
    again = [t.clone().requires_grad_(True) for t in tensors]
    loss(again, True).backward()
    assert all(torch.equal(a.grad, c.grad) for a, c in zip(got, again))
    leaves = [t.clone().requires_grad_(True) for t in tensors]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(loss(leaves, True), leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grads = torch.autograd.grad(loss(leaves, True), leaves)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.grad, c) for a, c in zip(got, grads))


def test_example_runs():
    ex = load_example()
    ex.sys.argv = ["freeze_decoder.py", "12"]
    ex.main()
