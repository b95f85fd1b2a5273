"""Norm of whole rows (fi_layer_norm) and its gradients against the formulas in 64 bits.

Bounds (u = 2^-24).  A sum over a row passes at most 42 additions one after another, so a mean is off by 44 u of the mean of sizes (e); 1/s by
e / s + 50 u + 2^-22 of itself; n by that of itself and e / s; results by a few u of their parts and one rounding to their type.
"""
import math

import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}
TYPES = [(a, b) for a in (torch.bfloat16, torch.float32) for b in (torch.bfloat16, torch.float32)]
DIMS = [1, 2, 3, 7, 8, 16, 31, 33, 100, 255, 256, 257, 512, 520, 1000, 1001, 1024, 1025, 1032, 2048, 2056, 4095, 4096, 5000, 8192, 8200, 16383, 16384]


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def parts(x, rms, eps):
    """n, its error, 1/s, its relative error."""
    x = x.double()
    mean = x.mean(-1, keepdim=True) * (0 if rms else 1)
    e = (0 if rms else 44 * U) * x.abs().mean(-1, keepdim=True)
    d = x - mean
    r = 1 / ((d * d).mean(-1, keepdim=True) + eps).sqrt()
    rel = e * r + 50 * U + 2.0 ** -22
    n = d * r
    return n, n.abs() * (rel + 2 * U) + e * r, r, rel


def forward(x, w, b, rms, eps, dtype):
    n, off, _, _ = parts(x, rms, eps)
    w = torch.ones(x.shape[1], device=DEV).double() if w is None else w.double()
    b = torch.zeros(x.shape[1], device=DEV).double() if b is None else b.double()
    y = n * w + b
    bound = off * w.abs() + 4 * U * ((n * w).abs() + b.abs())
    return y, (1 + HALF[dtype]) * bound + HALF[dtype] * y.abs() + 1e-38


def within(got, want, bound):
    far = (got.double() - want).abs()
    assert (far <= bound).all(), (far / bound).max()


def check_backward(x, w, dy, rms, eps, with_bias, dx=None):
    got = fb.layer_norm_backward(x, w, dy, eps=eps, rms=rms, with_bias=with_bias, dx=dx)
    n, off, r, rel = parts(x, rms, eps)
    g = dy.double() if w is None else dy.double() * w.double()
    mean = lambda t: t.mean(-1, keepdim=True)
    c1, c2 = mean(g) * (0 if rms else 1), mean(g * n)
    e1, e2 = 45 * U * mean(g.abs()), 46 * U * mean((g * n).abs()) + mean(g.abs() * off)
    want = r * (g - c1 - n * c2)
    bound = r * (U * g.abs() + e1 + off * c2.abs() + n.abs() * e2 + 4 * U * (g.abs() + c1.abs() + (n * c2).abs())) + rel * want.abs()
    within(got[0], want, (1 + HALF[x.dtype]) * bound + HALF[x.dtype] * want.abs() + 1e-38)
    tokens = x.shape[0] + 50
    if w is not None:
        dn = dy.double() * n
        within(got[1], dn.sum(0), (dy.double().abs() * off).sum(0) + tokens * U * dn.abs().sum(0) + 1e-38)
    else:
        assert got[1] is None
    if with_bias:
        within(got[2], dy.double().sum(0), tokens * U * dy.double().abs().sum(0) + 1e-38)
    else:
        assert got[2] is None
    return got


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
def test_dims(dim, types):
    gen = torch.Generator(device=DEV).manual_seed(dim)
    for tokens, rms in ((1, False), (5, True), (67, False)):
        x = (rand(gen, tokens, dim) * (1 + rand(gen, dim).abs()) + 2 * rand(gen, dim)).to(types[0])
        w, b = 1 + 0.2 * rand(gen, dim), rand(gen, dim)
        y = fb.layer_norm(x, w, b, rms=rms, out_dtype=types[1])
        assert y.dtype is types[1]
        within(y, *forward(x, w, b, rms, 1e-5, types[1]))
        dy = rand(gen, tokens, dim).to(types[1])
        a = check_backward(x, w, dy, rms, 1e-5, True)
        c = fb.layer_norm_backward(x, w, dy, rms=rms, with_bias=True)
        assert all(torch.equal(s, t) for s, t in zip(a, c))


@pytest.mark.parametrize("tokens,dim", [(3001, 1001), (8191, 512), (2000, 4096), (40000, 64), (700, 16384), (1200, 8192)])
@pytest.mark.parametrize("rms", [False, True])
def test_many_rows(tokens, dim, rms):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w, b = rand(gen, tokens, dim).bfloat16(), 1 + 0.2 * rand(gen, dim), rand(gen, dim)
    within(fb.layer_norm(x, w, b, rms=rms), *forward(x, w, b, rms, 1e-5, torch.bfloat16))
    check_backward(x, w, rand(gen, tokens, dim).bfloat16(), rms, 1e-5, not rms)
    fb.layer_norm_poll_status()


@pytest.mark.parametrize("dim", [64, 1000, 4096])
def test_without_weight_or_bias_and_eps(dim):
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, w, b = rand(gen, 33, dim), rand(gen, dim), rand(gen, dim)
    for args in ((None, None), (w, None), (None, b)):
        for eps in (0.0, 1e-6, 3.0):
            within(fb.layer_norm(x, *args, eps=eps), *forward(x, *args, False, eps, torch.float32))
    dy = rand(gen, 33, dim)
    check_backward(x, None, dy, False, 1e-5, True)
    check_backward(x, None, dy, True, 1e-5, False)


@pytest.mark.parametrize("dim", [8, 100, 4096, 9000])
def test_large_means_small_spreads_and_equal_values(dim):
    """The deviations are squared once the mean is known: a mean 1,000 times the spread costs what its own error does, no more; a row of
    equal values has no spread and gives the bias."""
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, w, b = 1000 + rand(gen, 20, dim), 1 + 0.2 * rand(gen, dim), rand(gen, dim)
    within(fb.layer_norm(x, w, b), *forward(x, w, b, False, 1e-5, torch.float32))
    x[3] = 8.0
    x[5] = 0.0
    y = fb.layer_norm(x, w, b)
    assert torch.equal(y[3], b) and torch.equal(y[5], b)
    assert not fb.layer_norm(x, w, rms=True)[5].any()
    for big in (1e15, 1e-15):
        z = big * rand(gen, 7, dim)
        within(fb.layer_norm(z, w, b, eps=0.0 if big > 1 else 1e-38), *forward(z, w, b, False, 0.0 if big > 1 else 1e-38, torch.float32))


@pytest.mark.parametrize("tokens,alive", [(1, 0), (9, 9), (256, 251), (300, 7)])
@pytest.mark.parametrize("dim", [96, 1001, 4096])
def test_rows_and_count(tokens, alive, dim):
    gen = torch.Generator(device=DEV).manual_seed(alive)
    batch = tokens + 50
    x, w, b = rand(gen, batch, dim), 1 + 0.2 * rand(gen, dim), rand(gen, dim)
    rows = torch.randperm(batch, generator=gen, device=DEV)[:tokens].int()
    x[rows[alive:].long()] = math.nan
    out = torch.full((tokens, dim), 7.0, device=DEV).bfloat16()
    count = torch.tensor([alive], dtype=torch.int32, device=DEV)
    assert fb.layer_norm(x, w, b, rows=rows, count=count, out=out) is out
    within(out[:alive], *forward(x[rows[:alive].long()], w, b, False, 1e-5, torch.bfloat16))
    assert (out[alive:] == 7).all()
    # the same row twice is read twice; rows outside of x are left out
    again = torch.cat([rows[:1], rows[:1], rows.new_tensor([-1, batch])])
    x[rows[:1].long()] = 1.0 + rand(gen, dim)
    y = fb.layer_norm(x, w, b, rows=again, out=torch.full((4, dim), 7.0, device=DEV))
    assert torch.equal(y[0], y[1]) and (y[2:] == 7).all()
    within(y[:1], *forward(x[rows[:1].long()], w, b, False, 1e-5, torch.float32))
    for n in (-1, 10 ** 6):
        y = fb.layer_norm(x, w, b, count=torch.tensor([n], dtype=torch.int32, device=DEV), out=torch.full((batch, dim), 7.0, device=DEV))
        assert (y == 7).all() if n < 0 else not (y[rows[:1].long()] == 7).all()


@pytest.mark.parametrize("dim", [5, 8, 24, 32, 40, 64, 100, 128, 136])
@pytest.mark.parametrize("tokens", [1, 3, 17, 5001])
def test_short_rows_side_by_side(tokens, dim):
    """Rows that share a warp: one of NaN, one outside of x and the places past the last row leave the others as they are, also without eps."""
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x, w, b, dy = rand(gen, tokens, dim), 1 + 0.2 * rand(gen, dim), rand(gen, dim), rand(gen, tokens, dim)
    for rms in (False, True):
        check_backward(x, w, dy, rms, 0.0, True)
        want, bound = forward(x, w, b, rms, 0.0, torch.float32)
        rows = torch.arange(tokens, device=DEV).int()
        bad = torch.arange(tokens, device=DEV) % 3 == 1
        rows[bad] = tokens
        y = fb.layer_norm(x, w, b, eps=0.0, rms=rms, rows=rows, out=torch.full((tokens, dim), 7.0, device=DEV))
        within(y[~bad], want[~bad], bound[~bad])
        assert (y[bad] == 7).all()
        z = x.clone()
        z[bad] = math.nan
        y = fb.layer_norm(z, w, b, eps=0.0, rms=rms)
        within(y[~bad], want[~bad], bound[~bad])
        assert y[bad].isnan().all()
        dx = fb.layer_norm_backward(z, w, dy, eps=0.0, rms=rms)[0]
        assert dx[bad].isnan().all() and torch.equal(dx[~bad], fb.layer_norm_backward(x, w, dy, eps=0.0, rms=rms)[0][~bad])


@pytest.mark.parametrize("tokens,dim", [(9000, 1024), (1, 520), (4001, 776), (7000, 2048), (4999, 1032), (3000, 1500), (1500, 4100)])
def test_more_rows_than_run_at_one_time(tokens, dim):
    gen = torch.Generator(device=DEV).manual_seed(dim)
    for types, rms in ((TYPES[0], False), (TYPES[-1], True)):
        x, w, b = rand(gen, tokens, dim).to(types[0]), 1 + 0.2 * rand(gen, dim), rand(gen, dim)
        within(fb.layer_norm(x, w, b, rms=rms, out_dtype=types[1]), *forward(x, w, b, rms, 1e-5, types[1]))
        check_backward(x, w, rand(gen, tokens, dim).to(types[1]), rms, 1e-5, True)
    fb.layer_norm_poll_status()


def test_strides_alignment_and_in_place():
    gen = torch.Generator(device=DEV).manual_seed(4)
    wide, wb = rand(gen, 40, 1300), rand(gen, 2101)
    for start, dim in ((0, 1000), (4, 1024), (1, 1024), (3, 37)):
        x, w, b = wide[:, start:start + dim], wb[start:start + dim], wb[1000 + start:1000 + start + dim]
        big = torch.full((40, 1111), 5.0, device=DEV).bfloat16()
        out = big[:, 8:8 + dim]
        fb.layer_norm(x, w, b, out=out)
        within(out, *forward(x, w, b, False, 1e-5, torch.bfloat16))
        assert (big[:, :8] == 5).all() and (big[:, 8 + dim:] == 5).all()
        plain = fb.layer_norm(x, w, b)
        copy = wide.clone()
        fb.layer_norm(copy[:, start:start + dim], w, b, out=copy[:, start:start + dim])
        assert torch.equal(copy[:, start:start + dim], plain)
        dy = rand(gen, 40, 1300)
        ref = check_backward(x, w, dy[:, start:start + dim], False, 1e-5, True)
        into = dy.clone()[:, start:start + dim]
        got = fb.layer_norm_backward(x, w, into, with_bias=True, dx=into)
        assert all(torch.equal(a, c) for a, c in zip(ref, got))


def test_nan_and_infinity_stay_in_their_rows():
    gen = torch.Generator(device=DEV).manual_seed(5)
    for dim in (64, 4096):
        x, w, b = rand(gen, 10, dim), rand(gen, dim), rand(gen, dim)
        clean = fb.layer_norm(x, w, b)
        x[2, 3], x[4, 0] = math.nan, math.inf
        y = fb.layer_norm(x, w, b)
        assert y[2].isnan().all() and y[4].isnan().any()
        keep = [0, 1, 3, 5, 6, 7, 8, 9]
        assert torch.equal(y[keep], clean[keep])


def test_empty():
    x, w = torch.zeros(0, 64, device=DEV), torch.ones(64, device=DEV)
    assert fb.layer_norm(x, w).shape == (0, 64)
    dx, dw, db = fb.layer_norm_backward(x, w, x, with_bias=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()
    out = torch.full((3, 64), 2.0, device=DEV)
    rows = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert (fb.layer_norm(x, w, rows=rows, out=out) == 2).all()


@pytest.mark.parametrize("rms", [False, True])
def test_autograd_and_differences(rms):
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, w, b, dy = rand(gen, 30, 200), 1 + 0.2 * rand(gen, 200), rand(gen, 200), rand(gen, 30, 200)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    fb.layer_norm(*leaves, rms=rms).backward(dy)
    want = fb.layer_norm_backward(x, w, dy, rms=rms, with_bias=True)
    assert all(torch.equal(leaf.grad, g) for leaf, g in zip(leaves, want))

    def value(x, w, b):
        c = x if rms else x - x.mean(-1, keepdim=True)
        return ((c / ((c * c).mean(-1, keepdim=True) + 1e-5).sqrt() * w + b) * dy.double()).sum()

    base = [t.double() for t in (x, w, b)]
    for i, grad in enumerate(want):
        d = rand(gen, *base[i].shape).double()
        h = 1e-5
        up, down = ([t + s * h * d if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        slope = (value(*up) - value(*down)) / (2 * h)
        # gradients to float32 (200 u of their size); differences to h^2 of third derivatives and 2^-52 / h of the value
        assert abs((grad.double() * d).sum() - slope) <= 200 * U * (grad.double() * d).abs().sum() + 1e-6 * slope.abs() + 1e-6
    # an expanded gradient, a frozen bias, a bfloat16 result
    x2 = x.clone().requires_grad_(True)
    fb.layer_norm(x2, w, b, rms=rms, out_dtype=torch.bfloat16).sum().backward()
    assert torch.equal(x2.grad, fb.layer_norm_backward(x, w, torch.ones(30, 200, device=DEV).bfloat16(), rms=rms)[0])
    for kw in (dict(out=torch.empty_like(x)), dict(count=torch.ones(1, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError, match="gradient"):
            fb.layer_norm(x2, w, **kw)


def test_streams_and_capture():
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, w, b, dy = rand(gen, 500, 4096).bfloat16(), rand(gen, 4096), rand(gen, 4096), rand(gen, 500, 4096).bfloat16()
    y, ref = fb.layer_norm(x, w, b), fb.layer_norm_backward(x, w, dy, with_bias=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert torch.equal(fb.layer_norm(x, w, b), y)
        got = fb.layer_norm_backward(x, w, dy, with_bias=True)
    s.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(ref, got))
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        r1 = fb.layer_norm_backward(x, w, dy, with_bias=True)
    with torch.cuda.graph(g2):
        r2 = fb.layer_norm_backward(x[:77], w, dy[:77], with_bias=True)
    g1.replay(); g2.replay(); g1.replay(); g2.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(ref, r1))
    assert all(torch.equal(a, c) for a, c in zip(fb.layer_norm_backward(x[:77], w, dy[:77], with_bias=True), r2))


def test_offsets_past_32_bits():
    """140,000 rows of 16,384 values, and their last ones in other forms."""
    gen = torch.Generator(device=DEV).manual_seed(12)
    tokens, dim = 140000, 16384
    x = torch.zeros(tokens, dim, dtype=torch.bfloat16, device=DEV)
    last = torch.arange(tokens - 40, tokens, device=DEV)
    x[last] = rand(gen, 40, dim).bfloat16()
    w, b, dy = 1 + 0.2 * rand(gen, dim), rand(gen, dim), torch.zeros_like(x)
    dy[last] = rand(gen, 40, dim).bfloat16()
    want = forward(x[last], w, b, False, 1e-5, torch.bfloat16)
    within(fb.layer_norm(x, w, b)[last], *want)
    within(fb.layer_norm(x, w, b, rows=last.int()), *want)
    dx, dw, _ = fb.layer_norm_backward(x, w, dy)
    alone = fb.layer_norm_backward(x[last].clone(), w, dy[last].clone())
    assert torch.equal(dx[last], alone[0])
    n, off, _, _ = parts(x[last], False, 1e-5)
    d = dy[last].double()
    within(dw, (d * n).sum(0), (d.abs() * off).sum(0) + 90 * U * (d * n).abs().sum(0) + 1e-38)
    fb.layer_norm_poll_status()


def test_refusals():
    x, w = torch.zeros(4, 64, device=DEV), torch.zeros(64, device=DEV)
    ints = torch.zeros(4, dtype=torch.int32, device=DEV)
    bad = [lambda: fb.layer_norm(x.half(), w), lambda: fb.layer_norm(x[0], w), lambda: fb.layer_norm(x.cpu(), w.cpu()), lambda: fb.layer_norm(x, w[:63]),
           lambda: fb.layer_norm(x, w.bfloat16()), lambda: fb.layer_norm(x, w, w.cpu()), lambda: fb.layer_norm(x.t(), w[:4]),
           lambda: fb.layer_norm(x, w, out_dtype=torch.float16), lambda: fb.layer_norm(x, w, rows=ints.long()),
           lambda: fb.layer_norm(x, w, out=torch.zeros(3, 64, device=DEV)), lambda: fb.layer_norm(x, w, count=ints.float()),
           lambda: fb.layer_norm_backward(x, w, x[:3]), lambda: fb.layer_norm_backward(x, w, x, dx=x.bfloat16())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(2, 16392, device=DEV)
    unsound = [lambda: fb.layer_norm(wide), lambda: fb.layer_norm(x[:1].expand(4, 64), w), lambda: fb.layer_norm(torch.zeros(4, 0, device=DEV)),
               lambda: fb.layer_norm(x, w, out=torch.zeros(300, device=DEV).as_strided((4, 64), (32, 1)))]
    for call in unsound:
        with pytest.raises(fb.FiError, match="INVALID"):
            call()
