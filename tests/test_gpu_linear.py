"""The products of a layer (fi_linear) and their gradients against the formulas in 64 bits.

Bounds.  A sum of K products on the tensor cores is cut after each 16 of them: off by (K / 16 + 4) 2^-23 of the sum of sizes at most.
An activation has a slope of at most 1.13 and is itself off by 8 units of 2^-23 of 1 + |y| (exponential and error function as documented,
a few roundings of their arguments).  A result is rounded once: 2^-8 of itself in bfloat16, 2^-24 in float32.
"""
import math

import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    z = z.clone().requires_grad_(True)
    g, = torch.autograd.grad(act64(z, act).sum(), z)
    return torch.where(z > 0, 1.0, 0.0).double() if act == "relu" else g.detach()


def sums(x, w):
    """x w^T in 64 bits and how far the tensor cores may be from it."""
    k = x.shape[1]
    return x.double() @ w.double().t(), (k / 16 + 4) * 2.0 ** -23 * (x.double().abs() @ w.double().abs().t())


def expected(x, w, bias, act, residual, dtype):
    z, off = sums(x, w)
    if bias is not None:
        z = z + bias.double()
    y = act64(z, act)
    bound = 1.13 * off + 2.0 ** -22 * z.abs() + (8 * 2.0 ** -23 * (1 + y.abs()) if act not in ("none", "relu") else 0)
    if residual is not None:
        y = y + residual.double()
        bound = bound + 2.0 ** -22 * y.abs()
    return y, (1 + HALF[dtype]) * bound + HALF[dtype] * y.abs() + 1e-37


def within(got, want, bound):
    far = (got.double() - want).abs()
    assert (far <= bound).all(), (far / bound).max()


def operands(gen, tokens, n_in, n_out):
    return rand(gen, tokens, n_in).bfloat16(), (rand(gen, n_out, n_in) * n_in ** -0.5).bfloat16()


SIZES = [(1, 8, 8), (1, 4096, 1000), (2, 64, 128), (5, 72, 136), (15, 200, 120), (16, 128, 256), (17, 4096, 384), (33, 1000, 264), (64, 512, 1024),
         (65, 2048, 520), (127, 640, 2560), (128, 8192, 128), (129, 136, 1400), (255, 264, 72), (256, 1024, 1024), (257, 320, 648), (500, 96, 2048),
         (1000, 1512, 8), (1025, 776, 1288), (2311, 408, 600), (4099, 192, 136), (1, 16384, 2048), (7, 8, 16384), (31, 16384, 8)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,n_in,n_out", SIZES)
def test_sizes(tokens, n_in, n_out, dtype):
    gen = torch.Generator(device=DEV).manual_seed(tokens + n_in)
    x, w = operands(gen, tokens, n_in, n_out)
    bias = rand(gen, n_out)
    within(fb.linear(x, w, out_dtype=dtype), *expected(x, w, None, "none", None, dtype))
    within(fb.linear(x, w, bias, activation="silu", out_dtype=dtype), *expected(x, w, bias, "silu", None, dtype))
    fb.linear_poll_status()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens", [3, 200, 1111])
def test_bias_activation_residual_preact(tokens, dtype, act):
    gen = torch.Generator(device=DEV).manual_seed(7)
    x, w = operands(gen, tokens, 328, 712)
    w = (3 * w.float()).bfloat16()
    bias, r = rand(gen, 712), rand(gen, tokens, 712).to(dtype)
    preact = torch.full((tokens, 712), 7.0, device=DEV, dtype=torch.bfloat16)
    y = fb.linear(x, w, bias, activation=act, residual=r, preact=preact)
    assert y.dtype is dtype
    within(y, *expected(x, w, bias, act, r, dtype))
    within(preact, *expected(x, w, bias, "none", None, torch.bfloat16))
    assert torch.equal(y, fb.linear(x, w, bias, activation=act, residual=r))      # the same sums in the same order
    inplace = r.clone()
    assert fb.linear(x, w, bias, activation=act, residual=inplace, out=inplace) is inplace
    assert torch.equal(y, inplace)


def test_float32_sums_do_not_drift():
    """Long float32 sums of one sign, where cutting adds up: pieces of 512 values (a few more where few CTAs share a sum), so off by
    (2 * 512 / 16 + 64) 2^-23 of the sum, not by K / 16 of them."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    for tokens, n_in, n_out in [(1, 16384, 512), (40, 16384, 4096), (300, 16384, 2048), (2000, 16384, 1024), (5000, 8192, 512)]:
        x, w = (t.abs().bfloat16() for t in operands(gen, tokens, n_in, n_out))
        y, z = fb.linear(x, w, out_dtype=torch.float32).double(), x.double() @ w.double().t()
        assert ((y - z).abs() <= 128 * 2.0 ** -23 * z).all(), (tokens, ((y - z).abs() / z).max() * 2 ** 23)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,alive", [(1, 0), (1, 1), (40, 17), (256, 251), (700, 1), (700, 513), (700, 700)])
def test_rows_and_count(tokens, alive, dtype):
    """Survivors' rows of a residual stream are added to in place; other rows, and tokens past the count (NaN here), leave no trace."""
    gen = torch.Generator(device=DEV).manual_seed(alive)
    batch = tokens + 77
    x, w = operands(gen, tokens, 520, 392)
    x[alive:] = float("nan")
    bias = rand(gen, 392)
    stream = rand(gen, batch, 392).to(dtype)
    rows = torch.randperm(batch, generator=gen, device=DEV)[:tokens].sort().values.int()
    count = torch.tensor([alive], dtype=torch.int32, device=DEV)
    want, bound = expected(x[:alive], w, bias, "gelu", stream[rows[:alive].long()], dtype)
    out = stream.clone()
    preact = torch.full((tokens, 392), 5.0, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, activation="gelu", residual=out, out=out, rows=rows, count=count, preact=preact)
    within(out[rows[:alive].long()], want, bound)
    others = torch.ones(batch, dtype=torch.bool, device=DEV)
    others[rows[:alive].long()] = False
    assert torch.equal(out[others], stream[others])
    assert (preact[alive:] == 5.0).all()
    # without a residual, without a count
    if alive == tokens:
        out = stream.clone()
        fb.linear(x, w, out=out, rows=rows)
        within(out[rows.long()], *expected(x, w, None, "none", None, dtype))
        assert torch.equal(out[others], stream[others])


def test_count_out_of_range_and_rows_out_of_range():
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, w = operands(gen, 20, 64, 64)
    full = fb.linear(x, w)
    for count, real in ((-3, 0), (99, 20)):
        out = torch.zeros(20, 64, dtype=torch.bfloat16, device=DEV)
        fb.linear(x, w, out=out, count=torch.tensor([count], dtype=torch.int32, device=DEV))
        assert torch.equal(out[:real], full[:real]) and not out[real:].any()
    rows = torch.arange(20, dtype=torch.int32, device=DEV)
    rows[3], rows[5] = -1, 20
    out = torch.zeros(20, 64, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, out=out, rows=rows)
    keep = torch.ones(20, dtype=torch.bool, device=DEV)
    keep[[3, 5]] = False
    assert torch.equal(out[keep], full[keep]) and not out[~keep].any()


@pytest.mark.parametrize("tokens", [5, 300, 1300])
def test_strides(tokens):
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, w = operands(gen, tokens, 1024, 512)
    bias = rand(gen, 300)
    xs, ws = x[:, 256:256 + 392], w[:304, 64:64 + 392]
    big, res = torch.full((tokens, 701), 9.0, device=DEV), rand(gen, tokens, 333)
    out, r = big[:, 5:309], res[:, 7:311]
    fb.linear(xs, ws, rand(gen, 304) * 0, residual=r, out=out)
    within(out, *expected(xs, ws, None, "none", r, torch.float32))
    assert (big[:, :5] == 9).all() and (big[:, 309:] == 9).all()
    del bias
    # gradients of slices
    dy = rand(gen, tokens, 512).bfloat16()[:, 8:312]
    dxb, dwb = torch.full((tokens, 400), 9.0, device=DEV).bfloat16(), torch.full((304, 401), 9.0, device=DEV).bfloat16()
    check_backward(xs, ws, dy, None, "none", True, dx=dxb[:, 3:395], dweight=dwb[:, 1:393])
    assert (dxb[:, :3] == 9).all() and (dxb[:, 395:] == 9).all() and (dwb[:, :1] == 9).all() and (dwb[:, 393:] == 9).all()


def check_backward(x, w, dy, preact, act, with_bias, **into):
    dx, dw, db = fb.linear_backward(x, w, dy, preact=preact, activation=act, with_bias=with_bias, **into)
    g = dy.double()
    off = 0.0
    if act != "none":
        s = slope64(preact.double(), act)
        g = g * s
        # the slope is off by 16 units of 2^-23 of its parts (at most 1.5), the rounding of dz by 2^-8 of it
        off = 16 * 1.5 * 2.0 ** -23 * dy.double().abs()
    each = off + (2.0 ** -8 * g.abs() if act != "none" else 0)
    size = g.abs() + each
    for got, a, b, steps in ((dx, size, w.double().abs(), dy.shape[1]), (dw, size.t(), x.double().abs(), dy.shape[0])):
        left = g if got is dx else g.t()
        right = w.double() if got is dx else x.double()
        err = (each if got is dx else (each.t() if act != "none" else 0))
        bound = (steps / 16 + 4) * 2.0 ** -23 * (a @ b) + (err @ b if act != "none" else 0)
        want = left @ right
        within(got, want, (1 + 2.0 ** -8) * bound + 2.0 ** -8 * want.abs() + 1e-37)
    if with_bias:
        # float32 sums in a fixed order: every addition is off by 2^-24 of the sum of sizes at most
        within(db, g.sum(0), (off.sum(0) if act != "none" else 0) + (dy.shape[0] + 1) * 2.0 ** -24 * size.sum(0) + 1e-37)
    else:
        assert db is None
    again = fb.linear_backward(x, w, dy, preact=preact, activation=act, with_bias=with_bias)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1]) and (db is None or torch.equal(db, again[2]))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 8, 8), (3, 72, 136), (64, 64, 64), (65, 200, 72), (130, 1000, 264), (777, 520, 1400), (1500, 136, 328)])
def test_backward_sizes(tokens, n_in, n_out, act):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w = operands(gen, tokens, n_in, n_out)
    dy, preact = rand(gen, tokens, n_out).bfloat16(), (3 * rand(gen, tokens, n_out)).bfloat16()
    check_backward(x, w, dy, None if act == "none" else preact, act, tokens % 2 == 1)
    fb.linear_poll_status()


@pytest.mark.parametrize("tokens,n_in,n_out", [(4095, 2048, 1024), (2000, 4096, 2304), (300, 8192, 4096), (9000, 264, 520)])
def test_backward_large(tokens, n_in, n_out):
    gen = torch.Generator(device=DEV).manual_seed(5)
    x, w = operands(gen, tokens, n_in, n_out)
    check_backward(x, w, rand(gen, tokens, n_out).bfloat16(), rand(gen, tokens, n_out).bfloat16(), "gelu_tanh", True)


@pytest.mark.parametrize("tokens,n_in,n_out", [(5000, 512, 6144), (7001, 1544, 520), (4104, 1024, 4096), (2056, 2048, 2056)])
def test_both_gradients_whichever_sums_are_longer(tokens, n_in, n_out):
    """Sizes at which both products are large: over the tokens (dweight) longer than over the outputs (dx), shorter, and alike."""
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w = operands(gen, tokens, n_in, n_out)
    dy = rand(gen, tokens, n_out).bfloat16()
    check_backward(x, w, dy, None, "none", False)
    dx, dw, _ = fb.linear_backward(x, w, dy)
    # each alone: two such results are twice their bound apart at most
    for got, want, steps, left, right in ((fb.linear_backward(None, w, dy)[0], dx, n_out, dy, w), (fb.linear_backward(x, None, dy)[1], dw, tokens, dy.t(), x)):
        size = want.double().abs()
        within(got, want.double(), 1.01 * (2.0 ** -7 * size + 2 * (steps / 16 + 4) * 2.0 ** -23 * (left.double().abs() @ right.double().abs())) + 1e-37)
    fb.linear_poll_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,n_in,n_out,act", [(256, 4096, 4096, "none"), (251, 4104, 4040, "gelu"), (1000, 8192, 1024, "silu"), (256, 14336, 1032, "relu"),
                                                   (220, 4096, 6144, "none"), (777, 1400, 1000, "gelu_tanh"), (150, 2048, 2056, "none")])
def test_long_sums_of_a_few_hundred_tokens(tokens, n_in, n_out, act, dtype):
    """Sizes whose sums are shared, with all that an epilogue does, for listed rows of a stream, and their gradients."""
    gen = torch.Generator(device=DEV).manual_seed(n_in)
    x, w = operands(gen, tokens, n_in, n_out)
    bias, r = rand(gen, n_out), rand(gen, tokens + 30, n_out).to(dtype)
    preact = torch.full((tokens, n_out), 7.0, device=DEV, dtype=torch.bfloat16)
    y = fb.linear(x, w, bias, activation=act, residual=r[:tokens], preact=preact)
    within(y, *expected(x, w, bias, act, r[:tokens], dtype))
    within(preact, *expected(x, w, bias, "none", None, torch.bfloat16))
    assert torch.equal(y, fb.linear(x, w, bias, activation=act, residual=r[:tokens]))
    rows, alive = torch.randperm(tokens + 30, generator=gen, device=DEV)[:tokens].int(), tokens - 19
    x[alive:] = math.nan
    stream = r.clone()
    fb.linear(x, w, bias, activation=act, residual=stream, out=stream, rows=rows, count=torch.tensor([alive], dtype=torch.int32, device=DEV))
    at = rows[:alive].long()
    within(stream[at], *expected(x[:alive], w, bias, act, r[at], dtype))
    left = torch.ones(tokens + 30, dtype=torch.bool, device=DEV)
    left[at] = False
    assert torch.equal(stream[left], r[left])
    fb.linear_poll_status()
    if dtype is torch.bfloat16:
        dy, x = rand(gen, tokens, n_out).bfloat16(), rand(gen, tokens, n_in).bfloat16()
        check_backward(x, w, dy, preact, act, True)
        dx = fb.linear_backward(None, w, dy)[0]
        want, size = dy.double() @ w.double(), dy.double().abs() @ w.double().abs()
        within(dx, want, (1 + 2.0 ** -8) * (n_out / 16 + 4) * 2.0 ** -23 * size + 2.0 ** -8 * want.abs() + 1e-37)
        fb.linear(x, w, wait_limit=1000)                       # (and a wait that runs out is reported)
        with pytest.raises(fb.FiError, match="TIMEOUT"):
            fb.linear_poll_status()


def test_backward_of_extreme_preactivations():
    """Slopes that have reached 0 or 1 are that; nothing becomes NaN but what is NaN."""
    z = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 30.0, -30.0, 150.0, -150.0, 1e30, -1e30, math.inf, -math.inf, 5.0, -5.0, 19.0, -19.0], device=DEV)
    preact = z.bfloat16()[None].contiguous()
    x = torch.zeros(1, 8, device=DEV).bfloat16()
    w = torch.zeros(16, 8, device=DEV).bfloat16()
    dy = torch.ones(1, 16, device=DEV).bfloat16()
    for act in ACTS[1:]:
        _, _, db = fb.linear_backward(x, w, dy, preact=preact, activation=act, with_bias=True)
        safe = preact[0].double().clamp(-300, 300)
        # (at 0 the slope of relu is 0)
        within(db, slope64(safe, act), torch.full((16,), 16 * 1.5 * 2.0 ** -23, device=DEV).double())
        preact_nan = preact.clone()
        preact_nan[0, 3] = math.nan
        _, _, db = fb.linear_backward(x, w, dy, preact=preact_nan, activation=act, with_bias=True)
        assert db[3].isnan() and not db[[0, 1, 2, 4]].isnan().any()


def test_infinite_and_nan_inputs_stay_in_their_rows():
    gen = torch.Generator(device=DEV).manual_seed(6)
    x, w = operands(gen, 150, 264, 136)
    clean = fb.linear(x, w, activation="relu")
    x[7, 100], x[9, 0] = math.nan, math.inf
    y = fb.linear(x, w, activation="relu")
    assert y[7].isnan().all()                              # (a NaN passes the activation)
    assert ((y[9] == math.inf) | (y[9] == 0)).all()
    keep = torch.ones(150, dtype=torch.bool, device=DEV)
    keep[[7, 9]] = False
    assert torch.equal(y[keep], clean[keep])


def test_partial_gradients_and_empty():
    gen = torch.Generator(device=DEV).manual_seed(8)
    x, w = operands(gen, 100, 64, 72)
    dy, z = rand(gen, 100, 72).bfloat16(), rand(gen, 100, 72).bfloat16()
    dx, dw, db = fb.linear_backward(x, w, dy, preact=z, activation="silu", with_bias=True)
    a = fb.linear_backward(None, w, dy, preact=z, activation="silu")
    b = fb.linear_backward(x, None, dy, preact=z, activation="silu")
    c = fb.linear_backward(None, None, dy, preact=z, activation="silu", with_bias=True)
    assert torch.equal(a[0], dx) and a[1] is None and a[2] is None
    assert b[0] is None and torch.equal(b[1], dw) and b[2] is None
    assert c[0] is None and c[1] is None and torch.equal(c[2], db)
    x0, dy0, z0 = x[:0], dy[:0], z[:0]
    assert fb.linear(x0, w).shape == (0, 72)
    dx, dw, db = fb.linear_backward(x0, w, dy0, preact=z0, activation="silu", with_bias=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any()


@pytest.mark.parametrize("act", ["none", "gelu"])
def test_autograd(act):
    gen = torch.Generator(device=DEV).manual_seed(9)
    x, w = operands(gen, 77, 136, 264)
    bias, r, dy = rand(gen, 264), rand(gen, 77, 264), rand(gen, 77, 264)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, bias, r)]
    y = fb.linear(leaves[0], leaves[1], leaves[2], activation=act, residual=leaves[3])
    y.backward(dy)
    z = torch.empty(77, 264, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, activation=act, residual=r, preact=z)
    dx, dw, db = fb.linear_backward(x, w, dy.bfloat16(), preact=z, activation=act, with_bias=True)
    for leaf, g in zip(leaves, (dx, dw, db, dy)):
        assert leaf.grad.dtype is leaf.dtype and torch.equal(leaf.grad, g)
    # only what is asked for; an expanded gradient
    only = w.clone().requires_grad_(True)
    fb.linear(x, only, bias, activation=act).sum().backward()
    ones = torch.ones(77, 264, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, activation=act, preact=z)
    assert torch.equal(only.grad, fb.linear_backward(x, None, ones, preact=z, activation=act)[1])
    # a bias of another shape; a gradient that starts off a 16-byte boundary
    wide = bias[None].clone().requires_grad_(True)
    y = fb.linear(x, only, wide, activation=act)
    off = torch.empty(77 * 264 + 4, dtype=torch.bfloat16, device=DEV)[4:].view(77, 264).copy_(dy)
    g = torch.autograd.grad(y, (only, wide), off)
    want = fb.linear_backward(x, None, dy.bfloat16(), preact=z, activation=act, with_bias=True)
    assert torch.equal(g[0], want[1]) and g[1].shape == wide.shape and torch.equal(g[1][0], want[2])
    for kw in (dict(out=torch.empty(77, 264, device=DEV)), dict(preact=z), dict(count=torch.ones(1, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError, match="gradient"):
            fb.linear(x, only, **kw)


def test_gradient_against_differences():
    """The slope of sum(y g) along a direction, from values in 64 bits beside the gradients: off by dz's and the results' roundings."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    x, w = operands(gen, 64, 128, 192)
    bias, g = rand(gen, 192), rand(gen, 64, 192).bfloat16()
    z = torch.empty(64, 192, dtype=torch.bfloat16, device=DEV)
    fb.linear(x, w, bias, activation="gelu", preact=z)
    dx, dw, db = fb.linear_backward(x, w, g, preact=z, activation="gelu", with_bias=True)
    value = lambda x, w, b: (act64(x @ w.t() + b, "gelu") * g.double()).sum()
    base = [t.double() for t in (x, w, bias)]
    for i, grad in enumerate((dx, dw, db)):
        d = rand(gen, *base[i].shape).double()
        h = 1e-4
        up, down = ([t + s * h * d if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        slope = (value(*up) - value(*down)) / (2 * h)
        # preact and dz rounded to bfloat16 (2^-8 each, the slope's slope is at most 0.8), the result too; random signs
        size = (grad.double() * d).norm()
        assert abs((grad.double() * d).sum() - slope) <= 6 * 2.0 ** -8 * size * 3


def test_two_streams_and_capture():
    gen = torch.Generator(device=DEV).manual_seed(11)
    x, w = operands(gen, 300, 1024, 1032)
    x2, w2 = operands(gen, 9, 4096, 512)
    want, want2 = fb.linear(x, w), fb.linear(x2, w2)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(one):
            a = fb.linear(x, w)
        with torch.cuda.stream(two):
            b = fb.linear(x2, w2)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want2)
    dy = rand(gen, 300, 1032).bfloat16()
    ref = fb.linear_backward(x, w, dy, preact=want, activation="silu", with_bias=True)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        y1 = fb.linear(x, w)
        r1 = fb.linear_backward(x, w, dy, preact=want, activation="silu", with_bias=True)
    with torch.cuda.graph(g2):
        y2 = fb.linear(x2, w2)
    x.mul_(2)                                              # exact in bfloat16
    g1.replay(); g2.replay(); g1.replay()
    torch.cuda.synchronize()
    assert torch.equal(y1, fb.linear(x, w)) and torch.equal(y2, want2)
    assert torch.equal(r1[0], ref[0]) and torch.equal(r1[1], fb.linear_backward(x, w, dy, preact=want, activation="silu")[1])
    assert torch.equal(r1[2], ref[2])


def test_a_wait_that_runs_out_is_reported():
    gen = torch.Generator(device=DEV).manual_seed(12)
    for tokens in (4, 700):
        x, w = operands(gen, tokens, 512, 1024)
        want = fb.linear(x, w)
        fb.linear_poll_status()
        fb.linear(x, w, wait_limit=1000)
        with pytest.raises(fb.FiError, match="TIMEOUT"):
            fb.linear_poll_status()
        fb.linear_poll_status()
        assert torch.equal(fb.linear(x, w), want)


def test_offsets_past_32_bits():
    """140,000 rows of 16,384 values: more than 2^31 of them in the result, the residual and the gradients' inputs."""
    gen = torch.Generator(device=DEV).manual_seed(15)
    tokens, n_in, n_out = 140000, 16, 16384
    x, w = operands(gen, tokens, n_in, n_out)
    bias, stream = rand(gen, n_out), torch.zeros(tokens, n_out, dtype=torch.bfloat16, device=DEV)
    stream[:, ::5] = 2
    last = torch.arange(tokens - 70, tokens, device=DEV)
    preact = torch.empty(tokens, n_out, dtype=torch.bfloat16, device=DEV)
    r = stream[last].clone()
    assert fb.linear(x, w, bias, activation="silu", residual=stream, out=stream, preact=preact) is stream
    within(stream[last], *expected(x[last], w, bias, "silu", r, torch.bfloat16))
    within(preact[last], *expected(x[last], w, bias, "none", None, torch.bfloat16))
    # few tokens whose rows are the last ones
    r = stream[last].clone()
    fb.linear(x[:70], w, bias, residual=stream, out=stream, rows=last.int())
    within(stream[last], *expected(x[:70], w, bias, "none", r, torch.bfloat16))
    # gradients: dx of the last rows; dweight of rows that only the last tokens have
    dx = fb.linear_backward(None, w, stream, preact=preact, activation="relu")[0]
    g = torch.where(preact[last].double() > 0, stream[last].double(), 0)
    within(dx[last], g @ w.double(), (1 + 2.0 ** -8) * ((n_out / 16 + 4) * 2.0 ** -23 + 2.0 ** -8) * (g.abs() @ w.double().abs()) + 2.0 ** -8 * (g @ w.double()).abs())
    stream[:tokens - 70] = 0
    dw = fb.linear_backward(x, None, stream)[1]
    a, b = stream[last].double().t(), x[last].double()
    within(dw, a @ b, (1 + 2.0 ** -8) * (tokens / 16 + 4) * 2.0 ** -23 * (a.abs() @ b.abs()) + 2.0 ** -8 * (a @ b).abs() + 1e-37)
    fb.linear_poll_status()


def test_refusals():
    x, w = torch.zeros(4, 64, device=DEV).bfloat16(), torch.zeros(16, 64, device=DEV).bfloat16()
    flat = torch.zeros(4 * 64 + 8, device=DEV).bfloat16()
    ints = torch.zeros(4, dtype=torch.int32, device=DEV)
    dy = torch.zeros(4, 16, device=DEV).bfloat16()
    bad = [lambda: fb.linear(x.float(), w), lambda: fb.linear(x, w.float()), lambda: fb.linear(x[0], w), lambda: fb.linear(x, w[:, :56]),
           lambda: fb.linear(x.cpu(), w), lambda: fb.linear(x, w.cpu()), lambda: fb.linear(x, w, torch.zeros(15, device=DEV)),
           lambda: fb.linear(x, w, torch.zeros(16, device=DEV).bfloat16()), lambda: fb.linear(x, w, activation="tanh"),
           lambda: fb.linear(x, w, out_dtype=torch.float16), lambda: fb.linear(x, w, residual=torch.zeros(3, 16, device=DEV)),
           lambda: fb.linear(x, w, residual=torch.zeros(4, 16, device=DEV), out_dtype=torch.bfloat16), lambda: fb.linear(x, w, rows=ints),
           lambda: fb.linear(x, w, rows=ints[:3], out=torch.zeros(9, 16, device=DEV)), lambda: fb.linear(x, w, out=torch.zeros(16, 4, device=DEV).t()),
           lambda: fb.linear(x.t(), w), lambda: fb.linear_backward(x, w, dy, activation="gelu"), lambda: fb.linear_backward(x, w, dy.float()),
           lambda: fb.linear_backward(x, w, dy, dx=torch.zeros(4, 63, device=DEV).bfloat16()),
           lambda: fb.linear_backward(None, w, dy, dweight=torch.zeros(16, 64, device=DEV).bfloat16())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    unsound = [lambda: fb.linear(flat[4:260].view(4, 64), w), lambda: fb.linear(x[:, :60], w[:, :60]), lambda: fb.linear(x, w[:12]),
               lambda: fb.linear(torch.as_strided(flat, (4, 64), (60, 1)), w), lambda: fb.linear(torch.as_strided(flat, (4, 64), (32, 1)), w),
               lambda: fb.linear(x, w, out=torch.as_strided(torch.zeros(99, device=DEV), (4, 16), (8, 1))),
               lambda: fb.linear_backward(flat[4:260].view(4, 64), w, dy), lambda: fb.linear(x, w, wait_limit=-1),
               lambda: fb.linear(x, w, residual=torch.zeros(1, 16, device=DEV).expand(4, 16), out_dtype=torch.float32)]
    for call in unsound:
        with pytest.raises(fb.FiError, match="INVALID"):
            call()
