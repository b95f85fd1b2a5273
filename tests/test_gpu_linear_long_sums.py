"""Products whose sums are long and of one sign, where what the tensor cores cut adds up.

Bounds.  The tensor cores cut a running sum after each 16 products, by 2^-23 of it at most.  A float32 result is taken out of them every 512
values, a bfloat16 one every 16,384, and the pieces are added up with roundings of 2^-24; so a sum is off by (512 / 16 + 4) or (16,384 / 16
+ 4) times 2^-23 of itself and by 2^-24 for each piece, however long it is.  A bfloat16 result is then rounded to half a step.
"""
import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def positive(gen, *shape, spread=False):
    """Values of 0.5 to 1.5; spread: each column has a scale of 1 to 2, so that sums lie at all places of a step."""
    t = 0.5 + torch.rand(*shape, generator=gen, device=DEV)
    return (t * (1 + torch.rand(shape[-1], generator=gen, device=DEV)) if spread else t).bfloat16()


def spread_rows(gen, *shape):
    return positive(gen, shape[1], shape[0], spread=True).t().contiguous()


def half_step(z):
    return torch.exp2(torch.floor(torch.log2(z)) - 8)


def check(got, z, k):
    piece = 512 if got.dtype is torch.float32 else 16384
    off = ((piece / 16 + 4) * 2.0 ** -23 + k / piece * 2.0 ** -24) * z
    if got.dtype is torch.bfloat16:
        off = off * (1 + 2.0 ** -8) + half_step(z + off)
    else:
        off = off + 2.0 ** -24 * z
    far = (got.double() - z).abs()
    assert (far <= off).all(), (far / off).max()


@pytest.mark.parametrize("tokens,n_in,n_out", [(1 << 18, 64, 72), (400000, 72, 128), (1000003, 136, 264), (300001, 512, 1024), (40000, 1024, 2048)])
def test_gradient_of_the_weight_over_many_tokens(tokens, n_in, n_out):
    gen = torch.Generator(device=DEV).manual_seed(n_in)
    x, w, dy = positive(gen, tokens, n_in), positive(gen, n_out, n_in), positive(gen, tokens, n_out, spread=True)
    z = sum(dy[i:i + 65536].double().t() @ x[i:i + 65536].double() for i in range(0, tokens, 65536))
    check(fb.linear_backward(x, None, dy)[1], z, tokens)
    dx, dw, _ = fb.linear_backward(x, w, dy)                  # both in one launch, where that is taken
    check(dw, z, tokens)
    check(dx, dy.double() @ w.double(), n_out)
    again = fb.linear_backward(x, w, dy)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    fb.linear_poll_status()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 1 << 20, 24), (5, 262152, 520), (64, 400000, 64), (300, 524288, 264), (700, 131080, 1032)])
def test_values_of_long_rows(tokens, n_in, n_out, dtype):
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w = positive(gen, tokens, n_in), spread_rows(gen, n_out, n_in)
    bias, r = torch.rand(n_out, generator=gen, device=DEV), torch.rand(tokens, n_out, generator=gen, device=DEV).to(dtype)
    z = x.double() @ w.double().t()
    y = fb.linear(x, w, out_dtype=dtype)
    check(y, z, n_in)
    # with all that comes behind the sum, which is above 2^17: silu is its argument there
    full = fb.linear(x, w, bias, activation="silu", residual=r, out_dtype=dtype)
    check(full, z + bias.double() + r.double(), n_in)
    assert torch.equal(y, fb.linear(x, w, out_dtype=dtype))
    fb.linear_poll_status()


@pytest.mark.parametrize("tokens,n_in,n_out", [(3, 40, 262144), (300, 264, 300000), (2100, 136, 131080)])
def test_gradient_of_the_input_over_many_outputs(tokens, n_in, n_out):
    gen = torch.Generator(device=DEV).manual_seed(n_in)
    w, dy = positive(gen, n_out, n_in, spread=True), positive(gen, tokens, n_out)
    check(fb.linear_backward(None, w, dy)[0], dy.double() @ w.double(), n_out)
    fb.linear_poll_status()


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 1 << 20, 24), (1, 1 << 22, 24), (64, 400000, 64), (5, 1 << 18, 520), (300, 1 << 19, 264)])
def test_float32_sums_of_any_length_do_not_drift(tokens, n_in, n_out):
    """What is cut has one sign, so the mean over all results shows it: half of (512 / 16 + 4) 2^-23, as a piece grows evenly.  Roundings of the
    pieces' sum have none: each at most 2^-24 of it, a third of that squared on average, six deviations of the mean over the results."""
    gen = torch.Generator(device=DEV).manual_seed(n_in)
    x, w = positive(gen, tokens, n_in), spread_rows(gen, n_out, n_in)
    z = x.double() @ w.double().t()
    mean = ((fb.linear(x, w, out_dtype=torch.float32).double() - z) / z).mean().abs().item()
    assert mean <= 36 * 2.0 ** -24 + 6 * (n_in / 512 / 3 / n_out) ** 0.5 * 2.0 ** -24, mean * 2 ** 24
