"""Activations in the products' epilogue against their formulas in 64 bits, relative to the value itself, far into their tails.

The argument is a float32 bias behind a product of zeros, so it is what it is to the last bit.  Bounds, in units of u = 2^-24: an exponential and
a reciprocal are off by 4 each; an exponent e (of 2) is off by 3 e / 1.44 (its square, its factor, its product), with a cubic argument by 5 e / 1.44;
the polynomial of the normal distribution by 3 as a fit and by 8 as a chain of roundings; a few roundings of products: 6.
"""
import math

import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24


def reference(z, act):
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2)), (25 + 3 * 0.5 * z * z) * U
    if act == "gelu_tanh":
        e = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
        return z / (1 + torch.exp(-e)), (14 + 5 * e.abs()) * U
    return z / (1 + torch.exp(-z)), (14 + 3 * z.abs()) * U


@pytest.mark.parametrize("act,lowest", [("gelu", -12.5), ("gelu_tanh", -9.5), ("silu", -80.0)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [1, 300])
def test_tails(act, lowest, dtype, tokens):
    n = 16384
    z = torch.linspace(lowest, 20.0, n, device=DEV)
    z[::7] = torch.linspace(-1e-3, 1e-3, z[::7].numel(), device=DEV)
    x, w = torch.zeros(tokens, 8, device=DEV).bfloat16(), torch.zeros(n, 8, device=DEV).bfloat16()
    y = fb.linear(x, w, z, activation=act, out_dtype=dtype)
    want, rel = reference(z.double(), act)
    half = 2.0 ** -8 if dtype is torch.bfloat16 else U
    far = (y.double() - want).abs()
    bound = ((1 + half) * rel + half) * want.abs() + 1e-37
    assert (far <= bound).all(), ((far / bound).max(), z[(far / bound).max(0).values.argmax()])


def test_slope_of_the_normal_distribution_far_out():
    """The gradient's slope Phi(z) + z phi(z): left of -2 both parts are small and of different signs."""
    z = torch.linspace(-12.0, 12.0, 8192, device=DEV).bfloat16()[None].contiguous()
    w, x = torch.zeros(8192, 8, device=DEV).bfloat16(), torch.zeros(1, 8, device=DEV).bfloat16()
    db = fb.linear_backward(x, w, torch.ones_like(z), preact=z, activation="gelu", with_bias=True)[2]
    d = z[0].double()
    cdf, pdf = 0.5 * torch.erfc(-d / math.sqrt(2)), torch.exp(-d * d / 2) / math.sqrt(2 * math.pi)
    far = (db.double() - (cdf + d * pdf)).abs()
    bound = (25 + 3 * 0.5 * d * d) * U * (cdf + d.abs() * pdf) + 1e-36
    assert (far <= bound).all(), (far / bound).max()
