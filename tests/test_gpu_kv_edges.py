"""Attention layers behind the caches at the edges of what their formulas are given: value vectors without a spread, peaked and
very long softmaxes, numbers near the ends of their types, prompts whose first queries see few keys, refused requests.

Everything is compared with the formula in 64 bits over what the store holds.  Bounds follow from the roundings the calls state
(u = 2^-24): see each test.
"""
import math

import numpy as np
import pytest
import torch

from paper_2002_02645_b200 import binding as fb
from test_gpu_kv_ops import DEV, MANY, Attention, ints, pools, unpack

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


def put(a, which, i, x):
    """Stores x [keys, kv_heads, dim] as the keys ("k") or values ("v") of request i, as the append call does."""
    pages = a.table[a.rows[i], :-(-a.lens[i] // a.page)].long()
    t = torch.arange(a.lens[i], device=DEV)
    slots = pages[t // a.page] * a.page + t % a.page
    kc, km = pools(a.kc.shape[0], a.kv_heads, a.page, a.dim)
    tmp = fb.KvCache(kc, km, *pools(a.kc.shape[0], a.kv_heads, a.page, a.dim), q_heads=a.kv_heads)
    tmp.append(x.float().contiguous(), x.float().contiguous(), slots)
    codes, meta = (a.kc, a.km) if which == "k" else (a.vc, a.vm)
    codes[pages], meta[pages] = kc[pages], km[pages]


# ------------------------------------------------------------------------------ value vectors without a spread of their own

SPREADS = {   # requests' lengths and queries; which keys' values are constant
    "one-step": (dict(lens=[64], queries=[1]), lambda t: t % 4 == 0),
    "earlier-step": (dict(lens=[600], queries=[1]), lambda t: t < 256),
    "later-step": (dict(lens=[600], queries=[1]), lambda t: t >= 256),
    "another-warp": (dict(lens=[256], queries=[2]), lambda t: (t >= 64) & (t < 128)),
    "one-among-ordinary": (dict(lens=[200, 77], queries=[1, 3]), lambda t: t == 31),
    "all-but-one": (dict(lens=[200, 77], queries=[1, 3]), lambda t: t != 31),
    "cut": (dict(lens=[20011], queries=[1]), lambda t: t % 3 == 1),
    "none-ordinary": (dict(lens=[130], queries=[1]), lambda t: t >= 0),
}


@BOTH
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("spread", [0.0, 1e-6, 1e-3, 0.1, 0.5])
@pytest.mark.parametrize("name", SPREADS)
def test_values_of_hardly_any_spread_count_beside_ordinary_ones(name, spread, dim, dtype):
    """A constant vector is stored with the smallest scale and all of it in the offset; its weight in the sums is that of any
    other.  Bound: as for ordinary values (weights rounded once, to halves or pairs of them; float32 sums)."""
    case, constant = SPREADS[name]
    a = Attention(q_heads=8, kv_heads=2, dim=dim, dtype=dtype, seed=4, **case)
    gen = torch.Generator(device=DEV).manual_seed(7)
    for i, length in enumerate(a.lens):
        v = torch.randn(length, 2, dim, generator=gen, device=DEV)
        flat = spread * torch.rand(length, 2, dim, generator=gen, device=DEV)
        flat[..., 0] = 0.0                       # the least value is a bf16 number: nothing but `spread` makes the scale
        flat += 3.0 + 0.25 * torch.randint(-8, 9, (length, 2, 1), generator=gen, device=DEV)
        put(a, "v", i, torch.where(constant(torch.arange(length, device=DEV))[:, None, None], flat, v))
    a.q *= 0.2                                   # many keys share the weight
    out, lse = a.run()
    a.check(out, lse)
    again, _ = a.run()
    assert torch.equal(out[:a.cu[-1]], again[:a.cu[-1]])
