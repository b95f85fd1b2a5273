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


def formula(a, i, g, q, scale):
    """Of head g of request i: weights [queries, keys], scores, values, in 64 bits."""
    n, length = a.queries[i], a.lens[i]
    h = g // a.group
    x = q[a.cu[i]:a.cu[i + 1], g].double() @ a.values("k", i, h).T * scale
    pos = torch.arange(length - n, length, device=DEV)[:, None]
    t = torch.arange(length, device=DEV)
    seen = t <= pos
    if a.window:
        seen = seen & (t > pos - a.window)
    x = x.masked_fill(~seen, -math.inf)
    return torch.softmax(x, -1), x, a.values("v", i, h)


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


# --------------------------------------------------------------------------------------------------- peaked and long softmaxes

def one_number_keys(a, i, codes0):
    """Keys of request i: code codes0 (per key) in the first dimension, 0 in the others, scale 1 and offset 0, so that a query
    (t, 0, 0, ...) scores t * code * scale exactly."""
    pages = a.table[a.rows[i], :-(-a.lens[i] // a.page)].long()
    t = torch.arange(a.lens[i], device=DEV)
    where, off = pages[t // a.page], t % a.page
    a.kc[where, :, off] = 0
    a.kc[where, :, off, 0] = codes0.to(torch.uint8)[:, None]
    a.km[where, :, off] = torch.tensor([1.0, 0.0], device=DEV, dtype=torch.bfloat16)


def equal_spread_values(a, i, offset, gen):
    """Values of request i: random codes, the same scale (2^-5) and offset everywhere."""
    pages = a.table[a.rows[i], :-(-a.lens[i] // a.page)].long()
    a.vc[pages] = torch.randint(0, 256, a.vc[pages].shape, generator=gen, device=DEV, dtype=torch.uint8)
    a.vm[pages] = torch.tensor([2.0 ** -5, offset], device=DEV, dtype=torch.bfloat16)


def everywhere(a, q, **kw):
    """Attention of request 0 alone, as often as fills the device, so that a CTA takes a whole request."""
    n = 6 * torch.cuda.get_device_properties(0).multi_processor_count
    table = a.table[a.rows[0]:a.rows[0] + 1].expand(n, -1).contiguous()
    out, lse = a.kv.attend(q.expand(n, -1, -1).contiguous(), ints([a.lens[0]] * n), table, with_lse=True, **kw)
    return out[n // 2], lse[n // 2]


SINKS = [5, 70, 140, 200]       # one in the share of each of a CTA's four warps


@pytest.mark.parametrize("keys", [2048, 32768])
@pytest.mark.parametrize("gap", [8.0, 9.0, 10.0])
def test_float32_weights_far_below_the_largest_keep_their_bits(keys, gap):
    """Four keys some nats above all others, which are equal.  Every weight may be off by 2^-21 of itself (a pair of halves and
    the exponential, 2^-22 each) and by what float32 does to its exponent: four roundings of numbers up to the score's parts.
    (The parts of a value are at most 15/2 scales and the offset moved by as much.)"""
    heads = 16
    a = Attention(lens=[keys], queries=[1], q_heads=heads, kv_heads=1, dim=128, page=64, dtype=torch.float32, seed=5)
    gen = torch.Generator(device=DEV).manual_seed(11)
    codes0 = torch.zeros(keys, device=DEV)
    codes0[SINKS] = 15
    one_number_keys(a, 0, codes0)
    equal_spread_values(a, 0, 1.0, gen)
    gaps = gap + torch.linspace(0.0, 1.0, heads, device=DEV)
    q = torch.zeros(1, heads, 128, device=DEV)
    q[0, :, 0] = gaps / 15
    a.q = q
    out, lse = everywhere(a, q, scale=1.0)
    for g in range(heads):
        p, x, v = formula(a, 0, g, q, 1.0)
        want = (p @ v)[0]
        gap = gaps[g].item()
        each = 2.0 ** -21 + 4 * 2.0 ** -24 * (1 + 2 * gap)
        size = (v.abs().amax(-1) + 7.5 * 2.0 ** -5 + 1.25).max()
        assert ((out[g].double() - want).abs() <= each * size).all(), ((out[g].double() - want).abs() / (each * size)).max()
        assert (lse[g].double() - torch.logsumexp(x, -1)[0]).abs() <= each + 2.0 ** -22 * gap


@pytest.mark.parametrize("prompt", [False, True])
def test_bf16_weights_far_below_the_largest_are_not_lost_together(prompt):
    """Four keys 14 nats above 16,380 equal others; in half of the dimensions their value is zero, so that there the others' mean is
    all there is.  Each of the others' weights may be off by 2^-11 (a half; for prompts the value too), exponents by a few u of
    14, the result by its rounding."""
    keys = 16384
    a = Attention(lens=[keys], queries=[1], q_heads=4, kv_heads=1, dim=128, page=64, seed=6)
    gen = torch.Generator(device=DEV).manual_seed(12)
    codes0 = torch.zeros(keys, device=DEV)
    codes0[SINKS] = 14
    one_number_keys(a, 0, codes0)
    x = torch.randint(0, 16, (keys, 1, 128), generator=gen, device=DEV) * 0.125         # 0 .. 15/8: offset 0, scale 1/8
    x[:, :, 0], x[:, :, 1] = 0.0, 15 * 0.125
    x[SINKS, 0, 2:65] = 0.0
    put(a, "v", 0, x)
    q = torch.zeros(1, 4, 128, device=DEV, dtype=torch.bfloat16)
    q[0, :, 0] = torch.tensor([1.0, 0.9375, 0.875, 0.75], device=DEV)
    a.q = q
    out = a.run(q=q, scale=1.0, max_query=MANY)[0][0] if prompt else everywhere(a, q, scale=1.0)[0]
    for g in range(4):
        p, _, v = formula(a, 0, g, q, 1.0)
        want = (p @ v)[0]
        each = 2.0 ** -11 * (2 if prompt else 1) + 2.0 ** -18
        assert ((out[g].double() - want).abs() <= (each + 2.0 ** -8) * want.abs()).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_bf16_sums_over_many_keys_do_not_drift(dim):
    """Requests that fill the device, each 400,000 keys long (all of them read the same pages), with weights that hardly differ: the
    result is the mean of the values, a few hundred times smaller than they are.  Roundings of the weights (2^-12 at most, each for
    itself) add up like independent errors: six times the root of the sum of their squares.  Sums in float32 may be off by 2^-19 of
    the sum of the parts' sizes (codes less 7.5, offsets moved by as much), whatever the number of keys; the rounding to bf16 is 2^-8."""
    keys, heads, page = 400000, 8, 256
    blocks = -(-keys // page)
    gen = torch.Generator(device=DEV).manual_seed(dim)
    kc, km = pools(blocks, 1, page, dim)
    vc, vm = pools(blocks, 1, page, dim)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=heads)
    x = torch.randn(2, keys, 1, dim, generator=gen, device=DEV)
    kv.append(x[0], x[1], torch.arange(keys, device=DEV))
    requests = 3 * torch.cuda.get_device_properties(0).multi_processor_count
    table = torch.arange(blocks, dtype=torch.int32, device=DEV).expand(requests, blocks).contiguous()
    q = (0.1 * torch.randn(requests, heads, dim, generator=gen, device=DEV)).to(torch.bfloat16)
    out = kv.attend(q, ints([keys] * requests), table)
    value = lambda c, m: unpack(c.view(-1, dim // 2)[:keys]).double() * m.view(-1, 2)[:keys, :1].double() + m.view(-1, 2)[:keys, 1:].double()
    k, v = value(kc, km), value(vc, vm)
    scale, offset = (vm.view(-1, 2)[:keys, j:j + 1].double() for j in (0, 1))
    parts = 7.5 * scale + (offset + 7.5 * scale).abs()
    for r in (0, 1, requests // 2, requests - 1):
        p = torch.softmax(q[r].double() @ k.T * dim ** -0.5, -1)
        want = p @ v
        bound = 6 * 2.0 ** -12 * (p.square() @ v.square()).sqrt() + 2.0 ** -19 * (p @ parts) + 2.0 ** -8 * want.abs()
        off = (out[r].double() - want).abs() / bound
        assert (off <= 1).all(), off.max().item()


# ------------------------------------------------------------------------------------------------- the ends of the types

@BOTH
@pytest.mark.parametrize("prompt", [False, True])
def test_scores_below_minus_1e30_are_scores(prompt, dtype):
    """All scores are about -2.5e30: the result is a mean of the values, not that of a query without keys.  (Exponents are off by some u
    of the scores' size, so that at this size any weights are as good.)"""
    if prompt and dtype is torch.float32:
        pytest.skip("prompts of float32 take the same kernel")
    a = Attention(lens=[37], queries=[2], q_heads=2, kv_heads=1, dim=64, dtype=dtype, seed=8)
    put(a, "k", 0, torch.full((37, 1, 64), 2.0 ** 50, device=DEV))
    a.q[:] = -(2.0 ** 48)
    out, lse = a.run(max_query=MANY if prompt else 2)
    for g in range(2):
        _, x, v = formula(a, 0, g, a.q, 64 ** -0.5)
        parts = (v.abs().amax(-1) + 15 * a.vm_scale(0, 0)).max()
        slack = 2 * 2.0 ** -11 * parts + 2.0 ** -8 * v.abs().max()
        got = out[:2, g].double()
        assert (got >= v.min(0).values - slack).all() and (got <= v.max(0).values + slack).all()
        ref = torch.logsumexp(x, -1)
        assert ((lse[:2, g].double() - ref).abs() <= 2.0 ** -20 * ref.abs()).all()


@BOTH
@pytest.mark.parametrize("size", [2.0 ** e for e in (14, 20, 23, 24, 25, 26, 30, 60)])
@pytest.mark.parametrize("prompt", [False, True])
def test_scores_of_any_size_choose_the_largest(prompt, size, dtype):
    """Where one score is above all others by more than float32's roundings of its parts, its value is the result."""
    if prompt and dtype is torch.float32:
        pytest.skip("prompts of float32 take the same kernel")
    a = Attention(lens=[300, 700, 40], queries=[150, 2, 30], q_heads=8, kv_heads=2, dim=64, dtype=dtype, seed=22, room=1024)
    a.q *= size
    chosen = 0
    for with_lse in (True, False):
        got = a.run(max_query=MANY if prompt else 150, with_lse=with_lse)
        out = got[0] if with_lse else got
        assert out[:a.cu[-1]].isfinite().all()
        for i, n in enumerate(a.queries):
            for g in range(8):
                _, x, v = formula(a, i, g, a.q, 64 ** -0.5)
                reach = (a.q[a.cu[i]:a.cu[i + 1], g].double().abs().sum(-1, keepdim=True) * a.k_reach(i, g // a.group) / 8).amax(-1)
                best = x.topk(2, -1).values if x.shape[1] > 1 else x.new_zeros(n, 2)
                clear = best[:, 0] - best[:, 1] > 2.0 ** -18 * reach + 40
                want = v[x.argmax(-1)][clear]
                # a weight as a half, a value as another, the result as bf16 (float32: pairs of halves); codes and offset are summed apart
                parts = v.abs().amax() + 15 * a.vm_scale(i, g // a.group).max()
                bound = (2.0 ** -10 if dtype is torch.bfloat16 else 2.0 ** -19) * parts + (2.0 ** -8 if dtype is torch.bfloat16 else 0) * want.abs()
                assert ((out[a.cu[i]:a.cu[i + 1], g][clear].double() - want).abs() <= bound).all()
                chosen += int(clear.sum())
    assert chosen > 300 or size < 2.0 ** 20


@BOTH
@pytest.mark.parametrize("value", [2.0 ** 90, -(2.0 ** 100), 1.75 * 2.0 ** 125])
def test_constant_values_of_any_size(value, dtype):
    """A constant vector's offset over its scale (2^-40) is no float32 number any more; the vector is.  Bound: the roundings of the
    result, and of sums and quotients in float32."""
    a = Attention(lens=[1, 2, 37, 700], queries=[1, 2, 5, 3], q_heads=4, kv_heads=2, dim=128, dtype=dtype, seed=20)
    for i, n in enumerate(a.lens):
        put(a, "v", i, torch.full((n, 2, 128), value, device=DEV))
    out, _ = a.run()
    assert ((out[:a.cu[-1]].double() - value).abs() <= (2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -18) * abs(value)).all()


@pytest.mark.parametrize("key,query,scale", [(0.0, 2.0 ** -90, None), (0.0, 2.0 ** -100, None), (0.0, 1.0, 2.0 ** -100),
                                             (0.0, 2.0 ** -60, -2.0 ** -60), (2.0 ** -70, 2.0 ** -70, None)])
def test_prompts_of_tiny_scores_average_the_values(key, query, scale):
    """Scores of (almost) nothing: all visible keys weigh the same, and hidden ones stay hidden."""
    a = Attention(lens=[300, 40], queries=[200, 3], q_heads=4, kv_heads=2, dim=128, seed=9, room=1024)
    for i, n in enumerate(a.lens):
        put(a, "k", i, torch.full((n, 2, 128), key, device=DEV))
    a.q[:] = (a.q.sign() * query).to(a.q.dtype)
    out, lse = a.run(max_query=MANY, scale=scale)
    a.check(out, lse, scale=scale, halves=True)
    a.check(a.run(max_query=MANY, scale=scale, with_lse=False), None, scale=scale, halves=True)


@pytest.mark.parametrize("key,query", [(2.0 ** 112, 2.0 ** -112), (2.0 ** 120, 2.0 ** -110), (2.0 ** 123, 2.0 ** -115), (2.0 ** -60, 2.0 ** 116)])
def test_prompts_whose_keys_or_queries_reach_the_end_of_the_type(key, query):
    a = Attention(lens=[300, 40], queries=[200, 3], q_heads=4, kv_heads=2, dim=128, seed=10, room=1024)
    gen = torch.Generator(device=DEV).manual_seed(3)
    for i, n in enumerate(a.lens):
        put(a, "k", i, torch.randn(n, 2, 128, generator=gen, device=DEV) * key)
    a.q[:] = (torch.randn(a.q.shape, generator=gen, device=DEV) * query).to(a.q.dtype)
    scale = 0.05 / (key * query)
    if not 2.0 ** -120 < abs(scale) < 2.0 ** 120:
        pytest.skip("no float32 scale")
    out, lse = a.run(max_query=MANY, scale=scale)
    a.check(out, lse, scale=scale, halves=True)
    a.check(a.run(max_query=MANY, scale=scale, with_lse=False), None, scale=scale, halves=True)


def test_prompt_values_reach_the_end_of_the_type():
    a = Attention(lens=[200], queries=[70], q_heads=2, kv_heads=1, dim=64, seed=10, room=1024)
    gen = torch.Generator(device=DEV).manual_seed(3)
    put(a, "v", 0, torch.randn(200, 1, 64, generator=gen, device=DEV) * 2.0 ** 121)
    out, lse = a.run(max_query=MANY)
    a.check(out, lse, halves=True)
    a.check(a.run(max_query=MANY, with_lse=False), None, halves=True)


# --------------------------------------------------------------------------------- prompts: queries that see few keys

def check_logarithms(a, lse):
    """The softmax sum's logarithm is a float32 output: off by float32's roundings of a score's parts (2^-20 of their sum, as in the
    tests of the kernel for few rows), however few keys a query sees and however many columns the block table has."""
    scale = a.dim ** -0.5
    for i, n in enumerate(a.queries):
        for g in range(a.group * a.kv_heads):
            _, x, _ = formula(a, i, g, a.q, scale)
            ref = torch.logsumexp(x, -1)
            reach = (a.q[a.cu[i]:a.cu[i + 1], g].double().abs().sum(-1, keepdim=True) * a.k_reach(i, g // a.group) * scale).amax(-1)
            off = (lse[a.cu[i]:a.cu[i + 1], g].double() - ref).abs() / (2.0 ** -20 * (1 + reach) + 2.0 ** -20 * ref.abs())
            assert (off <= 1).all(), off.max().item()


@BOTH
@pytest.mark.parametrize("value", [0.0, 3.0, 2.0 ** 100])
@pytest.mark.parametrize("prompt", [False, True])
def test_logarithms_do_not_depend_on_the_values(prompt, value, dtype):
    """Scores of 0: the logarithm is that of the number of keys, whatever scale the values are stored with (a constant vector's is
    2^-40).  Off by float32's roundings of itself."""
    if prompt and dtype is torch.float32:
        pytest.skip("prompts of float32 take the same kernel")
    a = Attention(lens=[1, 2, 37, 700], queries=[1, 2, 5, 300], q_heads=4, kv_heads=2, dim=128, dtype=dtype, seed=20)
    for i, n in enumerate(a.lens):
        put(a, "v", i, torch.full((n, 2, 128), value, device=DEV))
    out, lse = a.run(scale=0.0, max_query=MANY if prompt else 300)
    for i, (n, length) in enumerate(zip(a.queries, a.lens)):
        ref = torch.log(torch.arange(length - n + 1, length + 1, dtype=torch.float64, device=DEV))[:, None]
        assert ((lse[a.cu[i]:a.cu[i + 1]].double() - ref).abs() <= 2.0 ** -21 * (1 + ref)).all()
        assert ((out[a.cu[i]:a.cu[i + 1]].double() - value).abs() <= 2.0 ** -10 * value).all()


FEW_KEYS = {
    "prompt-from-nothing": dict(lens=[300, 7], queries=[300, 7], room=8192),
    "short-requests": dict(lens=[1, 2, 9, 50], queries=[1, 1, 2, 30], room=4096),
    "narrow-window": dict(lens=[900], queries=[200], window=3, room=2048),
    "narrow-table": dict(lens=[300, 7], queries=[300, 7]),
}


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("name", FEW_KEYS)
def test_prompt_kernel_logarithms_of_few_keys(name, dim):
    a = Attention(q_heads=8, kv_heads=2, dim=dim, seed=13, **FEW_KEYS[name])
    for i, n in enumerate(a.lens):
        put(a, "k", i, torch.randn(n, 2, dim, device=DEV) + 2.0)
    out, lse = a.run(max_query=MANY)
    a.check(out, None, halves=True)
    check_logarithms(a, lse)


def test_wider_block_table_keeps_the_results_as_exact():
    """The same requests behind a table with room for 48 times the keys, which may choose another kernel."""
    a = Attention(q_heads=32, kv_heads=4, dim=128, lens=[600, 900], queries=[600, 400], seed=14)
    for room in (0, 48):
        if room:
            wide = torch.full((a.table.shape[0], 48 * a.table.shape[1]), -1, dtype=torch.int32, device=DEV)
            wide[:, :a.table.shape[1]] = a.table
            a.table = wide
        out, lse = a.run()
        a.check(out, None, halves=True)
        check_logarithms(a, lse)


# ------------------------------------------------------------------------------------------------- refused requests

@BOTH
@pytest.mark.parametrize("prompt", [False, True])
def test_refused_requests_get_zeros_through_the_whole_layer(prompt, dtype):
    """Too few pages: some requests are refused, between granted ones.  Their queries see nothing, as the attention call is told by
    `granted`; the others are as without them."""
    page, blocks, batch, heads, dim = 16, 8, 7, 2, 64
    gen = torch.Generator(device=DEV).manual_seed(21)
    kv = fb.KvCache(*pools(9, heads, page, dim), *pools(9, heads, page, dim), q_heads=4)
    tables = fb.KvTables(page_size=page, max_blocks=blocks, max_batch=batch)
    table = torch.full((batch, blocks), -1, dtype=torch.int32, device=DEV)
    free, count, lens = ints(list(range(9))), ints([9]), ints([0] * batch)
    news = [[20, 3, 40, 1, 16, 0, 5], [30, 2, 9, 1, 60, 1, 1]]
    stored = [[] for _ in range(batch)]
    for new in news:
        total = sum(new)
        step = tables.extend(lens, free, count, table, new_lens=ints(new), max_tokens=total)
        k, v = torch.randn(2, total, heads, dim, generator=gen, device=DEV).to(dtype)
        q = torch.randn(total, 4, dim, generator=gen, device=DEV).to(dtype)
        granted = step.granted.tolist()
        for i, n in enumerate(new):
            if n and not granted[i]:
                q[step.cu_tokens[i]:step.cu_tokens[i + 1]] = math.nan          # a position past the rope table gives this
        ks, vs = kv.append(k, v, step.slot_map, with_stored=True)
        out, lse = kv.attend(q, step.lens, table, cu_tokens=step.cu_tokens, granted=step.granted, with_lse=True,
                             max_query=MANY if prompt else max(new))
        cu = step.cu_tokens.tolist()
        for i, n in enumerate(new):
            at = slice(cu[i], cu[i + 1])
            if granted[i] < n:
                assert (out[at] == 0).all() and (lse[at] == -math.inf).all()
                continue
            stored[i] += [(ks[t].double(), vs[t].double()) for t in range(cu[i], cu[i + 1])]
            for j in range(n):
                see = stored[i][:len(stored[i]) - n + j + 1]
                kk, vv = torch.stack([s[0] for s in see]), torch.stack([s[1] for s in see])
                x = torch.einsum("hgd,thd->hgt", q[cu[i] + j].double().view(heads, 2, dim), kk) / 8
                want = torch.einsum("hgt,thd->hgd", torch.softmax(x, -1), vv).reshape(4, dim)
                # `stored` is rounded to bf16 (2^-8 of numbers up to 4): scores move by 2^-8 of their parts, values by 2^-8 of theirs
                assert (out[cu[i] + j].double() - want).abs().max() <= 2.0 ** -8 * (4 + 2 * 8 * 4)
        lens, count = step.lens, step.free_count
    assert 0 in granted and max(granted) > 0
    kv.poll_status()
    with pytest.raises(ValueError):
        kv.attend(q, lens, table, cu_tokens=step.cu_tokens, granted=step.granted[:3])


# --------------------------------------------------------------------------------------------- mixed batches

def test_one_prompt_among_many_single_tokens():
    """A chunk of a prompt beside requests of one token: the choice of the kernel goes by the tokens there are."""
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(1, 900, 100)]
    queries = [1] * 100
    lens[40], queries[40] = 700, 500
    a = Attention(lens=lens, queries=queries, q_heads=16, kv_heads=4, dim=128, seed=15, room=2048)
    out, lse = a.run()
    a.check(out, lse)


def test_prompts_the_rule_gives_to_the_prompt_kernel():
    """Many rows of many heads, no hint but the true number of queries."""
    a = Attention(lens=[1500, 1400], queries=[1200, 1100], q_heads=32, kv_heads=4, dim=64, page=64, seed=16)
    out, lse = a.run()
    a.check(out, lse, halves=True)
    again = a.run()
    assert torch.equal(out[:2300], again[0][:2300]) and torch.equal(lse[:2300], again[1][:2300])


def test_prompts_and_gradients_in_a_graph():
    a = Attention(lens=[500, 33], queries=[300, 20], q_heads=8, kv_heads=2, dim=128, seed=17)
    cu, rows, out = ints(a.cu), ints(a.rows), torch.empty_like(a.q)
    x = torch.randn(200, 4, 64, device=DEV)
    w, dy = torch.ones(64, device=DEV), torch.randn(200, 4, 64, device=DEV)

    def call():
        a.kv.attend(a.q, a.d_lens, a.table, cu_tokens=cu, row_idx=rows, max_query=MANY, out=out)
        return fb.head_norm_rope_backward(x, None, w, None, None, None, dy, None)
    want = [t.clone() for t in call() if t is not None] + [out.clone()]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = [t for t in call() if t is not None]
    out.zero_()
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for p, r in zip(got + [out[:320]], want[:-1] + [want[-1][:320]]):
        assert torch.equal(p, r)


# ---------------------------------------------------------------------------------------------- a single token's strides

@BOTH
def test_single_tokens_may_have_any_token_stride(dtype):
    """The distance to a next token that is not there does not matter, whatever number the tensor has for it."""
    flat = torch.randn(4 * 64, device=DEV).to(dtype)
    odd = flat.as_strided((1, 4, 64), (4 * 64 + 3, 64, 1))
    plain = flat.view(1, 4, 64)
    w = torch.ones(64, device=DEV)
    for args in ((odd, None), (odd, odd), (plain, odd)):
        q, k = fb.head_norm_rope(*args, w, w, None, None)
        want, _ = fb.head_norm_rope(plain, None, w, None, None, None)
        assert torch.equal(q, want) and (k is None or torch.equal(k, want))
    got = fb.head_norm_rope_backward(odd, odd, w, w, None, None, odd, odd)
    ref = fb.head_norm_rope_backward(plain, plain, w, w, None, None, plain, plain)
    assert all(torch.equal(x, y) for x, y in zip(got, ref))
    kv = fb.KvCache(*pools(2, 4, 16, 64), *pools(2, 4, 16, 64), q_heads=4)
    kv.append(odd, odd, ints([0], torch.int64))
    table = ints([[0, 1]])
    assert torch.equal(kv.attend(odd, ints([1]), table), kv.attend(plain, ints([1]), table))


# ---------------------------------------------------------------------------------------------------------- gradients

@BOTH
def test_head_norm_rope_takes_part_in_backpropagation(dtype):
    gen = torch.Generator(device=DEV).manual_seed(31)
    qkv = torch.randn(9, 8, 64, generator=gen, device=DEV).to(dtype).requires_grad_()
    wq, wk = ((1 + 0.1 * torch.randn(64, generator=gen, device=DEV)).requires_grad_() for _ in range(2))
    angle = torch.rand(50, 16, generator=gen, device=DEV)
    rope = torch.cat([angle.cos(), angle.sin()], 1)
    pos = torch.randint(0, 50, (9,), generator=gen, device=DEV, dtype=torch.int32)
    q, k, _ = qkv.split([5, 2, 1], 1)
    yq, yk = fb.head_norm_rope(q, k, wq, wk, rope, pos, eps=1e-5, interleaved=True)
    aq, ak = (torch.randn(t.shape, generator=gen, device=DEV).to(dtype) for t in (yq, yk))
    ((yq * aq).sum() + (yk * ak).sum()).backward()
    with torch.no_grad():
        dq, dk, dwq, dwk = fb.head_norm_rope_backward(q, k, wq, wk, rope, pos, aq, ak, eps=1e-5, interleaved=True)
        same = fb.head_norm_rope(q, k, wq, wk, rope, pos, eps=1e-5, interleaved=True)
    assert torch.equal(same[0], yq) and torch.equal(same[1], yk) and not same[0].requires_grad
    assert torch.equal(qkv.grad[:, :5], dq) and torch.equal(qkv.grad[:, 5:7], dk) and (qkv.grad[:, 7] == 0).all()
    assert torch.equal(wq.grad, dwq) and torch.equal(wk.grad, dwk)
    # only one result is used, only the weights learn, no keys
    wq.grad = wk.grad = None
    fb.head_norm_rope(q.detach(), k.detach(), wq, wk, rope, pos)[0].float().sum().backward()
    assert wq.grad is not None and (wk.grad is None or (wk.grad == 0).all())
    x = torch.randn(3, 2, 64, generator=gen, device=DEV).to(dtype).requires_grad_()
    fb.head_norm_rope(x, None, None, None, None, None)[0].float().square().sum().backward()
    assert x.grad.isfinite().all()
    # tokens past the count: no gradient, whatever is in theirs
    x.grad = None
    y = fb.head_norm_rope(x, None, None, None, None, None, count=ints([2]))[0]
    y.backward(torch.full_like(y, math.nan).index_fill_(0, ints([0, 1], torch.int64), 1.0))
    assert x.grad[:2].isfinite().all() and (x.grad[2] == 0).all()
    # tokens past the count: no gradient, whatever is in theirs
    x.grad = None
    y = fb.head_norm_rope(x, None, None, None, None, None, count=ints([2]))[0]
    y.backward(torch.full_like(y, math.nan).index_fill_(0, ints([0, 1], torch.int64), 1.0))
    assert x.grad[:2].isfinite().all() and (x.grad[2] == 0).all()
    with pytest.raises(ValueError):             # results written in place keep no way back
        fb.head_norm_rope(q, None, wq, None, None, None, q_out=torch.empty_like(q))


# ------------------------------------------------------------------------------------------------------- bounded waits

def test_prompt_waits_that_run_out_are_reported_and_harm_nothing():
    """With a limit of nothing the first wait that is not over at once is given up: the kernel ends, the next poll says so, and the next
    call is right."""
    a = Attention(lens=[900, 300], queries=[400, 260], q_heads=8, kv_heads=2, dim=128, seed=18, room=1024)
    want = a.run(max_query=MANY)
    a.kv.poll_status()
    a.kv.set_wait_limit(1)
    a.run(max_query=MANY)
    with pytest.raises(fb.FiError) as e:
        a.kv.poll_status()
    assert e.value.status == fb.FI_ERR_TIMEOUT and "bounded wait" in str(e.value)
    a.kv.set_wait_limit()
    for _ in range(2):
        got = a.run(max_query=MANY)
        a.kv.poll_status()                       # reported once
        assert torch.equal(got[0][:660], want[0][:660]) and torch.equal(got[1][:660], want[1][:660])
    for bad in (1 << 40, -5):
        with pytest.raises(fb.FiError):
            a.kv.set_wait_limit(bad)
