"""The rings that bring long rows: waits that run out, rings of one stage, results written where rows come from while later rows are on their
way."""
import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [(a, b) for a in (torch.bfloat16, torch.float32) for b in (torch.bfloat16, torch.float32)]


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


@pytest.mark.parametrize("tokens,dim", [(1500, 2048), (1400, 4096), (2000, 8192), (1300, 16384), (1250, 1032)])
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
def test_a_wait_that_runs_out_is_reported(tokens, dim, types):
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x, w, b, dy = rand(gen, tokens, dim).to(types[0]), 1 + 0.2 * rand(gen, dim), rand(gen, dim), rand(gen, tokens, dim).to(types[1])
    for rms in (False, True):
        forward = lambda **kw: (fb.layer_norm(x, w, b, rms=rms, out_dtype=types[1], **kw),)
        backward = lambda **kw: fb.layer_norm_backward(x, w, dy, rms=rms, with_bias=True, **kw)
        for call in (forward, backward):
            want = call()
            fb.layer_norm_poll_status()
            call(wait_limit=1000)
            with pytest.raises(fb.FiError, match="TIMEOUT"):
                fb.layer_norm_poll_status()
            fb.layer_norm_poll_status()
            assert all(torch.equal(s, t) for s, t in zip(want, call()))
            assert all(torch.equal(s, t) for s, t in zip(want, call(wait_limit=1 << 40)))
            fb.layer_norm_poll_status()


def test_rings_of_rows_of_700_values_and_limits_that_are_refused():
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = rand(gen, 3000, 704), rand(gen, 3000, 704)
    want = fb.layer_norm_backward(x, None, dy)
    fb.layer_norm_backward(x, None, dy, wait_limit=1000)
    with pytest.raises(fb.FiError, match="TIMEOUT"):
        fb.layer_norm_poll_status()
    assert torch.equal(want[0], fb.layer_norm_backward(x, None, dy)[0])
    fb.layer_norm_poll_status()
    for call in (lambda: fb.layer_norm(x, wait_limit=-1), lambda: fb.layer_norm_backward(x, None, dy, wait_limit=-1)):
        with pytest.raises(fb.FiError, match="INVALID"):
            call()


def near(got, want, dtype):
    """The same sums in another order: a few hundred roundings of 2^-24 of sums over a row, and one to the type."""
    half = 2.0 ** -7 if dtype is torch.bfloat16 else 2.0 ** -23
    got, want = got.double(), want.double()
    size = want.abs().amax(-1, keepdim=True)
    far, bound = (got - want).abs(), half * want.abs() + 300 * 2.0 ** -24 * size
    assert (far <= bound).all(), (far / bound).max()


@pytest.mark.parametrize("tokens,dim", [(1400, 16384), (700, 12000), (500, 11168), (1300, 11160), (900, 8200)])
@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
def test_long_rows_many_times_round_the_ring(tokens, dim, types):
    """From 11,168 values on a CTA has room for one row of float32 and its gradient: loading and work take turns there."""
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x, w, dy = rand(gen, tokens, dim).to(types[0]), 1 + 0.2 * rand(gen, dim), rand(gen, tokens, dim).to(types[1])
    dx, dw, db = fb.layer_norm_backward(x, w, dy, with_bias=True)
    y = fb.layer_norm(x, w, out_dtype=types[1])
    fb.layer_norm_poll_status()
    d = x.double()
    d = d - d.mean(-1, keepdim=True)
    r = 1 / ((d * d).mean(-1, keepdim=True) + 1e-5).sqrt()
    n, g = d * r, dy.double() * w.double()
    near(y, n * w.double(), types[1])
    near(dx, r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True)), types[0])
    for got, each in ((dw, dy.double() * n), (db, dy.double())):
        # a sum over the rows, in float32: each addition is off by 2^-24 of the sum of sizes at most, n by 60 2^-24 of 1 + |n|
        bound = (tokens + 60) * 2.0 ** -24 * each.abs().sum(0) + 60 * 2.0 ** -24 * dy.double().abs().sum(0)
        assert ((got.double() - each.sum(0)).abs() <= bound).all()
    again = fb.layer_norm_backward(x, w, dy, with_bias=True)
    assert all(torch.equal(s, t) for s, t in zip((dx, dw, db), again))


@pytest.mark.parametrize("tokens,dim", [(5000, 2048), (4000, 4096), (3000, 8192), (1500, 16384), (6000, 1032)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_in_place_while_later_rows_are_on_their_way(tokens, dim, dtype):
    gen = torch.Generator(device=DEV).manual_seed(dim)
    x, w, b, dy = rand(gen, tokens, dim).to(dtype), 1 + 0.2 * rand(gen, dim), rand(gen, dim), rand(gen, tokens, dim).to(dtype)
    for rms in (False, True):
        want = fb.layer_norm(x, w, b, rms=rms)
        into = x.clone()
        assert fb.layer_norm(into, w, b, rms=rms, out=into) is into
        assert torch.equal(into, want)
        ref = fb.layer_norm_backward(x, w, dy, rms=rms, with_bias=True)
        into = dy.clone()
        got = fb.layer_norm_backward(x, w, into, rms=rms, with_bias=True, dx=into)
        assert got[0] is into and all(torch.equal(s, t) for s, t in zip(ref, got))
    fb.layer_norm_poll_status()


def test_the_report_names_both_directions():
    gen = torch.Generator(device=DEV).manual_seed(2)
    x = rand(gen, 1500, 2048)
    for call in (lambda: fb.layer_norm(x, wait_limit=1000), lambda: fb.layer_norm_backward(x, None, x, wait_limit=1000)):
        call()
        with pytest.raises(fb.FiError, match=r"fi_layer_norm, fi_layer_norm_backward: a wait"):
            fb.layer_norm_poll_status()
