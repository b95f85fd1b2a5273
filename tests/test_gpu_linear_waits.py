"""Waits inside the products that run out: reported, nothing left on its way, and the call after them is right."""
import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV).bfloat16()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 2048, 2560), (1, 64, 128), (4, 512, 1024), (48, 4096, 4096), (251, 4096, 4096), (700, 512, 1024),
                                               (1000, 8192, 1024), (5000, 1024, 2048), (1, 131072, 520), (300, 65536, 520)])
def test_right_after_a_wait_that_ran_out(tokens, n_in, n_out, dtype):
    """Calls whose waits run out and whole ones in turn: copies that landed late would land in the shared memory of the next call."""
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w = rand(gen, tokens, n_in), rand(gen, n_out, n_in)
    want = fb.linear(x, w, out_dtype=dtype)
    fb.linear_poll_status()
    for limit in (1, 200, 1000, 5000):
        fb.linear(x, w, out_dtype=dtype, wait_limit=limit)
        got = fb.linear(x, w, out_dtype=dtype)
        with pytest.raises(fb.FiError, match="TIMEOUT"):
            fb.linear_poll_status()
        fb.linear_poll_status()
        assert torch.equal(got, want)


@pytest.mark.parametrize("tokens,n_in,n_out", [(3, 72, 136), (64, 4096, 4096), (777, 1000, 1400), (256, 4096, 4096), (4095, 2048, 2048), (5000, 512, 6144),
                                               (7001, 1544, 520), (200000, 64, 72), (40000, 1024, 1024)])
def test_gradients_right_after_a_wait_that_ran_out(tokens, n_in, n_out):
    """Both in one launch, in two, and each alone; with and without slopes."""
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    x, w, dy, z = rand(gen, tokens, n_in), rand(gen, n_out, n_in), rand(gen, tokens, n_out), rand(gen, tokens, n_out)
    for a, b in ((x, w), (None, w), (x, None)):
        for kw in ({}, dict(preact=z, activation="silu", with_bias=True)):
            want = fb.linear_backward(a, b, dy, **kw)
            fb.linear_poll_status()
            for limit in (1, 1000, 5000):
                fb.linear_backward(a, b, dy, wait_limit=limit, **kw)
                got = fb.linear_backward(a, b, dy, **kw)
                with pytest.raises(fb.FiError, match="TIMEOUT"):
                    fb.linear_poll_status()
                fb.linear_poll_status()
                assert all(s is t or torch.equal(s, t) for s, t in zip(got, want))
    with pytest.raises(fb.FiError, match="INVALID"):
        fb.linear_backward(x, w, dy, wait_limit=-1)
