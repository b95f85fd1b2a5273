"""The example decoder turns queries and keys by the tokens' places in their requests, whatever was frozen before, and ends where its
rope table ends."""
import pytest
import torch

from test_gpu_freeze_decoder import load_example

pytestmark = pytest.mark.gpu


def test_positions_count_frozen_tokens(monkeypatch):
    ex = load_example()
    model = ex.FreezeDecoder(layers=3, hidden=256, q_heads=4, kv_heads=2, head_dim=64, requests=9, max_keys=32, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(9, 256, generator=gen, device="cuda").to(torch.bfloat16)
    model.calibrate(h, 0.3)
    seen = []
    call = ex.fb.head_norm_rope

    def spy(q, k, qw, kw, rope, positions, *, count, **rest):
        seen.append((positions.clone(), int(count)))
        return call(q, k, qw, kw, rope, positions, count=count, **rest)

    monkeypatch.setattr(ex.fb, "head_norm_rope", spy)
    frozen = 0
    for step in range(32):
        out, state = model.step(h)
        assert len(seen) == 3
        for positions, count in seen:
            assert (positions[:count] == step).all()
        seen.clear()
        frozen += int((state.exit_stage < 3).sum())
        assert out.isfinite().all()
        h = (0.7 * (out + torch.randn(out.shape, generator=gen, device="cuda"))).to(torch.bfloat16)
    assert frozen > 9                                             # the layers' stores have holes
    assert min(model.layers[-1].out.lens.tolist()) < 32
    with pytest.raises(RuntimeError):
        model.step(h)
