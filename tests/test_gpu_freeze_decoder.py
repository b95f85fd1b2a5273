"""The example decoder: cascade, page tables, norm with rotation, 4-bit store and attention run together, against an
attention in 64 bits over the keys and values that each layer's survivors left in it."""
import importlib.util
import os

import pytest
import torch

from test_gpu_kv_ops import plain_pack

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def load_example():
    spec = importlib.util.spec_from_file_location("freeze_decoder", os.path.join(ROOT, "examples", "freeze_decoder.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_decoder_steps_match_attention_over_what_survivors_left():
    ex = load_example()
    model = ex.FreezeDecoder(layers=3, hidden=256, q_heads=6, kv_heads=2, head_dim=64, requests=9, max_keys=64, seed=1)
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(9, 256, generator=gen, device="cuda").to(torch.bfloat16)
    model.calibrate(h, 0.3)
    stored = [[[] for _ in range(9)] for _ in model.layers]      # (keys, values) of each request in each layer, as stored

    def observe(i, rows, count, q, k, v, a):
        n = int(count)
        rows = rows[:n].tolist()
        assert sorted(rows) == rows
        packed = [plain_pack(t[:n].float().cpu().numpy()) for t in (k, v)]
        kv = [torch.tensor(p[3], device="cuda") for p in packed]
        # codes and offset of a value are summed apart: at most this large each
        parts = torch.tensor(15 * packed[1][1][..., 0].astype("float64"), device="cuda") + kv[1].abs().amax(-1)
        for s, row in enumerate(rows):
            stored[i][row].append((kv[0][s], kv[1][s], parts[s]))
            ks, vs, sizes = (torch.stack([t[j] for t in stored[i][row]]) for j in (0, 1, 2))   # [keys, kv heads(, head_dim)]
            qs = q[s].double().view(2, 3, 64)
            p = torch.softmax(torch.einsum("kgd,tkd->kgt", qs, ks) / 8.0, -1)
            want = torch.einsum("kgt,tkd->kgd", p, vs).reshape(6, 64)
            # the result's rounding to bf16 (2^-8), weights rounded to halves (2^-11), scores and sums in float32
            weighed = torch.einsum("kgt,tk->kg", p, sizes).reshape(6, 1)
            bound = 1.01 * 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -14) * weighed
            assert ((a[s].double() - want).abs() <= bound).all(), (i, row)

    exits = []
    for _ in range(30):
        out, state = model.step(h, observe)
        exits += state.exit_stage.tolist()
        h = (0.7 * (out + torch.randn(out.shape, generator=gen, device="cuda"))).to(torch.bfloat16)
    assert len(set(exits)) >= 3                                   # some frozen early, some later, some never
    for i, layer in enumerate(model.layers):
        layer.kv.poll_status()
        assert layer.out.lens.tolist() == [len(r) for r in stored[i]]
        assert layer.out.lens.tolist() == [sum(1 for s in range(30) if exits[9 * s + r] > i) for r in range(9)]
        free = layer.free_pages[:int(layer.out.free_count)].tolist()
        used = [p for r, n in enumerate(layer.out.lens.tolist()) for p in layer.block_table[r, :-(-n // 16)].tolist()]
        assert sorted(free + used) == list(range(36))            # every page is free or belongs to one request
        layer.release(torch.tensor([2, 5], dtype=torch.int32, device="cuda"))
        assert layer.out.lens[[2, 5]].tolist() == [0, 0]
    model.step(h)
