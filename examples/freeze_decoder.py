"""Decoding with attention layers behind freeze caches: a small random-weight model, run step by step.

Every layer first looks its input up in its freeze cache; the requests that it freezes skip the layer and all later ones,
the others (known on the device only) run it: their query, key and value heads are normed and rotated, a place is found in the
layer's paged key/value store, keys and values are stored there in 4 bits, and the queries attend to what is stored.  A
request that was frozen before a layer leaves no token there, so every layer has its own lengths and page tables; a
token's angle goes by its place in the request, not in a layer's store, which has holes where the request was frozen.  No
call waits for the host.

    python examples/freeze_decoder.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_02645_b200 import binding as fb  # noqa: E402


class FreezeDecoderLayer:
    """Weights, freeze cache, and key/value store of one layer."""

    def __init__(self, hidden, q_heads, kv_heads, head_dim, requests, max_keys, page_size, gen, cache_entries=256):
        dev = gen.device
        rand = lambda *s: torch.randn(*s, generator=gen, device=dev)
        self.heads, self.kv_heads, self.head_dim = q_heads, kv_heads, head_dim
        self.w_qkv = (rand(hidden, (q_heads + 2 * kv_heads) * head_dim) * hidden ** -0.5).to(torch.bfloat16)
        self.w_out = (rand(q_heads * head_dim, hidden) * (q_heads * head_dim) ** -0.5).to(torch.bfloat16)
        self.q_weight, self.k_weight = 1 + 0.1 * rand(head_dim), 1 + 0.1 * rand(head_dim)
        # the freeze cache: stand-ins for the activations a trained network would have left
        self.cache = fb.FreezeCache(dim=hidden, capacity=cache_entries, num_classes=10, k=3, max_batch=requests)
        self.cache.insert(rand(cache_entries, hidden).to(torch.bfloat16),
                          torch.randint(0, 10, (cache_entries,), generator=gen, device=dev, dtype=torch.int32))
        # the key/value store: pools, page tables, all of them on the device
        blocks = -(-max_keys // page_size)
        pages = requests * blocks
        codes = lambda: torch.zeros(pages, kv_heads, page_size, head_dim // 2, dtype=torch.uint8, device=dev)
        meta = lambda: torch.zeros(pages, kv_heads, page_size, 2, dtype=torch.bfloat16, device=dev)
        self.kv = fb.KvCache(codes(), meta(), codes(), meta(), q_heads=q_heads)
        self.tables = fb.KvTables(page_size=page_size, max_blocks=blocks, max_batch=requests, device=dev.index or 0)
        self.block_table = torch.full((requests, blocks), -1, dtype=torch.int32, device=dev)
        self.free_pages = torch.arange(pages, dtype=torch.int32, device=dev)
        self.out = fb.ExtendOut(requests, requests, requests, dev)
        self.out.lens.zero_()
        self.out.free_count.fill_(pages)

    def run(self, x, rope, positions, rows, count):
        """x [requests, hidden]: the survivors' activations, in the order of `rows` ([requests], `count` of them real), at
        `positions` in their requests.  Returns what the layer adds to them (rows past the count hold anything) and what its attention saw."""
        n = x.shape[0]
        step = self.tables.extend(self.out.lens, self.free_pages, self.out.free_count, self.block_table, row_idx=rows,
                                  batch_count=count, out=self.out)             # lengths and free count are updated in place
        normed = torch.nn.functional.rms_norm(x.float(), x.shape[1:]).to(x.dtype)
        qkv = (normed @ self.w_qkv).view(n, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], 1)
        q, k = fb.head_norm_rope(q, k, self.q_weight, self.k_weight, rope, positions, count=count)
        self.kv.append(k, v, step.slot_map)
        # (a request that found no place, because it is longer than the table or pages are out, sees nothing here)
        a = self.kv.attend(q, step.lens, self.block_table, cu_tokens=step.cu_tokens, row_idx=rows, batch_count=count,
                           granted=step.granted)
        return a.reshape(n, -1) @ self.w_out, (q, k, v, a)

    def release(self, rows):
        """The requests in these rows have ended: their pages are free again."""
        self.tables.release(rows, self.out.lens, self.free_pages, self.out.free_count, self.block_table,
                            out=(self.out.lens, self.out.free_count))


class FreezeDecoder:
    def __init__(self, *, layers=4, hidden=512, q_heads=8, kv_heads=2, head_dim=64, requests=16, max_keys=256, page_size=16,
                 device="cuda:0", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.layers = [FreezeDecoderLayer(hidden, q_heads, kv_heads, head_dim, requests, max_keys, page_size, gen)
                       for _ in range(layers)]
        angles = torch.arange(max_keys, device=device)[:, None] * 10000.0 ** (-torch.arange(0, head_dim, 2, device=device) / head_dim)
        self.rope = torch.cat([angles.cos(), angles.sin()], 1).contiguous()
        self.requests, self.hidden, self.device = requests, hidden, torch.device(device)
        self.slots = torch.arange(requests, device=device)
        self.max_keys, self.steps = max_keys, 0
        self.positions = torch.zeros(requests + 1, dtype=torch.int32, device=device)    # of each request's next token

    def calibrate(self, h, share):
        """Sets every layer's threshold so that it would freeze `share` of the requests at the activations that reach it."""
        rows = torch.arange(self.requests, dtype=torch.int32, device=self.device)
        count = torch.full((1,), self.requests, dtype=torch.int32, device=self.device)
        for layer in self.layers:
            layer.cache.set_threshold(float(layer.cache.lookup_batch(h).conf.quantile(1 - share)))
            h = h + layer.run(h, self.rope, self.positions, rows, count)[0]
        for layer in self.layers:
            layer.release(rows)

    def step(self, h, observe=None):
        """One token of every request: h [requests, hidden] bf16 -> (h behind the layers, CascadeState with labels, exit stages and
        confidences).  A frozen request's h stays what the layer that froze it was given."""
        if self.steps == self.max_keys:
            raise RuntimeError(f"a request has room for {self.max_keys} tokens")
        state = fb.CascadeState(self.requests, self.device)
        fb.cascade_init(state, len(self.layers))
        work = torch.cat([h, h[:1]])                                            # one row more, for slots without a request
        for i, layer in enumerate(self.layers):
            fb.cascade_step(layer.cache, work[:-1], state, i)
            rows, count = state.survivors(i)
            here = torch.where(self.slots < count, rows, self.requests).long()
            x = work[here]
            y, seen = layer.run(x, self.rope, self.positions[here], rows, count)
            if observe:
                observe(i, rows, count, *seen)
            work[here] = x + y
        self.positions += 1
        self.steps += 1
        return work[:-1], state


def main():
    steps = int(sys.argv[1]) if len(sys.argv) > 1 else 64
    torch.manual_seed(0)
    model = FreezeDecoder(max_keys=max(256, steps))
    h = torch.randn(model.requests, model.hidden, device=model.device).to(torch.bfloat16)
    model.calibrate(h, 0.1)
    frozen = torch.zeros(len(model.layers) + 1, dtype=torch.int64)
    for _ in range(steps):
        h, state = model.step(h)
        h = (h + torch.randn_like(h)).to(torch.bfloat16) * 0.7                  # stands in for the next token's embedding
        frozen += torch.bincount(state.exit_stage.cpu().long(), minlength=len(model.layers) + 1)
    for i, layer in enumerate(model.layers):
        layer.kv.poll_status()
        print(f"layer {i}: froze {int(frozen[i])} of {steps * model.requests} tokens, keys stored per request "
              f"{layer.out.lens.tolist()}")
    print(f"never frozen: {int(frozen[-1])}")


if __name__ == "__main__":
    main()
