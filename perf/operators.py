"""The operators of a transformer layer behind a freeze cache, as they are measured: their cases, inputs, plain forms and
64-bit values.

When a network's layers are attention layers, the requests that a layer's cache did not freeze go on to the next one:
their queries and keys are normed and rotated ("norm"), pages of that layer's key/value cache are found for their new
tokens on the GPU ("tables"), the keys and values are stored there in 4 bits ("append"), and the queries attend to what
is stored ("attend").

Layout of the 4-bit cache: codes [pages, kv_heads, page_size, head_dim / 2] bytes, byte j of a vector holds value 2j in
its low and value 2j + 1 in its high half; meta [pages, kv_heads, page_size, 2] bf16, scale and offset of the vector;
a value is code * scale + offset.  `own` chooses who computes: elementary torch operations, or the library.
"""
import math

import torch

own = False

TINY = 2.0 ** -40          # smallest scale a vector is stored with
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one token for each of the 256 requests that are left of 1,024: a decode step's tables
        {"name": "tables-decode", "op": "tables", "rows": 1024, "batch": 256, "alive": 251, "page": 16, "blocks": 512,
         "new": 1, "finished": 0},
        # 512 prompts of up to 2,500 tokens join at once, behind 64 requests that have ended
        {"name": "tables-prompts", "op": "tables", "rows": 4096, "batch": 512, "alive": 512, "page": 64, "blocks": 160,
         "new": 2500, "finished": 64},
        # decode step of 16 requests
        {"name": "norm-decode", "op": "norm", "tokens": 16, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "dtype": "bf16", "backward": False},
        # prompts of 16,384 tokens in all
        {"name": "norm-prompts", "op": "norm", "tokens": 16384, "q_heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "dtype": "bf16", "backward": False},
        # training of the norm weights and what is before them; half of each head is rotated, odd token count
        {"name": "norm-gradient", "op": "norm", "tokens": 8191, "q_heads": 16, "kv_heads": 4, "dim": 128, "rot": 64,
         "interleaved": True, "dtype": "bf16", "backward": True},
        # a decode step's 64 new tokens
        {"name": "append-decode", "op": "append", "tokens": 64, "kv_heads": 8, "dim": 128, "page": 16, "pages": 64,
         "dtype": "bf16"},
        # prompts of 16,383 tokens, pages of 64 that the last tokens do not fill
        {"name": "append-prompts", "op": "append", "tokens": 16383, "kv_heads": 8, "dim": 128, "page": 64, "pages": 300,
         "dtype": "bf16"},
        # one request with a short context: the latency of a single token
        {"name": "attend-one", "op": "attend", "batch": 1, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16,
         "context": 511, "spread": 0.0, "queries": 1, "window": 0, "dtype": "bf16"},
        # decode step of 64 requests whose contexts differ widely
        {"name": "attend-batch", "op": "attend", "batch": 64, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 16,
         "context": 8192, "spread": 0.9, "queries": 1, "window": 0, "dtype": "bf16"},
        # one request with a long context: a single token, work cut along the cache
        {"name": "attend-long", "op": "attend", "batch": 1, "q_heads": 64, "kv_heads": 8, "dim": 128, "page": 64,
         "context": 262143, "spread": 0.0, "queries": 1, "window": 0, "dtype": "bf16"},
        # a few drafted tokens for each request, windowed layer, float32 activations, five queries to a key head
        {"name": "attend-draft", "op": "attend", "batch": 16, "q_heads": 20, "kv_heads": 4, "dim": 64, "page": 16,
         "context": 4000, "spread": 0.5, "queries": 5, "window": 1024, "dtype": "f32"},
        # a chunk of two prompts behind what is cached already
        {"name": "attend-chunk", "op": "attend", "batch": 2, "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 64,
         "context": 8192, "spread": 0.1, "queries": 1024, "window": 0, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("tables", "norm", "append", "attend", "attend"))
    if op == "tables":
        batch = _log(rng, 1, 1024)
        new = 1 if rng.random() < 0.5 else _log(rng, 2, max(2, min(4096, 1200000 // batch)))
        page = rng.choice((16, 32, 64, 128))
        return {"op": op, "rows": batch + _log(rng, 64, 3000), "batch": batch, "alive": rng.randint(0, batch), "page": page,
                "blocks": (2 * new + 4095) // page + rng.randint(1, 9), "new": new,
                "finished": 0 if rng.random() < 0.5 else rng.randint(1, 64)}
    if op == "norm":
        kv_heads, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 80, 112, 128, 192, 256))
        group = rng.choice((1, 2, 4, 5, 7, 8))
        most = 16384 * 40 * 128 // ((group + 1) * kv_heads * dim)
        backward = rng.random() < 0.4
        return {"op": op, "tokens": _log(rng, 1, min(16384, most // 2 if backward else most)), "q_heads": group * kv_heads,
                "kv_heads": kv_heads, "dim": dim, "rot": rng.choice((dim, dim, dim // 32 * 16)),
                "interleaved": rng.random() < 0.3, "dtype": rng.choice(("bf16", "bf16", "f32")), "backward": backward}
    if op == "append":
        kv_heads, dim, page = rng.choice((1, 2, 4, 5, 8)), rng.choice((64, 128, 192, 256)), rng.choice((16, 32, 64, 128))
        tokens = _log(rng, 1, min(16384, 16384 * 8 * 128 // (kv_heads * dim)))
        return {"op": op, "tokens": tokens, "kv_heads": kv_heads, "dim": dim, "page": page,
                "pages": tokens // page + rng.randint(2, 40), "dtype": rng.choice(("bf16", "bf16", "f32"))}
    kv_heads, group = rng.choice((1, 2, 4, 5, 8)), rng.choice((1, 2, 4, 5, 7, 8, 16))
    dim, page = rng.choice((64, 128, 128, 192, 256)), rng.choice((16, 32, 64, 128))
    batch = _log(rng, 1, 256)
    queries = rng.choice((1, 1, 1, rng.randint(2, 8), _log(rng, 9, 1024)))
    most = 262144 * 8 * 128 // (batch * kv_heads * dim)
    most = min(most, 2 * 32 * 1024 * 8192 * 128 // (batch * group * kv_heads * queries * dim), 131072)
    context = _log(rng, 1, max(1, most))
    return {"op": op, "batch": batch, "q_heads": group * kv_heads, "kv_heads": kv_heads, "dim": dim, "page": page,
            "context": context, "spread": rng.choice((0.0, 0.3, 0.9)), "queries": min(queries, context),
            "window": rng.choice((0, 0, 0, _log(rng, 1, 4096))), "dtype": rng.choice(("bf16", "bf16", "f32"))}


# ------------------------------------------------------------------------------------------------------------ inputs

def _lens(case, gen, dev):
    """Context lengths (the new tokens among them): `spread` of 0 gives them all alike."""
    lo = max(case["queries"], int(case["context"] * (1.0 - case["spread"])))
    return torch.randint(lo, case["context"] + 1, (case["batch"],), generator=gen, device=dev, dtype=torch.int32)


def _tables(case, gen, dev):
    rows, batch, page, blocks = case["rows"], case["batch"], case["page"], case["blocks"]
    most = blocks * page - case["new"]
    lens = torch.randint(0, min(most, 4096) + 1, (rows,), generator=gen, device=dev, dtype=torch.int32)
    order = torch.randperm(rows, generator=gen, device=dev)
    row_idx = order[:batch].sort().values.to(torch.int32)
    ended = order[batch:batch + case["finished"]].to(torch.int32)
    if case["new"] > 1:
        lens[row_idx.long()] = 0                       # prompts join with nothing cached
        new_lens = torch.randint(1, case["new"] + 1, (batch,), generator=gen, device=dev, dtype=torch.int32)
    else:
        new_lens = None
    used = (lens + page - 1) // page
    start = used.cumsum(0) - used
    taken = int(used.sum())
    spare = batch * ((case["new"] + page - 1) // page + 1) // 2 + 1   # about what is wanted: now and then too few
    pages = torch.randperm(taken + spare, generator=gen, device=dev).to(torch.int32)
    col = torch.arange(blocks, device=dev)
    at = (start[:, None] + col).clamp(max=max(taken - 1, 0))
    table = torch.where(col < used[:, None], pages[at], -1).to(torch.int32)
    free = torch.cat([pages[taken:], torch.full((taken,), -1, dtype=torch.int32, device=dev)])
    return {"lens": lens, "row_idx": row_idx, "ended": ended, "new_lens": new_lens, "table": table, "free": free,
            "free_count": torch.tensor([spare], dtype=torch.int32, device=dev),
            "alive": torch.tensor([case["alive"]], dtype=torch.int32, device=dev),
            "max_tokens": batch * case["new"]}


def _rope(positions, rot, dev):
    """[positions, rot]: cosines, then sines, of position * 10000^(-2 i / rot)."""
    i = torch.arange(rot // 2, device=dev, dtype=torch.float64)
    a = torch.arange(positions, device=dev, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * i / rot)
    return torch.cat([a.cos(), a.sin()], 1).float()


def _norm(case, gen, dev):
    t, hq, hk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["dim"]
    dtype = _DTYPE[case["dtype"]]
    make = lambda: torch.randn(t, hq + 2 * hk, d, generator=gen, device=dev).to(dtype)   # one product's q, k and v
    qkv = make()
    st = {"q": qkv[:, :hq], "k": qkv[:, hq:hq + hk],
          "q_weight": 1 + 0.1 * torch.randn(d, generator=gen, device=dev),
          "k_weight": 1 + 0.1 * torch.randn(d, generator=gen, device=dev),
          "rope": _rope(32768, case["rot"], dev),
          "positions": torch.randint(0, 32768 - t, (1,), generator=gen, device=dev, dtype=torch.int32)
          + torch.arange(t, device=dev, dtype=torch.int32)}
    if case["backward"]:
        grad = make()
        st["dq"], st["dk"] = grad[:, :hq], grad[:, hq:hq + hk]
    return st


def _empty_cache(pages, heads, page, dim, dev):
    return {"codes": torch.zeros(pages, heads, page, dim // 2, dtype=torch.uint8, device=dev),
            "meta": torch.zeros(pages, heads, page, 2, dtype=torch.bfloat16, device=dev)}


def _append(case, gen, dev):
    t, h, d, page, pages = case["tokens"], case["kv_heads"], case["dim"], case["page"], case["pages"]
    qkv = torch.randn(t, 6 * h, d, generator=gen, device=dev).to(_DTYPE[case["dtype"]])
    order = torch.randperm(pages, generator=gen, device=dev)
    at = torch.arange(t, device=dev)
    st = {"k": qkv[:, 4 * h:5 * h], "v": qkv[:, 5 * h:], "slots": order[at // page] * page + at % page}
    for n in ("k", "v"):
        c = _empty_cache(pages, h, page, d, dev)
        st[n + "_codes"], st[n + "_meta"] = c["codes"], c["meta"]
    return st


def _attend(case, gen, dev):
    b, hk, d, page = case["batch"], case["kv_heads"], case["dim"], case["page"]
    lens = _lens(case, gen, dev)
    blocks = (case["context"] + page - 1) // page
    pages = b * blocks
    table = torch.randperm(pages, generator=gen, device=dev).to(torch.int32).view(b, blocks)
    most = case["queries"]
    new = torch.full((b,), most, device=dev, dtype=torch.int32)
    if 1 < most <= 8:                                      # drafted tokens: 1 to `most`, whoever got how many
        new = (torch.randperm(b, generator=gen, device=dev) % most + 1).to(torch.int32)
    cu = torch.zeros(b + 1, dtype=torch.int32, device=dev)
    cu[1:] = new.cumsum(0)
    st = {"q": torch.randn(int(cu[-1]), case["q_heads"], d, generator=gen, device=dev).to(_DTYPE[case["dtype"]]),
          "lens": lens, "table": table, "cu": cu, "max_query": most}
    for n in ("k", "v"):
        c = _empty_cache(pages, hk, page, d, dev)
        part = max(1, (1 << 27) // (hk * page * d))
        for p in range(0, pages, part):                    # what append stores for normal values
            x = torch.randn(min(part, pages - p), hk, page, d, generator=gen, device=dev)
            c["codes"][p:p + part], c["meta"][p:p + part] = _pack(*_quantise(x))
        st[n + "_codes"], st[n + "_meta"] = c["codes"], c["meta"]
    return st


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"tables": _tables, "norm": _norm, "append": _append, "attend": _attend}[case["op"]](case, gen, dev)
    st["case"] = case
    if own:                                                # the handle of the layer's cache, which a program keeps
        from paper_2002_02645_b200 import binding as fb
        st["fb"] = fb
        if case["op"] == "tables":
            st["kv"] = fb.KvTables(page_size=case["page"], max_blocks=case["blocks"], max_batch=case["batch"] + 64)
        elif case["op"] in ("append", "attend"):
            st["kv"] = fb.KvCache(st["k_codes"], st["k_meta"], st["v_codes"], st["v_meta"],
                                  q_heads=case.get("q_heads", case["kv_heads"]))
    return st


# ------------------------------------------------------------------------------------------------------- plain forms

def _release_plain(st, page):
    lens, table, free, count = st["lens"], st["table"], st["free"], st["free_count"]
    rows = st["ended"].long()
    used = (lens[rows] + page - 1) // page
    cum = used.cumsum(0)
    col = torch.arange(table.shape[1], device=table.device)
    at = torch.where(col < used[:, None], count + (cum - used)[:, None] + col, free.numel())
    longer = torch.cat([free, free[:1]])                   # one place more, for what is not written
    longer[at] = table[rows]
    lens = lens.clone()
    lens[rows] = 0
    return lens, longer[:-1], count + cum[-1:].to(torch.int32)


def _tables_plain(st):
    case = st["case"]
    page, blocks, batch = case["page"], case["blocks"], case["batch"]
    lens, table, free, count = st["lens"], st["table"].clone(), st["free"], st["free_count"]
    if case["finished"]:
        lens, free, count = _release_plain(st, page)
    rows = st["row_idx"].long()
    dev = rows.device
    alive = torch.arange(batch, device=dev) < st["alive"]
    have = lens[rows]
    new = torch.ones_like(have) if st["new_lens"] is None else st["new_lens"]
    new = torch.where(alive, new, 0)
    cu = torch.zeros(batch + 1, dtype=torch.int32, device=dev)
    cu[1:] = new.cumsum(0)
    had, want = (have + page - 1) // page, (have + new + page - 1) // page
    fits = alive & (want <= blocks) & (cu[1:] <= st["max_tokens"])
    need = torch.where(fits, want - had, 0)
    cum = need.cumsum(0)
    given = fits & ((need == 0) | (cum <= count))
    first = count - 1 - (cum - need)                       # pages are taken from the end of the list
    col = torch.arange(blocks, device=dev)
    fresh = given[:, None] & (col >= had[:, None]) & (col < want[:, None])
    page_of = torch.where(fresh, free[(first[:, None] - (col - had[:, None])).clamp(0, free.numel() - 1)], table[rows])
    table[rows] = page_of
    t = torch.arange(st["max_tokens"], device=dev, dtype=torch.int32)
    i = torch.searchsorted(cu[1:], t, right=True).clamp(max=batch - 1)
    real = t < cu[-1]
    pos = have[i] + t - cu[i]
    slot = page_of[i, (pos // page).clamp(0, blocks - 1)].long() * page + pos % page
    granted = torch.where(given, new, 0)
    lens_out = lens.clone()
    lens_out[rows] = have + granted
    got = torch.where(given, need, 0).sum().to(torch.int32)
    return {"slot_map": torch.where(real & given[i], slot, -1), "positions": torch.where(real, pos, -1).to(torch.int32),
            "cu_tokens": cu, "granted": granted.to(torch.int32), "lens": lens_out, "free_count": count - got, "table": table}


def _rotate(x, c, s, rot, interleaved, back):
    """Rotation of each pair of the first `rot` values; `back`: by the opposite angle."""
    if back:
        s = -s
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    ra, rb = a * c - b * s, b * c + a * s
    r = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _norm_plain(st):
    case = st["case"]
    rot, eps = case["rot"], 1e-6
    table = st["rope"][st["positions"].long()][:, None]
    c, s = table[..., :rot // 2], table[..., rot // 2:]

    def one(x, w):
        x32 = x.float()
        y = x32 * torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + eps) * w
        return _rotate(y, c, s, rot, case["interleaved"], False).to(x.dtype)

    def back(x, w, dy):
        x32, g = x.float(), _rotate(dy.float(), c, s, rot, case["interleaved"], True)
        r = torch.rsqrt((x32 * x32).mean(-1, keepdim=True) + eps)
        n = x32 * r
        gw = g * w
        dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
        return dx.to(x.dtype), (g * n).sum((0, 1))

    if not case["backward"]:
        return {"q": one(st["q"], st["q_weight"]), "k": one(st["k"], st["k_weight"])}
    dq, dwq = back(st["q"], st["q_weight"], st["dq"])
    dk, dwk = back(st["k"], st["k_weight"], st["dk"])
    return {"dq": dq, "dk": dk, "dq_weight": dwq, "dk_weight": dwk}


def _down(x):
    """Largest bf16 value that is not above x, as float32."""
    bits = x.view(torch.int32)
    cut = bits & -65536
    return torch.where((x < 0) & (bits != cut), cut + 65536, cut).view(torch.float32)


def _quantise(x):
    """Codes, scale and offset of each vector along the last axis, in float32."""
    low, high = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    offset = _down(low)
    scale = (-_down(-((high - offset) / torch.full((), 15.0, device=x.device)))).clamp(min=TINY)
    code = ((x - offset) / scale).round().clamp(0, 15)
    return code, scale, offset


def _pack(code, scale, offset):
    c = code.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.cat([scale, offset], -1).to(torch.bfloat16)


def _append_plain(st):
    page, out = st["k_codes"].shape[2], {}
    where, off = st["slots"] // page, st["slots"] % page

    def one(x, n):
        code, scale, offset = _quantise(x.float())
        codes, meta = _pack(code, scale, offset)
        st[n + "_codes"][where, :, off], st[n + "_meta"][where, :, off] = codes, meta
        out.update({n + "_codes": st[n + "_codes"], n + "_meta": st[n + "_meta"],
                    n + "_stored": (code * scale + offset).to(x.dtype)})

    one(st["k"], "k")
    one(st["v"], "v")
    return out


def _attend_plain(st):
    case = st["case"]
    b, hq, hk, d, page = case["batch"], case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    most, lens, cu, table = st["max_query"], st["lens"], st["cu"], st["table"].long()
    dev, span = table.device, table.shape[1] * page

    def values(n):                                         # [b, hk, span, d]
        codes, meta = st[n + "_codes"][table], st[n + "_meta"][table].float()
        x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
        return (x * meta[..., :1] + meta[..., 1:]).transpose(1, 2).reshape(b, hk, span, d)

    new = cu[1:] - cu[:-1]
    j = torch.arange(most, device=dev)
    at = (cu[:-1, None] + j).clamp(max=st["q"].shape[0] - 1)
    q = st["q"].float()[at].view(b, most, hk, hq // hk, d).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, d)
    x = (q @ values("k").transpose(-1, -2)).view(b, hk, hq // hk, most, span) / math.sqrt(d)
    last = (lens - new)[:, None] + j                       # the last position a query sees: its own
    t = torch.arange(span, device=dev)
    seen = (t <= last[..., None]) & (j < new[:, None])[..., None]
    if case["window"]:
        seen = seen & (t > last[..., None] - case["window"])
    x = x.masked_fill(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    o = (p.view(b, hk, -1, span) @ values("v")).view(b, hk, hq // hk, most, d) / total.clamp(min=1e-37)
    lse = (top + total.log()).squeeze(-1)
    tokens = st["q"].shape[0]
    to = torch.where(j < new[:, None], at, tokens)         # one row more, for the queries that there are not
    out = torch.empty(tokens + 1, hq, d, dtype=st["q"].dtype, device=dev)
    out[to] = o.permute(0, 3, 1, 2, 4).reshape(b, most, hq, d).to(out.dtype)
    lse_out = torch.empty(tokens + 1, hq, device=dev)
    lse_out[to] = lse.permute(0, 3, 1, 2).reshape(b, most, hq)
    return {"out": out[:-1], "lse": lse_out[:-1]}


# -------------------------------------------------------------------------------------------------------------- runs

def _tables_own(st):
    kv, case = st["kv"], st["case"]
    lens, count = st["lens"], st["free_count"]
    if case["finished"]:
        lens, count = kv.release(st["ended"], lens, st["free"], count, st["table"])
    out = kv.extend(lens, st["free"], count, st["table"], new_lens=st["new_lens"], row_idx=st["row_idx"],
                    batch_count=st["alive"], max_tokens=st["max_tokens"])
    return {"slot_map": out.slot_map, "positions": out.positions, "cu_tokens": out.cu_tokens, "granted": out.granted,
            "lens": out.lens, "free_count": out.free_count, "table": st["table"]}


def _norm_own(st):
    case, fb = st["case"], st["fb"]
    if not case["backward"]:
        q, k = fb.head_norm_rope(st["q"], st["k"], st["q_weight"], st["k_weight"], st["rope"], st["positions"],
                                 eps=1e-6, interleaved=case["interleaved"])
        return {"q": q, "k": k}
    dq, dk, dwq, dwk = fb.head_norm_rope_backward(st["q"], st["k"], st["q_weight"], st["k_weight"], st["rope"],
                                                  st["positions"], st["dq"], st["dk"], eps=1e-6,
                                                  interleaved=case["interleaved"])
    return {"dq": dq, "dk": dk, "dq_weight": dwq, "dk_weight": dwk}


def _append_own(st):
    ks, vs = st["kv"].append(st["k"], st["v"], st["slots"], with_stored=True)
    return {"k_codes": st["k_codes"], "k_meta": st["k_meta"], "k_stored": ks,
            "v_codes": st["v_codes"], "v_meta": st["v_meta"], "v_stored": vs}


def _attend_own(st):
    out, lse = st["kv"].attend(st["q"], st["lens"], st["table"], cu_tokens=st["cu"], max_query=st["max_query"],
                               window=st["case"]["window"], with_lse=True)
    return {"out": out, "lse": lse}


def run(state):
    ops = {"tables": (_tables_plain, _tables_own), "norm": (_norm_plain, _norm_own),
           "append": (_append_plain, _append_own), "attend": (_attend_plain, _attend_own)}
    return ops[state["case"]["op"]][1 if own else 0](state)


# -------------------------------------------------------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: each input once, each output once (expected values where lengths are drawn)."""
    op = case["op"]
    if op == "tables":
        tokens = case["alive"] * (1 if case["new"] == 1 else (case["new"] + 1) / 2)
        padded = case["batch"] * case["new"] if case["new"] > 1 else case["batch"]
        # lengths read and written, rows, page list in, slots (8 bytes) and positions out, new entries of the tables
        moved = 8 * case["rows"] + 16 * case["batch"] + 12 * padded + 8 * tokens / case["page"] + 12 * case["finished"]
        return {"bytes": moved, "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    if op == "norm":
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        moved = values * size * (3 if case["backward"] else 2) + case["tokens"] * (4 + 4 * case["rot"]) + 16 * case["dim"]
        return {"bytes": moved, "flops": values * (16 if case["backward"] else 8)}
    if op == "append":
        vectors = 2 * case["tokens"] * case["kv_heads"]
        return {"bytes": vectors * (case["dim"] * (2 * size + 0.5) + 4) + 8 * case["tokens"], "flops": 8 * vectors * case["dim"]}
    low = max(case["queries"], int(case["context"] * (1 - case["spread"])))
    context = (low + case["context"]) / 2
    queries = case["queries"]
    if 1 < queries <= 8:
        queries = sum(i % queries + 1 for i in range(case["batch"])) / case["batch"]
    keys = context - (queries - 1) / 2                     # that a query sees
    read = context
    if case["window"]:
        keys, read = min(keys, case["window"]), min(read, case["window"] + queries - 1)
    q_bytes = case["batch"] * queries * case["q_heads"] * (2 * case["dim"] * size + 4)
    kv_bytes = case["batch"] * read * case["kv_heads"] * (case["dim"] + 8)
    return {"bytes": q_bytes + kv_bytes, "flops": 4 * case["batch"] * queries * case["q_heads"] * keys * case["dim"]}


# ------------------------------------------------------------------------------------------------------------- exact

def _norm_exact(st):
    case = st["case"]
    rot, half = case["rot"], case["rot"] // 2
    angle = st["rope"][st["positions"].long()].double()
    turn = torch.complex(angle[:, :half], angle[:, half:])[:, None]

    def pairs(x):
        return torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) if case["interleaved"] else torch.complex(x[..., :half], x[..., half:rot])

    def turned(x, by):
        z, y = pairs(x) * by, x.clone()
        if case["interleaved"]:
            y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
        else:
            y[..., :half], y[..., half:rot] = z.real, z.imag
        return y

    out = {}
    for n in ("q", "k"):
        x, w = st[n].double(), st[n + "_weight"].double()
        rms = ((x ** 2).sum(-1, keepdim=True) / case["dim"] + 1e-6).sqrt()
        if not case["backward"]:
            out[n] = turned(w * x / rms, turn)
            continue
        g = turned(st["d" + n].double(), turn.conj())
        along = (g * w * x).sum(-1, keepdim=True) / case["dim"]
        out["d" + n] = g * w / rms - x * along / rms ** 3
        out["d" + n + "_weight"] = torch.einsum("thd,thd->d", g, x / rms)
    return {k: out[k] for k in (("dq", "dk", "dq_weight", "dk_weight") if case["backward"] else ("q", "k"))}


def _append_exact(st):
    out = {}
    for n in ("k", "v"):
        x = st[n].double()
        low, high = torch.aminmax(x, dim=-1, keepdim=True)
        step = lambda y: torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1e-300))) - 7)   # one place of bf16 at y
        offset = torch.floor(low / step(low)) * step(low)
        scale = (high - offset) / 15
        scale = (torch.ceil(scale / step(scale)) * step(scale)).clamp(min=TINY)
        code = torch.clamp(torch.round((x - offset) / scale), 0, 15)
        meta = st[n + "_meta"].double()
        page = meta.shape[2]
        meta[st["slots"] // page, :, st["slots"] % page] = torch.cat([scale, offset], -1)
        out.update({n + "_codes": None, n + "_meta": meta, n + "_stored": code * scale + offset})
    return out


def _attend_exact(st):
    case = st["case"]
    hq, hk, d, page = case["q_heads"], case["kv_heads"], case["dim"], case["page"]
    lens, cu = st["lens"].tolist(), st["cu"].tolist()
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    lse = torch.full(out.shape[:2], -math.inf, dtype=torch.float64, device=out.device)
    for b, length in enumerate(lens):
        n = cu[b + 1] - cu[b]
        pages = st["table"][b, :-(-length // page)].long()
        q = st["q"][cu[b]:cu[b + 1]].double()
        position = torch.arange(length - n, length, device=out.device)[:, None]
        t = torch.arange(length, device=out.device)
        hidden = t > position
        if case["window"]:
            hidden = hidden | (t <= position - case["window"])
        for h in range(hk):
            kv = []
            for name in ("k", "v"):
                c = st[name + "_codes"][pages, h].view(-1, d // 2)[:length]
                m = st[name + "_meta"][pages, h].view(-1, 2)[:length].double()
                x = torch.empty(length, d, dtype=torch.float64, device=out.device)
                x[:, 0::2], x[:, 1::2] = c % 16, c // 16
                kv.append(x * m[:, :1] + m[:, 1:])
            for g in range(h * (hq // hk), (h + 1) * (hq // hk)):
                x = (q[:, g] @ kv[0].T * d ** -0.5).masked_fill(hidden, -math.inf)
                lse[cu[b]:cu[b + 1], g] = torch.logsumexp(x, -1)
                out[cu[b]:cu[b + 1], g] = torch.softmax(x, -1) @ kv[1]
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] == "tables":
        return None
    st = prepare(case, seed)
    return {"norm": _norm_exact, "append": _append_exact, "attend": _attend_exact}[case["op"]](st)
