"""The rest of a transformer layer behind a freeze cache, as it is measured: cases, inputs, plain forms and 64-bit values.

The requests that a layer's cache did not freeze are known on the device only, as a list of rows and a count.  Their activations
are normed out of the batch ("norm"), pass the layer's products, whose epilogues add bias, activation and the residual stream in its
place in the batch ("linear"); both have their gradients, for the training of such a layer.  Requests that branch (several
continuations of one prompt) share the pages of the key/value store that they have in common; pages are forked, given back and
brought together in the low part of the pool ("pages").  `own` chooses who computes: elementary torch operations, or the
library.
"""
import math

import torch

own = False

EPS = 1e-5
_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one request's token through a small layer's joint query, key and value product: the latency of a call
        {"name": "linear-one", "op": "linear", "tokens": 1, "alive": 1, "batch": 0, "in": 2048, "out": 2560, "act": "none", "bias": False,
         "residual": False, "dtype": "bf16", "backward": False},
        # decode step: 251 requests left of 1,024, added to the float32 residual stream in its place
        {"name": "linear-survivors", "op": "linear", "tokens": 256, "alive": 251, "batch": 1024, "in": 4096, "out": 4096, "act": "none",
         "bias": True, "residual": True, "dtype": "f32", "backward": False},
        # decode step of 48 requests through the wide product of the feed-forward part: the weights have to be read
        {"name": "linear-decode", "op": "linear", "tokens": 48, "alive": 48, "batch": 0, "in": 4096, "out": 16384, "act": "gelu", "bias": True,
         "residual": False, "dtype": "bf16", "backward": False},
        # prompts of 8,191 tokens in all through the same product
        {"name": "linear-prompts", "op": "linear", "tokens": 8191, "alive": 8191, "batch": 0, "in": 4096, "out": 16384, "act": "gelu_tanh",
         "bias": True, "residual": False, "dtype": "bf16", "backward": False},
        # training: gradients of inputs, weights and bias behind an activation; odd token count
        {"name": "linear-gradient", "op": "linear", "tokens": 4095, "alive": 4095, "batch": 0, "in": 2048, "out": 8192, "act": "silu",
         "bias": True, "residual": False, "dtype": "bf16", "backward": True},
        # the same of a ragged small layer: sizes that fill no tile
        {"name": "linear-gradient-ragged", "op": "linear", "tokens": 777, "alive": 777, "batch": 0, "in": 1000, "out": 1400, "act": "gelu",
         "bias": True, "residual": False, "dtype": "bf16", "backward": True},
        # decode step: 251 survivors' rows of the float32 residual stream, for a bf16 product
        {"name": "norm-survivors", "op": "norm", "tokens": 256, "alive": 251, "batch": 1024, "dim": 4096, "rms": False, "dtype": "f32",
         "to": "bf16", "backward": False},
        # prompts of 16,384 tokens
        {"name": "norm-prompts", "op": "norm", "tokens": 16384, "alive": 16384, "batch": 0, "dim": 4096, "rms": False, "dtype": "bf16",
         "to": "bf16", "backward": False},
        # training: gradients of inputs, weight and bias, odd token count
        {"name": "norm-gradient", "op": "norm", "tokens": 8191, "alive": 8191, "batch": 0, "dim": 4096, "rms": False, "dtype": "bf16",
         "to": "bf16", "backward": True},
        # the same in float32 where a row starts on no 16-byte boundary, by root mean square
        {"name": "norm-gradient-odd", "op": "norm", "tokens": 3001, "alive": 3001, "batch": 0, "dim": 1001, "rms": True, "dtype": "f32",
         "to": "f32", "backward": True},
        # 8 prompts of up to 4,096 tokens get 8 continuations each
        {"name": "pages-fork", "op": "pages", "kind": "fork", "rows": 256, "batch": 64, "sources": 8, "alive": 64, "context": 4096, "page": 64,
         "kv_heads": 8, "dim": 128},
        # 96 of 256 requests, among them continuations of one prompt, have ended; then the pool's used pages are brought together
        {"name": "pages-compact", "op": "pages", "kind": "compact", "rows": 256, "batch": 96, "sources": 32, "alive": 93, "context": 2048,
         "page": 16, "kv_heads": 8, "dim": 128},
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear", "norm", "norm", "pages"))
    if op == "linear":
        backward = rng.random() < 0.4
        tokens, n_in, n_out = _log(rng, 1, 8192), 8 * _log(rng, 8, 2048), 8 * _log(rng, 8, 2048)
        most = (4095 * 2048 * 8192) if backward else 8191 * 4096 * 16384
        tokens = max(1, min(tokens, most // (n_in * n_out)))
        batch = 0 if backward or rng.random() < 0.6 else tokens + _log(rng, 1, 2000)
        return {"op": op, "tokens": tokens, "alive": tokens if not batch else rng.randint(0, tokens), "batch": batch, "in": n_in, "out": n_out,
                "act": rng.choice(_ACTS), "bias": rng.random() < 0.6, "residual": batch > 0 or not backward and rng.random() < 0.3, "dtype": "bf16" if backward else rng.choice(("bf16", "bf16", "f32")),
                "backward": backward}
    if op == "norm":
        dim = rng.choice((64, 96, 128, 1000, 1024, 4096, 8192, _log(rng, 16, 16384), 8 * _log(rng, 4, 2048)))
        backward = rng.random() < 0.5
        tokens = _log(rng, 1, min(65536, 16384 * 4096 // dim // (2 if backward else 1)))
        batch = 0 if backward or rng.random() < 0.6 else tokens + _log(rng, 1, 2000)
        dtype = rng.choice(("bf16", "f32"))
        if dtype == "f32":
            tokens = max(1, tokens // 2)
        return {"op": op, "tokens": tokens, "alive": tokens if not batch else rng.randint(0, tokens), "batch": batch, "dim": dim,
                "rms": rng.random() < 0.4, "dtype": dtype, "to": rng.choice(("bf16", dtype)), "backward": backward}
    kind = rng.choice(("fork", "free", "compact"))
    page, sources = rng.choice((16, 32, 64, 128)), _log(rng, 1, 64)
    batch = sources * rng.randint(1, 8)
    kv_heads, dim = rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 256))
    context = _log(rng, 1, min(8192, 600 * 2 ** 20 // (kv_heads * dim * (sources + batch)) + 1))
    return {"op": op, "kind": kind, "rows": batch + sources + rng.randint(0, 300), "batch": batch, "sources": sources, "alive": rng.randint(0, batch),
            "context": context, "page": page, "kv_heads": kv_heads, "dim": dim}


# ------------------------------------------------------------------------------------------------------------ inputs

def _survivors(case, gen, dev):
    """Rows of the batch in ascending order, as a cascade step lists them, and how many of them are real."""
    if not case["batch"]:
        return None, None
    rows = torch.randperm(case["batch"], generator=gen, device=dev)[:case["tokens"]].sort().values.to(torch.int32)
    return rows, torch.tensor([case["alive"]], dtype=torch.int32, device=dev)


def _linear(case, gen, dev):
    t, k, n = case["tokens"], case["in"], case["out"]
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev)
    rows, count = _survivors(case, gen, dev)
    st = {"x": rand(t, k).to(torch.bfloat16), "weight": (rand(n, k) * k ** -0.5).to(torch.bfloat16),
          "bias": 0.5 * rand(n) if case["bias"] else None, "rows": rows, "count": count,
          "stream": rand(case["batch"] or t, n).to(_DTYPE[case["dtype"]]) if case["residual"] else None}
    if case["batch"]:
        st["out"] = st["stream"].clone()                   # where the rows of the sums go; the others stay
    if case["backward"]:
        st["dy"] = rand(t, n).to(torch.bfloat16)
        # what the forward pass leaves for the gradient: the product before the activation, which is about normal
        st["preact"] = rand(t, n).to(torch.bfloat16) if case["act"] != "none" else None
    return st


def _norm(case, gen, dev):
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev)
    d = case["dim"]
    rows, count = _survivors(case, gen, dev)
    # a residual stream: every value has its own size and offset
    x = (rand(case["batch"] or case["tokens"], d) * (1 + rand(d).abs()) + 0.5 * rand(d)).to(_DTYPE[case["dtype"]])
    st = {"x": x, "weight": 1 + 0.1 * rand(d), "bias": None if case["rms"] else 0.1 * rand(d), "rows": rows, "count": count}
    if case["backward"]:
        st["dy"] = rand(case["tokens"], d).to(_DTYPE[case["to"]])
    if case["batch"]:
        st["out"] = torch.zeros(case["tokens"], d, dtype=_DTYPE[case["to"]], device=dev)   # rows past the count are left alone
    return st


def _num_pages(case):
    """Room for the prompts and the tails of their continuations, and some more; for a fork now and then too little."""
    prompts = case["sources"] * -(-case["context"] // case["page"])
    return prompts + prompts // 4 + 8 + (0 if case["kind"] == "fork" else case["batch"])


def _pages(case, gen, dev):
    """Prompts in the first `sources` rows.  For a fork `batch` other rows are empty; elsewhere these are continuations of them,
    which share their full pages, and `batch` of all these rows end."""
    rows, batch, sources, page = case["rows"], case["batch"], case["sources"], case["page"]
    blocks = -(-case["context"] // page) + 1
    order = torch.randperm(rows, generator=gen, device=dev)
    src, dst = order[:sources], order[sources:sources + batch]
    parent = torch.arange(batch, device=dev) % sources
    length = torch.randint((case["context"] + 1) // 2, case["context"] + 1, (sources,), generator=gen, device=dev)
    full, used = length // page, (length + page - 1) // page
    start = used.cumsum(0) - used
    first = int(used.sum())                                           # pages of the prompts, then of the continuations' tails
    num_pages = _num_pages(case)
    name = torch.randperm(num_pages, generator=gen, device=dev)
    col = torch.arange(blocks, device=dev)
    table = torch.full((rows, blocks), -1, dtype=torch.int64, device=dev)
    lens = torch.zeros(rows, dtype=torch.int64, device=dev)
    table[src] = torch.where(col < used[:, None], name[(start[:, None] + col).clamp(max=num_pages - 1)], -1)
    lens[src] = length
    shared = torch.zeros(num_pages, dtype=torch.int32, device=dev)
    taken = first
    st = {"src": src[parent].to(torch.int32), "dst": dst.to(torch.int32)}
    if case["kind"] != "fork":
        tails = torch.arange(first, first + batch, device=dev)
        here = torch.where(col < full[parent][:, None], table[src[parent]], -1)
        here[torch.arange(batch, device=dev), full[parent]] = name[tails]
        table[dst], lens[dst] = here, full[parent] * page + torch.randint(1, page + 1, (batch,), generator=gen, device=dev)
        shared.scatter_add_(0, here.clamp(min=0).flatten(), ((col < full[parent][:, None]) & (here >= 0)).flatten().int())
        taken += batch
        both = torch.cat([src, dst])
        st["ended"] = both[torch.randperm(both.numel(), generator=gen, device=dev)[:batch]].to(torch.int32)
    free = torch.full((num_pages,), -1, dtype=torch.int32, device=dev)
    free[:num_pages - taken] = name[taken:].to(torch.int32)
    st.update({"lens": lens.to(torch.int32), "table": table.to(torch.int32), "shared": shared, "free": free,
               "free_count": torch.tensor([num_pages - taken], dtype=torch.int32, device=dev),
               "alive": torch.tensor([case["alive"]], dtype=torch.int32, device=dev)})
    if case["kind"] != "free":
        for n in ("k", "v"):
            st[n + "_codes"] = torch.randint(0, 256, (num_pages, case["kv_heads"], page, case["dim"] // 2), generator=gen, device=dev, dtype=torch.uint8)
            st[n + "_meta"] = torch.randn(num_pages, case["kv_heads"], page, 2, generator=gen, device=dev).to(torch.bfloat16)
    return st


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    st = {"linear": _linear, "norm": _norm, "pages": _pages}[case["op"]](case, gen, dev)
    st["case"] = case
    if own:                                                # the handles of the layer's cache, which a program keeps
        from paper_2002_02645_b200 import binding as fb
        st["fb"] = fb
        if case["op"] == "pages":
            st["tables"] = fb.KvTables(page_size=case["page"], max_blocks=st["table"].shape[1], max_batch=case["batch"])
            if case["kind"] != "free":
                st["kv"] = fb.KvCache(st["k_codes"], st["k_meta"], st["v_codes"], st["v_meta"], q_heads=case["kv_heads"])
    return st


# ------------------------------------------------------------------------------------------------------- plain forms

def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":
        return z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        c = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(c * (z + 0.044715 * z ** 3))
        return s + z * s * (1 - s) * c * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _linear_plain(st):
    case = st["case"]
    x, w = st["x"].float(), st["weight"].float()
    if case["backward"]:
        dz = st["dy"].float()
        if case["act"] != "none":
            dz = dz * _act_slope(st["preact"].float(), case["act"])
        return {"dx": (dz @ w).to(torch.bfloat16), "dweight": (dz.t() @ x).to(torch.bfloat16), "dbias": dz.sum(0) if case["bias"] else None}
    z = x @ w.t()
    if case["bias"]:
        z = z + st["bias"]
    y, dtype = _act(z, case["act"]), _DTYPE[case["dtype"]]
    if not case["batch"]:
        return {"y": (y + st["stream"].float() if case["residual"] else y).to(dtype)}
    rows, out = st["rows"].long(), st["out"]
    real = (torch.arange(case["tokens"], device=rows.device) < st["count"])[:, None]
    out[rows] = torch.where(real, (st["stream"][rows].float() + y).to(dtype), out[rows])
    return {"y": out}


def _norm_plain(st):
    case = st["case"]
    x, d = st["x"], case["dim"]
    if case["batch"]:
        x = x[st["rows"].long()]
    x = x.float()
    mean = 0 if case["rms"] else x.mean(-1, keepdim=True)
    c = x - mean
    r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
    n = c * r
    if not case["backward"]:
        y = n * st["weight"]
        if st["bias"] is not None:
            y = y + st["bias"]
        y = y.to(_DTYPE[case["to"]])
        if case["batch"]:
            y = torch.where((torch.arange(case["tokens"], device=y.device) < st["count"])[:, None], y, st["out"])
        return {"y": y}
    dy = st["dy"].float()
    g = dy * st["weight"]
    dx = g - n * (g * n).mean(-1, keepdim=True)
    if not case["rms"]:
        dx = dx - g.mean(-1, keepdim=True)
    return {"dx": (dx * r).to(st["x"].dtype), "dweight": (dy * n).sum(0), "dbias": None if case["rms"] else dy.sum(0)}


def _fork_plain(st):
    case = st["case"]
    page, lens, table, free, count = case["page"], st["lens"], st["table"].clone(), st["free"], st["free_count"]
    src, dst, dev = st["src"].long(), st["dst"].long(), st["lens"].device
    real = torch.arange(case["batch"], device=dev) < st["alive"]
    length = lens[src]
    full, tail = length // page, length % page
    ok = real & (lens[dst] == 0) & (src != dst)
    need = (ok & (tail > 0)).int()
    cum = need.cumsum(0)
    granted = ok & ((need == 0) | (cum <= count))
    new = torch.where(granted & (need > 0), free[(count - cum).clamp(min=0).long()], -1)
    col = torch.arange(table.shape[1], device=dev)
    common = granted[:, None] & (col < full[:, None])
    theirs = table[src]
    here = torch.where(common, theirs, table[dst])
    at = full.long()[:, None]
    last = theirs.gather(1, at)
    here.scatter_(1, at, torch.where(new >= 0, new, here.gather(1, at)[:, 0])[:, None].int())
    table[dst] = here
    shared = st["shared"].clone()
    shared.scatter_add_(0, theirs.clamp(min=0).long().flatten(), common.int().flatten())
    copied = new >= 0
    copies = torch.stack([torch.where(copied, last[:, 0], -1), new, torch.where(copied, tail, 0)], 1).int()
    lens_out = lens.clone()
    lens_out[dst] = torch.where(granted, length, lens[dst])
    taken = (need * granted.int()).sum().int()
    # (where nothing is copied the prompt's first page, which is no target, stands for source and target)
    fill = (copied[:, None] & (torch.arange(page, device=dev) < tail[:, None]))[:, None, :, None]
    source, target = torch.where(copied, last[:, 0], theirs[:, 0]).long(), torch.where(copied, new, theirs[:, 0]).long()
    return {"granted": granted.int(), "lens": lens_out, "free_count": count - taken, "table": table, "shared": shared, "copies": copies,
            **_copy_plain(st, source, target, fill)}


def _copy_plain(st, source, target, fill):
    """Copies what `fill` marks of the pages `source` to the pages `target`; pages not marked are written as they are."""
    out = {}
    for n in ("k_codes", "k_meta", "v_codes", "v_meta"):
        pool = st[n]
        flat = pool.view(torch.int16) if pool.dtype == torch.bfloat16 else pool
        flat[target] = torch.where(fill, flat[source], flat[target])
        out[n] = pool
    return out


def _free_plain(st, lens, table, free, count, shared):
    """The rows that ended give up their pages; those without another owner go to the free pages, by their numbers."""
    case = st["case"]
    page, rows, dev = case["page"], st["ended"].long(), lens.device
    num_pages, blocks = free.numel(), table.shape[1]
    real = torch.arange(case["batch"], device=dev) < st["alive"]
    used = torch.where(real, (lens[rows] + page - 1) // page, 0)
    mine = torch.arange(blocks, device=dev) < used[:, None]
    shared = shared.clone()
    shared.scatter_add_(0, torch.where(mine, table[rows], 0).long().flatten(), -mine.int().flatten())
    gone = shared < 0
    place = count + gone.cumsum(0) - 1
    longer = torch.cat([free, free[:1]])                              # one place more, for what is not written
    longer[torch.where(gone, place, num_pages).long()] = torch.arange(num_pages, device=dev, dtype=torch.int32)
    lens = lens.clone()
    lens[torch.where(real, rows, rows[0])] = 0 if case["alive"] else lens[rows[0]]
    return lens, longer[:-1], (count + gone.sum()).int(), shared.clamp(min=0)


def _compact_plain(st, lens, table, free, count, shared):
    """Used pages above the number of used pages move to the free places below it, in order."""
    page, dev = st["case"]["page"], lens.device
    num_pages, blocks = free.numel(), table.shape[1]
    name = torch.arange(num_pages, device=dev, dtype=torch.int32)
    is_free = torch.zeros(num_pages + 1, dtype=torch.bool, device=dev)
    is_free[torch.where(name < count, free, num_pages).long()] = True
    is_free = is_free[:-1]
    used = num_pages - count
    high, hole = ~is_free & (name >= used), is_free & (name < used)
    rank = torch.where(high, high.cumsum(0) - 1, num_pages)
    hole_at = torch.full((num_pages + 1,), -1, dtype=torch.int32, device=dev)
    hole_at[torch.where(hole, hole.cumsum(0) - 1, num_pages)] = name
    to = torch.where(high, hole_at[rank], name)
    most = num_pages // 2
    copies = torch.full((most + 1, 3), -1, dtype=torch.int32, device=dev)
    copies[:, 2] = 0
    copies[torch.where(high, rank, most)] = torch.stack([name, to, torch.full_like(name, page)], 1)   # (the last one is nobody's)
    copies = copies[:-1]
    mine = torch.arange(blocks, device=dev) < ((lens + page - 1) // page)[:, None]
    table = torch.where(mine, to[table.clamp(min=0).long()], table)
    moved = torch.zeros_like(shared)
    moved.scatter_add_(0, to.long(), torch.where(is_free, 0, shared))
    free = torch.where(name < count, num_pages - 1 - name, free)
    return table, free, moved, copies, high.sum().int().view(1)


def _pages_plain(st):
    case = st["case"]
    if case["kind"] == "fork":
        return _fork_plain(st)
    lens, free, count, shared = _free_plain(st, st["lens"], st["table"], st["free"], st["free_count"], st["shared"])
    out = {"lens": lens, "free_count": count}
    if case["kind"] == "free":
        return {**out, "free": free, "shared": shared}
    table, free, shared, copies, moves = _compact_plain(st, lens, st["table"], free, count, shared)
    valid = torch.arange(copies.shape[0], device=lens.device) < moves
    # (a page that is no target of a copy stands for those that there are not)
    source, target = copies[:, 0].clamp(min=0).long(), torch.where(valid, copies[:, 1], free.numel() - 1).long()
    return {**out, "table": table, "free": free, "shared": shared, "copies": copies, "moves": moves,
            **_copy_plain(st, source, target, valid[:, None, None, None])}


# -------------------------------------------------------------------------------------------------------------- runs

def _linear_own(st):
    case, fb = st["case"], st["fb"]
    if case["backward"]:
        dx, dw, db = fb.linear_backward(st["x"], st["weight"], st["dy"], preact=st["preact"], activation=case["act"], with_bias=case["bias"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if not case["batch"]:
        return {"y": fb.linear(st["x"], st["weight"], st["bias"], activation=case["act"], residual=st["stream"], out_dtype=_DTYPE[case["dtype"]])}
    return {"y": fb.linear(st["x"], st["weight"], st["bias"], activation=case["act"], residual=st["stream"], out=st["out"], rows=st["rows"],
                           count=st["count"])}


def _norm_own(st):
    case, fb = st["case"], st["fb"]
    if case["backward"]:
        dx, dw, db = fb.layer_norm_backward(st["x"], st["weight"], st["dy"], eps=EPS, rms=case["rms"], with_bias=not case["rms"])
        return {"dx": dx, "dweight": dw, "dbias": db}
    if not case["batch"]:
        return {"y": fb.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS, rms=case["rms"], out_dtype=_DTYPE[case["to"]])}
    return {"y": fb.layer_norm(st["x"], st["weight"], st["bias"], eps=EPS, rms=case["rms"], rows=st["rows"], count=st["count"], out=st["out"])}


def _pages_own(st):
    case, tables = st["case"], st["tables"]
    shared, table = st["shared"].clone(), st["table"]      # counted in place
    if case["kind"] == "fork":
        out = tables.fork(st["src"], st["dst"], st["lens"], st["free"], st["free_count"], table, shared, batch_count=st["alive"])
        st["kv"].copy_pages(out.copies)
        return {"granted": out.granted, "lens": out.lens, "free_count": out.free_count, "table": table, "shared": shared, "copies": out.copies,
                **{n: st[n] for n in ("k_codes", "k_meta", "v_codes", "v_meta")}}
    free = st["free"]
    if case["kind"] == "compact":
        table, free = table.clone(), free.clone()          # so that the state can be used again
    lens, count = tables.free(st["ended"], st["lens"], free, st["free_count"], table, shared, batch_count=st["alive"])
    if case["kind"] == "free":
        return {"lens": lens, "free_count": count, "free": free, "shared": shared}
    copies, moves = tables.compact(lens, free, count, table, shared)
    st["kv"].copy_pages(copies, count=moves)
    return {"lens": lens, "free_count": count, "table": table, "free": free, "shared": shared, "copies": copies, "moves": moves,
            **{n: st[n] for n in ("k_codes", "k_meta", "v_codes", "v_meta")}}


def run(state):
    ops = {"linear": (_linear_plain, _linear_own), "norm": (_norm_plain, _norm_own), "pages": (_pages_plain, _pages_own)}
    return ops[state["case"]["op"]][1 if own else 0](state)


# -------------------------------------------------------------------------------------------------------------- work

def work(case):
    """Bytes and operations of one pass: each input once, each output once (expected values where lengths are drawn)."""
    op, t = case["op"], case["alive"]
    size = 2 if case.get("dtype") == "bf16" else 4
    if op == "linear":
        k, n = case["in"], case["out"]
        if case["backward"]:
            values = t * k * 2 + n * k * 2 + t * n * (1 if case["act"] == "none" else 2)
            return {"bytes": 2 * values + 4 * n * case["bias"], "flops": 4 * t * k * n}
        stream = size * n * (t * (2 if case["residual"] else 1))
        return {"bytes": 2 * (t * k + n * k) + stream + 4 * n * case["bias"] + (4 * t if case["batch"] else 0), "flops": 2 * t * k * n}
    if op == "norm":
        to, values = 2 if case["to"] == "bf16" else 4, t * case["dim"]
        if case["backward"]:
            return {"bytes": values * (2 * size + to) + 12 * case["dim"], "flops": 14 * values}
        return {"bytes": values * (size + to) + 8 * case["dim"] + (4 * t if case["batch"] else 0), "flops": 7 * values}
    page, batch, blocks, num_pages = case["page"], case["batch"], 0.75 * case["context"] / case["page"], _num_pages(case)
    token = 2 * case["kv_heads"] * (case["dim"] / 2 + 4)   # bytes of a token in the pools
    if case["kind"] == "fork":                             # entries read, written and counted; a tail copied for each
        return {"bytes": t * (blocks * 8 + 32) + 4 * num_pages + t * token * min(page, case["context"]), "flops": 0}
    ended = 4 * t * blocks + 16 * batch + 8 * num_pages
    if case["kind"] == "free":
        return {"bytes": ended, "flops": 0}
    # pages lie at random: of the used ones as large a share is above their number as there are free ones
    used = min(num_pages, case["sources"] * (blocks + 0.5) + batch)
    moves = used * (num_pages - used) / num_pages
    return {"bytes": ended + 8 * case["rows"] * blocks + 24 * num_pages + 2 * moves * page * token, "flops": 0}


# ------------------------------------------------------------------------------------------------------------- exact

def _slope_exact(z, act):
    """Slope of the activation at z, by its own derivation."""
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return torch.heaviside(z, torch.zeros_like(z))
    if act == "gelu":
        return (1 + torch.erf(z / 2 ** 0.5)) / 2 + z * torch.exp(-z ** 2 / 2) / (2 * math.pi) ** 0.5
    if act == "gelu_tanh":
        inner = (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)
        return (1 + torch.tanh(inner)) / 2 + z / 2 / torch.cosh(inner) ** 2 * (2 / math.pi) ** 0.5 * (1 + 0.134145 * z ** 2)
    e = torch.exp(-z)
    return (1 + e + z * e) / (1 + e) ** 2


def _value_exact(z, act):
    if act == "relu":
        return torch.maximum(z, torch.zeros_like(z))
    if act == "gelu":
        return z * (1 + torch.erf(z / 2 ** 0.5)) / 2
    if act == "gelu_tanh":
        return z / 2 * (1 + torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _linear_exact(st):
    case = st["case"]
    x, w = st["x"].double(), st["weight"].double()
    if case["backward"]:
        dz = st["dy"].double()
        if st["preact"] is not None:
            dz = dz * _slope_exact(st["preact"].double(), case["act"])
        return {"dx": torch.einsum("tn,nk->tk", dz, w), "dweight": torch.einsum("tn,tk->nk", dz, x),
                "dbias": torch.einsum("tn->n", dz) if case["bias"] else None}
    z = torch.einsum("tk,nk->tn", x, w)
    if case["bias"]:
        z += st["bias"].double()
    y = _value_exact(z, case["act"])
    if not case["batch"]:
        return {"y": y + st["stream"].double() if case["residual"] else y}
    out, n = st["stream"].double(), case["alive"]
    out[st["rows"][:n].long()] += y[:n]
    return {"y": out}


def _norm_exact(st):
    case, n = st["case"], st["case"]["alive"]
    x, w = st["x"].double(), st["weight"].double()
    if case["batch"]:
        y = torch.zeros(case["tokens"], case["dim"], dtype=torch.float64, device=x.device)
        x = x[st["rows"][:n].long()]
    if not case["rms"]:
        x = x - x.sum(-1, keepdim=True) / case["dim"]
    s = (torch.einsum("td,td->t", x, x) / case["dim"] + EPS).sqrt()[:, None]
    if not case["backward"]:
        z = w * x / s + (0 if st["bias"] is None else st["bias"].double())
        if not case["batch"]:
            return {"y": z}
        y[:n] = z
        return {"y": y}
    dy = st["dy"].double()
    g = dy * w
    dx = g / s - x * torch.einsum("td,td->t", g, x)[:, None] / (case["dim"] * s ** 3)
    if not case["rms"]:
        dx = dx - dx.mean(-1, keepdim=True)                # (the deviations of a row add up to zero)
    return {"dx": dx, "dweight": torch.einsum("td,td->d", dy, x / s), "dbias": None if case["rms"] else torch.einsum("td->d", dy)}


def exact(case, seed):
    if case["op"] == "pages":
        return None
    st = prepare(case, seed)
    return {"linear": _linear_exact, "norm": _norm_exact}[case["op"]](st)
