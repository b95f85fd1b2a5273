"""Page tables, norm with rotation, the 4-bit key/value store and attention over it, against plain 64-bit implementations.

Tolerances follow from the roundings the operators state (u = 2^-24 for float32; rounding to bfloat16, with its 8 significant bits, is off by up to 2^-8 of the value):
 - tables, codes, scales and offsets are whole numbers or exact roundings: compared for equality
 - norm: a few dozen float32 operations on values of size 1: 32 u relative to the largest factor, plus the final rounding
 - attention: weights go into the product as halves (2^-11 relative each; a pair of halves for float32 queries), exponents are
   off by some u times the size of the scores, the sums are float32
"""
import math

import numpy as np
import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device=DEV)


# ---------------------------------------------------------------------------------------------------------------- tables

class PlainTables:
    """The rules of fi_pages_extend / fi_pages_release on Python lists, one request after another."""

    def __init__(self, page, blocks, lens, table, free):
        self.page, self.blocks = page, blocks
        self.lens, self.table, self.free = list(lens), [list(r) for r in table], list(free)

    def extend(self, rows, new, max_tokens):
        slots, positions, cu, granted = [], [], [0], []
        wanted, start = 0, len(self.free)
        for row, n in zip(rows, new):
            have = self.lens[row]
            had, want = -(-have // self.page), -(-(have + n) // self.page)
            cu.append(cu[-1] + n)
            fits = want <= self.blocks and cu[-1] <= max_tokens
            need = want - had if fits else 0
            ok = fits and (need == 0 or wanted + need <= start)
            if ok:
                for b in range(had, want):
                    self.table[row][b] = self.free[start - 1 - wanted - (b - had)]
            for j in range(n):
                p = have + j
                positions.append(p)
                slots.append(self.table[row][p // self.page] * self.page + p % self.page if ok else -1)
            if ok:
                self.lens[row] = have + n
            wanted += need
            granted.append(n if ok else 0)
        self._taken(rows, granted)
        pad = max_tokens - len(slots)
        return ((slots + [-1] * pad)[:max_tokens], (positions + [-1] * pad)[:max_tokens], cu, granted)

    def _taken(self, rows, granted):
        n = 0
        for row, g in zip(rows, granted):
            n += -(-self.lens[row] // self.page) - -(-(self.lens[row] - g) // self.page)
        self.count = len(self.free) - n

    def release(self, rows):
        for row in rows:
            self.free += [self.table[row][b] for b in range(-(-self.lens[row] // self.page))]
            self.lens[row] = 0


def make_tables(rng, rows, page, blocks, top, spare):
    lens = rng.integers(0, top + 1, rows)
    used = [-(-int(x) // page) for x in lens]
    pages = rng.permutation(sum(used) + spare)
    table, at = [], 0
    for u in used:
        table.append(list(pages[at:at + u]) + [-1] * (blocks - u))
        at += u
    return lens.tolist(), [[int(x) for x in r] for r in table], [int(x) for x in pages[at:]]


@pytest.mark.parametrize("rows,batch,count,page,blocks,new_top,spare,max_tokens", [
    (1, 1, None, 16, 4, None, 3, None),            # one request, one token
    (40, 17, 13, 16, 9, None, 40, None),           # decode step of survivors
    (40, 17, 0, 16, 9, None, 40, None),            # nobody is left
    (300, 300, None, 32, 6, 70, 2000, 300 * 70),   # ragged new tokens, none among them
    (300, 257, 250, 32, 6, 70, 120, 257 * 70),     # too few pages: some are refused, later ones may still fit
    (50, 50, None, 16, 5, 100, 400, 50 * 100),     # block table too short for some
    (50, 50, None, 16, 9, 60, 400, 700),           # more tokens than the outputs hold
    (3000, 2049, 2048, 64, 8, 9, 9000, 2049 * 9),  # several requests per thread, several CTAs
])
@pytest.mark.parametrize("in_place", [False, True])
def test_extend_matches_one_request_after_another(rows, batch, count, page, blocks, new_top, spare, max_tokens, in_place):
    rng = np.random.default_rng(rows + batch + page)
    lens, table, free = make_tables(rng, rows, page, blocks, (blocks - 1) * page, spare)
    row_idx = np.sort(rng.permutation(rows)[:batch])
    new = [1] * batch if new_top is None else rng.integers(0, new_top + 1, batch).tolist()
    n = batch if count is None else count
    max_tokens = batch if max_tokens is None else max_tokens
    ref = PlainTables(page, blocks, lens, table, free)
    slots, positions, cu, granted = ref.extend(row_idx[:n].tolist(), new[:n], max_tokens)

    kv = fb.KvTables(page_size=page, max_blocks=blocks, max_batch=batch)
    pages = torch.full((spare + 500,), -7, dtype=torch.int32, device=DEV)
    pages[:spare] = ints(free)
    d_lens, d_table, d_count = ints(lens), ints(table), ints([spare])
    out = fb.ExtendOut(batch, max_tokens, rows, DEV)
    if in_place:
        out.lens, out.free_count = d_lens, d_count
    for _ in range(1 if in_place else 2):          # out of place the step can be repeated
        kv.extend(d_lens, pages, d_count, d_table, new_lens=None if new_top is None else ints(new), row_idx=ints(row_idx),
                  batch_count=None if count is None else ints([count]), max_tokens=max_tokens, out=out)
    assert out.slot_map.tolist() == slots and out.positions.tolist() == positions
    assert out.cu_tokens.tolist() == cu + [cu[-1]] * (batch - n)
    assert out.granted.tolist() == granted + [0] * (batch - n)
    assert out.lens.tolist() == ref.lens and out.free_count.item() == ref.count
    assert d_table.tolist() == ref.table
    kv.close()


@pytest.mark.parametrize("rows,batch,count,blocks", [(5, 1, None, 3), (200, 64, 50, 7), (3000, 2500, None, 40)])
@pytest.mark.parametrize("in_place", [False, True])
def test_release_then_extend(rows, batch, count, blocks, in_place):
    page = 16
    rng = np.random.default_rng(rows)
    lens, table, free = make_tables(rng, rows, page, blocks, blocks * page - 1, 5)
    ended = rng.permutation(rows)[:batch].tolist()
    n = batch if count is None else count
    ref = PlainTables(page, blocks, lens, table, free)
    ref.release(ended[:n])
    total = sum(-(-x // page) for x in lens) + 5
    pages = torch.full((total,), -7, dtype=torch.int32, device=DEV)
    pages[:5] = ints(free)
    kv = fb.KvTables(page_size=page, max_blocks=blocks, max_batch=max(batch, rows))
    d_lens, d_count, d_table = ints(lens), ints([5]), ints(table)
    lens1, count1 = kv.release(ints(ended), d_lens, pages, d_count, d_table, batch_count=None if count is None else ints([count]),
                               out=(d_lens, d_count) if in_place else None)
    assert lens1.tolist() == ref.lens and count1.item() == len(ref.free)
    assert pages[:len(ref.free)].tolist() == ref.free and (pages[len(ref.free):] == -7).all()
    out = kv.extend(lens1, pages, count1, d_table)            # one token for every row
    slots, positions, cu, granted = ref.extend(list(range(rows)), [1] * rows, rows)
    assert out.slot_map.tolist() == slots and out.lens.tolist() == ref.lens and out.free_count.item() == ref.count
    assert out.granted.tolist() == granted and out.cu_tokens.tolist() == cu and out.positions.tolist() == positions


def test_rows_that_do_not_exist_get_no_tokens():
    kv = fb.KvTables(page_size=16, max_blocks=2, max_batch=8)
    table = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    out = kv.extend(ints([0, -5]), ints([3, 4]), ints([2]), table, row_idx=ints([7, 0, -1, 1]), new_lens=ints([4, 2, 1, 3]), max_tokens=10)
    assert out.cu_tokens.tolist() == [0, 0, 2, 2, 2] and out.granted.tolist() == [0, 2, 0, 0]
    assert out.slot_map.tolist() == [64, 65] + [-1] * 8 and out.lens.tolist()[0] == 2 and table.tolist() == [[4, -1], [-1, -1]]


# ------------------------------------------------------------------------------------------------------------------ norm

def rope_table(max_pos, rot):
    i = torch.arange(rot // 2, dtype=torch.float64)
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-2.0 * i / max(rot, 1))
    return torch.cat([a.cos(), a.sin()], 1).float().to(DEV)


def norm_formula(x, w, rope, pos, eps, interleaved):
    """In 64 bits, differentiable."""
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    if w is not None:
        y = y * w
    if rope is None:
        return y
    half = rope.shape[1] // 2
    c, s = rope[pos.long()].double()[:, None].split(half, -1)
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if interleaved else (y[..., :half], y[..., half:2 * half])
    ra, rb = a * c - b * s, a * s + b * c
    turned = torch.stack([ra, rb], -1).flatten(-2) if interleaved else torch.cat([ra, rb], -1)
    return torch.cat([turned, y[..., 2 * half:]], -1)


NORM_CASES = [  # tokens, q heads, k heads, dim, rot, interleaved, weights, fused strides
    (1, 1, 0, 16, 16, False, True, False), (1, 8, 2, 128, 128, False, True, True), (37, 5, 1, 64, 32, False, True, True),
    (3, 3, 3, 80, 48, True, True, True), (129, 4, 2, 256, 256, True, True, False), (65, 7, 1, 112, 112, False, False, True),
    (40, 2, 2, 192, 64, False, True, True), (9, 2, 1, 32, 0, False, True, False), (700, 20, 4, 128, 64, True, True, True),
]


def norm_inputs(case, dtype, seed):
    tokens, hq, hk, d, rot, inter, weights, fused = case
    gen = torch.Generator(device=DEV).manual_seed(seed)
    make = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(dtype)
    if fused:
        qkv = make(tokens, hq + 2 * hk, d)
        q, k = qkv[:, :hq], qkv[:, hq:hq + hk] if hk else None
    else:
        q, k = make(hq, tokens, d).transpose(0, 1), make(tokens, hk, d) if hk else None   # heads outermost
    wq = 1 + 0.3 * torch.randn(d, generator=gen, device=DEV) if weights else None
    wk = 1 + 0.3 * torch.randn(d, generator=gen, device=DEV) if weights else None
    rope = rope_table(5000, rot) if rot else None
    pos = torch.randint(0, 5000, (tokens,), generator=gen, device=DEV, dtype=torch.int32) if rot else None
    return q, k, wq, wk, rope, pos, gen


def rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24


@pytest.mark.parametrize("case", NORM_CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_rope_matches_formula(case, dtype):
    q, k, wq, wk, rope, pos, _ = norm_inputs(case, dtype, 3)
    got = fb.head_norm_rope(q, k, wq, wk, rope, pos, eps=1e-5, interleaved=case[5])
    for g, x, w in ((got[0], q, wq), (got[1], k, wk)):
        if x is None:
            assert g is None
            continue
        want = norm_formula(x.double(), None if w is None else w.double(), rope, pos, 1e-5, case[5])
        size = want.abs().amax(-1, keepdim=True)     # a rotated pair is as exact as its larger member
        assert ((g.double() - want).abs() <= rounding(dtype) * want.abs() + 32 * 2.0 ** -24 * size).all()
    if not case[7]:
        return
    q2, k2 = q.clone(), None if k is None else k.clone()      # in place
    fb.head_norm_rope(q2, k2, wq, wk, rope, pos, eps=1e-5, interleaved=case[5], q_out=q2, k_out=k2)
    assert torch.equal(q2, got[0]) and (k is None or torch.equal(k2, got[1]))


@pytest.mark.parametrize("case", NORM_CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_rope_gradients_match_formula(case, dtype):
    q, k, wq, wk, rope, pos, gen = norm_inputs(case, dtype, 4)
    dq_out = torch.randn(q.shape, generator=gen, device=DEV).to(dtype)
    dk_out = None if k is None else torch.randn(k.shape, generator=gen, device=DEV).to(dtype)
    args = (q, k, wq, wk, rope, pos, dq_out, dk_out)
    got = fb.head_norm_rope_backward(*args, eps=1e-5, interleaved=case[5])
    again = fb.head_norm_rope_backward(*args, eps=1e-5, interleaved=case[5])
    for a, b in zip(got, again):
        assert (a is None and b is None) or torch.equal(a, b)           # sums in a fixed order
    for x, w, dy, dx, dw in ((q, wq, dq_out, got[0], got[2]), (k, wk, dk_out, got[1], got[3])):
        if x is None:
            assert dx is None and dw is None
            continue
        x64 = x.double().detach().requires_grad_()
        w64 = None if w is None else w.double().detach().requires_grad_()
        norm_formula(x64, w64, rope, pos, 1e-5, case[5]).backward(dy.double())
        size = x64.grad.abs().amax(-1, keepdim=True)
        assert ((dx.double() - x64.grad).abs() <= rounding(dtype) * x64.grad.abs() + 64 * 2.0 ** -24 * size).all()
        if w is None:
            assert dw is None
            continue
        n = x.double() / (x.double().square().mean(-1, keepdim=True) + 1e-5).sqrt()
        # every product is off by some u of its own size (a rotated gradient: of its pair's), the sum by some u of the partial sums
        terms = (dy.double().abs().amax(-1, keepdim=True) * 2 * n.abs()).sum((0, 1))
        assert ((dw.double() - w64.grad).abs() <= 16 * 2.0 ** -24 * terms).all()


def test_norm_rope_gradient_against_differences():
    """Directional derivative of the kernel's own forward pass (float32) against its backward pass.  Central differences with
    step h = 2^-7: truncation h^2 / 6 times a third derivative of order 10, and rounding 2^-24 * sqrt(outputs) / h: together
    below 2 % of a derivative of order sqrt(outputs)."""
    case = (6, 3, 2, 64, 32, True, True, False)
    q, k, wq, wk, rope, pos, gen = norm_inputs(case, torch.float32, 5)
    r = lambda t: torch.randn(t.shape, generator=gen, device=DEV)
    aq, ak, h = r(q), r(k), 2.0 ** -7
    dq, dk, dwq, dwk = fb.head_norm_rope_backward(q, k, wq, wk, rope, pos, aq, ak, interleaved=True)

    def value(q, k, wq, wk):
        yq, yk = fb.head_norm_rope(q.contiguous(), k.contiguous(), wq, wk, rope, pos, interleaved=True)
        return ((yq.double() * aq).sum() + (yk.double() * ak).sum()).item()

    base = (q, k, wq, wk)
    for i, grad in enumerate((dq, dk, dwq, dwk)):
        d = r(base[i])
        plus, minus = [list(base) for _ in range(2)]
        plus[i], minus[i] = base[i] + h * d, base[i] - h * d
        slope = (value(*plus) - value(*minus)) / (2 * h)
        assert abs(slope - (grad.double() * d).sum().item()) <= 0.02 * math.sqrt(aq.numel())


def test_norm_rope_counts_and_positions_out_of_range():
    q = torch.randn(6, 2, 32, device=DEV)
    rope = rope_table(10, 32)
    pos = ints([0, 9, 10, -1, 3, 4])
    out = torch.full_like(q, 5.0)
    fb.head_norm_rope(q, None, None, None, rope, pos, count=ints([5]), q_out=out)
    assert out[2:4].isnan().all() and out[[0, 1, 4]].isfinite().all() and (out[5] == 5).all()
    g = fb.head_norm_rope_backward(q, None, torch.ones(32, device=DEV), None, rope, pos, q, None, count=ints([0]), dq=out)
    assert (g[2] == 0).all() and (out[5] == 5).all()


# ---------------------------------------------------------------------------------------------------------- 4-bit append

def bf16_step_down(x):
    """Largest bf16 number <= x, on numpy float64."""
    with np.errstate(divide="ignore"):
        e = np.where(x == 0, 0.0, np.floor(np.log2(np.abs(np.where(x == 0, 1.0, x)))))
    step = 2.0 ** (np.maximum(e, -126) - 7)
    return np.floor(x / step) * step


def plain_pack(x):
    """(codes, scale, offset, value) of vectors along the last axis, in numpy: float32 where the format says float32."""
    x = x.astype(np.float32)
    offset = bf16_step_down(x.min(-1, keepdims=True).astype(np.float64)).astype(np.float32)
    quotient = ((x.max(-1, keepdims=True) - offset).astype(np.float32) / np.float32(15)).astype(np.float64)
    scale = np.maximum(-bf16_step_down(-quotient), 2.0 ** -40).astype(np.float32)
    code = np.clip(np.rint((x - offset) / scale), 0, 15)
    return code.astype(np.uint8), scale, offset, code.astype(np.float64) * scale + offset


def pools(pages, heads, page, dim, order="head", fill=0):
    """Codes and meta with the given memory order; `order` token: tokens outside of heads."""
    if order == "head":
        return (torch.full((pages, heads, page, dim // 2), fill, dtype=torch.uint8, device=DEV),
                torch.zeros(pages, heads, page, 2, dtype=torch.bfloat16, device=DEV))
    return (torch.full((pages, page, heads, dim // 2), fill, dtype=torch.uint8, device=DEV).transpose(1, 2),
            torch.zeros(pages, page, heads, 2, dtype=torch.bfloat16, device=DEV).transpose(1, 2))


def unpack(codes):
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2)


@pytest.mark.parametrize("tokens,heads,dim,page,order", [
    (1, 1, 64, 16, "head"), (33, 2, 128, 16, "token"), (100, 3, 192, 64, "head"), (17, 5, 256, 1024, "token"), (513, 8, 128, 32, "head")])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_append_stores_the_defined_codes(tokens, heads, dim, page, order, dtype):
    rng = np.random.default_rng(tokens + dim)
    pages = tokens // page + 4
    kc, km = pools(pages, heads, page, dim, order, fill=0xA5)
    vc, vm = pools(pages, heads, page, dim, order, fill=0xA5)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=heads)
    x = rng.normal(size=(2, tokens, heads, dim)) * 10.0 ** rng.integers(-4, 4, (2, tokens, heads, 1)) + rng.normal(size=(2, tokens, heads, 1))
    x[0, 0, 0] = 0.0                             # constant vectors: scale 2^-40, all codes 0
    x[1, 0, 0] = -1.5
    x[0, -1, -1, 1:] = 0.0
    both = torch.tensor(x, device=DEV).to(dtype)
    fused = torch.cat([both[0], both[1]], 1)     # k and v as slices of one product
    slots = torch.tensor(rng.permutation(pages * page)[:tokens], device=DEV)
    skipped = tokens > 20
    if skipped:
        slots[7] = -1
    ks, vs = kv.append(fused[:, :heads], fused[:, heads:], slots, with_stored=True)
    kv.poll_status()
    for codes, meta, stored, given in ((kc, km, ks, both[0]), (vc, vm, vs, both[1])):
        code, scale, offset, value = plain_pack(given.float().cpu().numpy())
        keep = slots >= 0
        p, o = slots[keep] // page, slots[keep] % page
        assert np.array_equal(unpack(codes[p, :, o]).cpu().numpy(), code[keep.cpu().numpy()])
        want = np.concatenate([scale, offset], -1)[keep.cpu().numpy()]
        assert np.array_equal(meta[p, :, o].float().cpu().numpy(), want)
        assert torch.equal(stored.cpu(), torch.tensor(value).float().to(dtype))
        assert (np.abs(value - given.double().cpu().numpy()) <= scale / 2 * (1 + 1e-6)).all()
        touched = torch.zeros(pages, page, dtype=torch.bool, device=DEV)
        touched[p, o] = True
        assert (codes.transpose(1, 2)[~touched] == 0xA5).all() and (meta.transpose(1, 2)[~touched] == 0).all()


def test_append_decides_ties_and_extreme_scales_as_division_does():
    """Values half-way between two codes (k + 1/2 scales above the least), one float32 to either side of it, and scales from
    2^-40 to 2^120: the code is round-to-even of the correctly rounded quotient."""
    rng = np.random.default_rng(8)
    rows = []
    for e in (-45, -38, -20, -3, 0, 7, 60, 105, 120):
        for _ in range(40):
            scale = np.float32((128 + rng.integers(0, 128)) * 2.0 ** (e - 7))
            x = (rng.integers(0, 15, 64) + 0.5) * np.float64(scale)
            x = x.astype(np.float32)
            x = np.where(rng.random(64) < 0.3, np.nextafter(x, np.float32(np.inf)), x)
            x = np.where(rng.random(64) < 0.2, np.nextafter(x, np.float32(-np.inf)), x)
            x[0], x[1] = 0.0, np.float32(15.0 * np.float64(scale))
            rows.append(x)
    x = np.stack(rows).astype(np.float32)[:, None]
    n = len(rows)
    kc, km = pools(-(-n // 16), 1, 16, 64)
    vc, vm = pools(-(-n // 16), 1, 16, 64)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=1)
    t = torch.tensor(x, device=DEV)
    kv.append(t, -t, torch.arange(n, device=DEV))
    for codes, meta, given in ((kc, km, x), (vc, vm, -x)):
        code, scale, offset, _ = plain_pack(given)
        assert np.array_equal(unpack(codes.view(-1, 32)[:n]).cpu().numpy(), code[:, 0])
        assert np.array_equal(meta.view(-1, 2)[:n].float().cpu().numpy(), np.concatenate([scale, offset], -1)[:, 0])


def test_append_vectors_without_a_range_read_as_nan_and_harm_no_other():
    kc, km = pools(2, 2, 16, 64)
    vc, vm = pools(2, 2, 16, 64)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=2)
    x = torch.randn(4, 2, 64, device=DEV)
    x[0, 0, 5], x[1, 1, 0], x[2, 0, 63] = math.nan, math.inf, -math.inf
    x[3, 0, 0], x[3, 0, 1] = 3.3e38, -3.3e38     # a range that float32 does not hold
    ks, vs = kv.append(x, torch.ones_like(x), ints([0, 1, 2, 3], torch.int64), with_stored=True)
    bad = torch.zeros(4, 2, dtype=torch.bool, device=DEV)
    bad[0, 0] = bad[1, 1] = bad[2, 0] = bad[3, 0] = True
    assert ks[bad].isnan().all() and ks[~bad].isfinite().all() and (vs == 1).all()
    assert km[0, :, :4, 1].T[bad].isnan().all() and (km[0, :, :4, 0].T[bad] == 1).all()


def test_append_count_and_slots_past_the_pool():
    kc, km = pools(2, 1, 16, 64)
    vc, vm = pools(2, 1, 16, 64)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=1)
    x = torch.randn(3, 1, 64, device=DEV)
    kv.append(x, x, ints([1, 2, 3], torch.int64), count=ints([2]))
    kv.poll_status()
    assert (km[0, 0, 3] == 0).all() and (km[0, 0, 1:3, 0] > 0).all()
    kv.append(x, x, ints([32, 1 << 40, 31], torch.int64))
    with pytest.raises(fb.FiError) as e:
        kv.poll_status()
    assert e.value.status == fb.FI_ERR_INVALID_ARG
    kv.poll_status()                             # reported once
    assert km[1, 0, 15, 0] > 0


# ------------------------------------------------------------------------------------------------------------- attention

class Attention:
    """A filled store, queries and the formula in 64 bits."""

    def __init__(self, *, lens, queries, q_heads, kv_heads, dim, page=16, dtype=torch.bfloat16, order="head", window=0, size=1.0,
                 rows=None, seed=0, room=0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.lens, self.queries, self.window, self.dim, self.group = lens, queries, window, dim, q_heads // kv_heads
        n = len(lens)
        self.rows = list(range(n)) if rows is None else rows
        blocks = max(1, max(-(-x // page) for x in lens), room // page)      # room: keys the table has columns for
        pages = sum(-(-x // page) for x in lens) + 3
        self.kc, self.km = pools(pages, kv_heads, page, dim, order)
        self.vc, self.vm = pools(pages, kv_heads, page, dim, order)
        for c in (self.kc, self.vc):
            c.copy_(torch.randint(0, 256, c.shape, generator=gen, device=DEV, dtype=torch.uint8))
        for m in (self.km, self.vm):             # scales differ by powers of ten from key to key
            m[..., 0] = (size * 0.3 * 10.0 ** (torch.rand(m.shape[:3], generator=gen, device=DEV) - 0.5)).to(torch.bfloat16)
            m[..., 1] = (size * (torch.randn(m.shape[:3], generator=gen, device=DEV) - 2)).to(torch.bfloat16)
        order_ = rng.permutation(pages)
        self.table = torch.full((max(self.rows) + 2, blocks + 2), pages + 99, dtype=torch.int32, device=DEV)   # what must not be read
        all_lens = [0] * self.table.shape[0]
        at = 0
        for row, x in zip(self.rows, lens):
            u = -(-x // page)
            self.table[row, :u] = ints(order_[at:at + u])
            at += u
            all_lens[row] = x
        self.d_lens = ints(all_lens)
        self.cu = np.concatenate([[0], np.cumsum(queries)]).tolist()
        tokens = self.cu[-1]
        self.q = (size * torch.randn(tokens + 2, q_heads, dim, generator=gen, device=DEV)).to(dtype)
        self.kv = fb.KvCache(self.kc, self.km, self.vc, self.vm, q_heads=q_heads)
        self.page, self.kv_heads = page, kv_heads

    def run(self, q=None, **kw):
        q = self.q if q is None else q
        args = dict(cu_tokens=ints(self.cu), row_idx=ints(self.rows), max_query=max(self.queries), window=self.window, with_lse=True)
        args.update(kw)
        return self.kv.attend(q, self.d_lens, self.table, **args)

    def values(self, which, i, h):
        c, m = (self.kc, self.km) if which == "k" else (self.vc, self.vm)
        x = self.lens[i]
        p = self.table[self.rows[i], :-(-x // self.page)].long()
        codes, meta = c[p][:, h].reshape(-1, self.dim // 2)[:x], m[p][:, h].reshape(-1, 2)[:x].double()
        return unpack(codes).double() * meta[:, :1] + meta[:, 1:]

    def check(self, out, lse, scale=None, q=None, halves=False):
        """`halves`: keys and values were rounded to half precision (relative 2^-11 each) before the products.  A score is then off by
        a sum of head_dim independent roundings: six times the root of the sum of their squares (Hoeffding: exceeded once in 3e7)."""
        q = self.q if q is None else q
        scale = self.dim ** -0.5 if scale is None else scale
        half_weights = 2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21
        if halves:
            half_weights *= 2
        for i, (length, n) in enumerate(zip(self.lens, self.queries)):
            if n == 0:
                continue
            a, b = self.cu[i], self.cu[i + 1]
            pos = torch.arange(length - n, length, device=DEV)[:, None]
            t = torch.arange(length, device=DEV)
            seen = t <= pos
            if self.window:
                seen = seen & (t > pos - self.window)
            empty = ~seen.any(-1)
            for h in range(self.kv_heads):
                k, v = self.values("k", i, h), self.values("v", i, h)
                parts = v.abs().amax(-1) + 15 * self.vm_scale(i, h)     # codes and offset are summed apart
                for g in range(h * self.group, (h + 1) * self.group):
                    x = q[a:b, g].double() @ k.T * scale
                    reach = (q[a:b, g].double().abs().sum(-1, keepdim=True) * self.k_reach(i, h) * abs(scale)).amax(-1)
                    x = x.masked_fill(~seen, -math.inf)
                    p = torch.softmax(x, -1).nan_to_num(0.0)
                    want = p @ v
                    # exponents: the scores' float32 sums, a few u of the largest parts of a score
                    exponent = 2.0 ** -20 * (1 + reach[:, None])
                    if halves and length:
                        exponent = exponent + 6 * 2.0 ** -11 * abs(scale) * (q[a:b, g].double().square() @ k.T.square()).sqrt().amax(-1, keepdim=True)
                    bound = (half_weights + 2 * exponent + 2.0 ** -18) * (p @ parts[:, None]) + rounding(q.dtype) * want.abs() * 1.01
                    got = out[a:b, g].double()
                    assert got.isfinite().all()
                    assert ((got - want).abs() <= bound).all(), (i, g, ((got - want).abs() / bound).max().item())
                    assert (got[empty] == 0).all()
                    if lse is not None:
                        ref = torch.logsumexp(x, -1)
                        assert (lse[a:b, g][empty] == -math.inf).all()
                        d = (lse[a:b, g].double() - ref)[~empty].abs()
                        assert (d <= exponent[~empty, 0] + 2.0 ** -20 * ref[~empty].abs()).all()

    def vm_scale(self, i, h):
        p = self.table[self.rows[i], :-(-self.lens[i] // self.page)].long()
        return self.vm[p][:, h].reshape(-1, 2)[:self.lens[i], 0].double()

    def k_reach(self, i, h):
        """Largest size a key's code and offset parts reach together, per key."""
        p = self.table[self.rows[i], :-(-self.lens[i] // self.page)].long()
        m = self.km[p][:, h].reshape(-1, 2)[:self.lens[i]].double()
        return (15 * m[:, 0] + m[:, 1].abs())[None] if m.numel() else torch.zeros(1, 1, dtype=torch.float64, device=DEV)


ATTEND_CASES = {
    "one-key": dict(lens=[1], queries=[1], q_heads=1, kv_heads=1, dim=64),
    "no-key": dict(lens=[0, 5, 0], queries=[1, 1, 2], q_heads=4, kv_heads=2, dim=128),
    "decode": dict(lens=[1, 15, 16, 17, 31, 33, 127, 128, 129, 300, 511, 1000], queries=[1] * 12, q_heads=8, kv_heads=2, dim=128),
    "groups-of-5": dict(lens=[70, 200], queries=[1, 1], q_heads=15, kv_heads=3, dim=64, page=32),
    "groups-of-16": dict(lens=[257, 64], queries=[1, 1], q_heads=32, kv_heads=2, dim=128, order="token"),
    "groups-of-40": dict(lens=[90, 300], queries=[1, 2], q_heads=40, kv_heads=1, dim=128),
    "head-192": dict(lens=[200, 3, 450], queries=[1, 3, 2], q_heads=8, kv_heads=2, dim=192, page=64),
    "head-256": dict(lens=[200, 3, 450], queries=[1, 2, 9], q_heads=6, kv_heads=2, dim=256, order="token"),
    "drafted": dict(lens=[40, 100, 8, 260], queries=[3, 8, 8, 1], q_heads=8, kv_heads=2, dim=128),
    "more-queries-than-keys": dict(lens=[5, 40], queries=[9, 41], q_heads=4, kv_heads=1, dim=64),
    "no-queries": dict(lens=[50, 60, 70, 80], queries=[0, 2, 0, 0], q_heads=4, kv_heads=4, dim=64),
    "prompt": dict(lens=[200, 333], queries=[200, 150], q_heads=4, kv_heads=2, dim=128, page=128),
    "window": dict(lens=[500, 20, 300, 257], queries=[1, 1, 4, 30], q_heads=8, kv_heads=2, dim=128, window=100),
    "window-of-one": dict(lens=[140, 129], queries=[3, 1], q_heads=4, kv_heads=4, dim=64, window=1),
    "long": dict(lens=[20011], queries=[1], q_heads=16, kv_heads=2, dim=128, page=256),
    "many": dict(lens=[int(x) for x in np.random.default_rng(1).integers(1, 400, 300)], queries=[1] * 300, q_heads=4, kv_heads=1, dim=64),
    "rows": dict(lens=[33, 90, 17], queries=[1, 1, 1], q_heads=4, kv_heads=2, dim=64, rows=[5, 0, 9]),
}


@pytest.mark.parametrize("name", ATTEND_CASES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_matches_formula(name, dtype):
    a = Attention(dtype=dtype, **ATTEND_CASES[name])
    out, lse = a.run()
    a.check(out, lse)
    again, _ = a.run()
    tokens = a.cu[-1]
    assert torch.equal(out[:tokens], again[:tokens])              # cuts and sums in a fixed order
    a.kv.poll_status()


PROMPT_CASES = {name: c for name, c in ATTEND_CASES.items() if c["dim"] <= 128 and name not in ("long", "many")}
PROMPT_CASES.update({
    "tiles": dict(lens=[128, 129, 384, 700], queries=[128, 127, 300, 1], q_heads=8, kv_heads=2, dim=128, page=32),
    "one-head": dict(lens=[600], queries=[260], q_heads=1, kv_heads=1, dim=64, page=16),
    "behind-a-context": dict(lens=[1000, 131], queries=[70, 3], q_heads=14, kv_heads=2, dim=128, order="token"),
    "narrow-window": dict(lens=[700, 300], queries=[400, 300], q_heads=4, kv_heads=2, dim=64, window=33),
    "wide-window": dict(lens=[900], queries=[150], q_heads=4, kv_heads=1, dim=128, window=500, page=64),
    "many-requests": dict(lens=[int(x) for x in np.random.default_rng(2).integers(1, 200, 90)],
                          queries=[int(x) for x in np.random.default_rng(3).integers(0, 40, 90)], q_heads=8, kv_heads=2, dim=64),
})
MANY = 20000        # a hint of this many queries takes the kernel for prompts, whatever there are


@pytest.mark.parametrize("name", PROMPT_CASES)
def test_attend_prompt_kernel_matches_formula(name):
    a = Attention(room=1024, **PROMPT_CASES[name])
    out, lse = a.run(max_query=MANY)
    a.check(out, lse, halves=True)
    again, _ = a.run(max_query=MANY)
    assert torch.equal(out[:a.cu[-1]], again[:a.cu[-1]])
    a.kv.poll_status()


@pytest.mark.parametrize("size,scale", [(1e-3, 1.0), (30.0, 1.0), (1e4, -1.0), (1.0, 0.0)])
def test_attend_prompt_kernel_sizes_of_values(size, scale):
    a = Attention(lens=[130, 700], queries=[100, 2], q_heads=4, kv_heads=2, dim=128, size=size, room=1024)
    scale = scale / (size * size * 128)
    out, lse = a.run(scale=scale, max_query=MANY)
    a.check(out, lse, scale=scale, halves=True)


def test_attend_prompt_kernel_hidden_nan_and_bad_pages():
    a = Attention(lens=[300], queries=[40], q_heads=4, kv_heads=2, dim=128, room=1024)
    whole, _ = a.run(max_query=MANY)
    page = a.table[0, 280 // a.page].long()
    a.vm[page, 0, 280 % a.page, 1] = math.nan                    # queries 0 .. 19 stand before it
    out, lse = a.run(max_query=MANY)
    assert torch.equal(out[:20], whole[:20]) and out[20:40, :2].isnan().all() and torch.equal(out[20:40, 2:], whole[20:40, 2:])
    a.kv.poll_status()
    b = Attention(lens=[300], queries=[40], q_heads=4, kv_heads=2, dim=128, room=1024)
    b.table[0, 3] = -1                                           # 16 keys hidden
    hidden = b.run(max_query=MANY)
    with pytest.raises(fb.FiError):
        b.kv.poll_status()
    few = b.run(max_query=1)
    with pytest.raises(fb.FiError):
        b.kv.poll_status()
    assert ((hidden[0][:40].double() - few[0][:40].double()).abs() <= 2.0 ** -6 * (1 + few[0][:40].double().abs())).all()
    assert ((hidden[1][:40] - few[1][:40]).abs() <= 2.0 ** -7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_strides_scale_count_and_untouched_rows(dtype):
    a = Attention(lens=[100, 37, 256, 80], queries=[1] * 4, q_heads=8, kv_heads=2, dim=128, dtype=dtype)
    wide = torch.randn(4, 20, 128, device=DEV).to(dtype)
    q = wide[:, 3:11]                                             # a slice of one product
    out = torch.full((8, 4, 128), 7.0, device=DEV, dtype=dtype).transpose(0, 1)
    lse = torch.full((4, 8), 7.0, device=DEV)
    a.kv.attend(q, a.d_lens, a.table, row_idx=ints(a.rows), batch_count=ints([3]), scale=-0.05, out=out, lse=lse)
    assert (out[3] == 7).all() and (lse[3] == 7).all()
    a.lens, a.queries, a.cu = a.lens[:3], a.queries[:3], a.cu[:4]
    a.check(out, lse, scale=-0.05, q=q)


@pytest.mark.parametrize("dim,queries,q_heads", [(64, 1, 1), (64, 3, 5), (64, 9, 3), (128, 1, 7), (128, 2, 5), (192, 3, 3), (256, 1, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_joins_many_parts(dim, queries, q_heads, dtype):
    """One key head over 20,001 keys: a row's result is added up from 79 or 157 parts, of tiles that rows do not fill."""
    a = Attention(lens=[20001], queries=[queries], q_heads=q_heads, kv_heads=1, dim=dim, page=64, dtype=dtype)
    out, lse = a.run()
    a.check(out, lse)
    again, _ = a.run()
    assert torch.equal(out[:queries], again[:queries])
    a.kv.poll_status()


@pytest.mark.parametrize("size", [1e-3, 30.0, 1e4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_sizes_of_values(size, dtype):
    """Queries, scales and offsets far from 1: halves must neither run over nor vanish."""
    a = Attention(lens=[130, 700], queries=[1, 2], q_heads=4, kv_heads=2, dim=128, dtype=dtype, size=size)
    out, lse = a.run(scale=1.0 / (size * size * 128))
    a.check(out, lse, scale=1.0 / (size * size * 128))


def test_attend_hidden_nan_and_garbage_stay_hidden():
    """Places behind the last key hold whatever was there; keys that a query does not see may read as NaN."""
    a = Attention(lens=[37, 150], queries=[1, 3], q_heads=4, kv_heads=2, dim=128, window=60)
    for i, (row, x) in enumerate(zip(a.rows, a.lens)):
        last = a.table[row, (x - 1) // a.page].long()
        for m in (a.km, a.vm):
            m[last, :, x % a.page if x % a.page else a.page:] = math.nan
    first = a.table[a.rows[1], 0].long()
    a.km[first], a.vm[first] = math.nan, math.inf                # outside of every query's window
    second = a.table[a.rows[1], 9].long()
    out, lse = a.run()
    assert out[:4].isfinite().all()
    ref, ref_lse = out.clone(), lse.clone()
    a.km[second, 0, 149 % a.page, 1] = math.nan                  # the newest key: only the last query sees it
    out, lse = a.run()
    assert torch.equal(out[1:3], ref[1:3]) and out[3, :2].isnan().all() and torch.equal(out[3, 2:], ref[3, 2:])


def test_attend_pages_outside_the_pool_are_hidden_and_reported():
    a = Attention(lens=[100], queries=[1], q_heads=2, kv_heads=1, dim=64)
    keep = a.table[0, 2].item()
    for bad in (-1, 10 ** 6):
        a.table[0, 2] = bad
        out, _ = a.run()
        with pytest.raises(fb.FiError):
            a.kv.poll_status()
        assert out[:1].isfinite().all()
    a.table[0, 2] = keep
    a.check(*a.run())
    a.kv.poll_status()


def test_attend_on_another_stream_and_handles_side_by_side():
    a = Attention(lens=[900, 33], queries=[1, 1], q_heads=8, kv_heads=2, dim=128)
    b = Attention(lens=[70, 600], queries=[1, 1], q_heads=8, kv_heads=2, dim=128, seed=3)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(s1):
        for _ in range(20):
            ra = a.run()
    with torch.cuda.stream(s2):
        for _ in range(20):
            rb = b.run()
    torch.cuda.synchronize()
    a.check(*ra)
    b.check(*rb)


def test_attend_in_a_graph():
    a = Attention(lens=[900, 33], queries=[1, 1], q_heads=8, kv_heads=2, dim=128)
    cu, rows, out = ints(a.cu), ints(a.rows), torch.empty_like(a.q)
    call = lambda: a.kv.attend(a.q, a.d_lens, a.table, cu_tokens=cu, row_idx=rows, out=out)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    a.check(out, None)


def test_store_past_four_gigabytes():
    """Offsets of codes beyond 2^32 bytes: the last pages of a large pool."""
    pages, heads, page, dim = 8300, 8, 1024, 128                 # 4.35 GB each
    kc = torch.zeros(pages, heads, page, dim // 2, dtype=torch.uint8, device=DEV)
    vc = torch.zeros_like(kc)
    km = torch.zeros(pages, heads, page, 2, dtype=torch.bfloat16, device=DEV)
    vm = torch.zeros_like(km)
    kv = fb.KvCache(kc, km, vc, vm, q_heads=heads)
    tokens = 40
    k, v = (torch.randn(tokens, heads, dim, device=DEV).to(torch.bfloat16) for _ in range(2))
    table = ints([[pages - 1]])
    slots = (pages - 1) * page + torch.arange(tokens, device=DEV)
    ks, vs = kv.append(k, v, slots, with_stored=True)
    q = torch.randn(1, heads, dim, device=DEV).to(torch.bfloat16)
    out = kv.attend(q, ints([tokens]), table)
    x = torch.einsum("hd,thd->ht", q[0].double(), ks.double()) / math.sqrt(dim)
    want = torch.einsum("ht,thd->hd", torch.softmax(x, -1), vs.double())
    # `stored` is rounded to bf16: scores move by 2^-8 of their parts, values and the result by 2^-8
    assert (out[0].double() - want).abs().max() <= 2.0 ** -8 * (4 + 2 * 8 * 4)
    assert (kc[: pages - 1].view(torch.int64) == 0).all()


# -------------------------------------------------------------------------------------------------------------- refusals

def test_refusals():
    def refused(f, *a, **k):
        with pytest.raises((fb.FiError, ValueError)) as e:
            f(*a, **k)
        if isinstance(e.value, fb.FiError):
            assert e.value.status == fb.FI_ERR_INVALID_ARG

    for bad in (dict(page_size=24, max_blocks=4), dict(page_size=8, max_blocks=4), dict(page_size=16, max_blocks=0),
                dict(page_size=1024, max_blocks=1 << 21), dict(page_size=16, max_blocks=4, max_batch=9000)):
        refused(fb.KvTables, **bad)
    t = fb.KvTables(page_size=16, max_blocks=4, max_batch=4)
    table = torch.zeros(8, 4, dtype=torch.int32, device=DEV)
    refused(t.extend, ints([0] * 8), ints([1]), ints([1]), table)                               # batch above max_batch
    refused(t.extend, ints([0] * 4), ints([1]), ints([1]), table[:, :3])                        # table too narrow
    refused(t.extend, ints([0] * 4), ints([1]), ints([1]), table, new_lens=ints([1] * 4))       # max_tokens missing
    refused(t.extend, ints([0] * 4, torch.int64), ints([1]), ints([1]), table)

    def cache(pages=2, heads=2, page=16, dim=64, q_heads=4):
        c, m = pools(pages, heads, page, dim)
        return fb.KvCache(c, m, c.clone(), m.clone(), q_heads=q_heads)
    refused(cache, dim=96)
    refused(cache, q_heads=3)
    refused(cache, page=24)
    kv = cache()
    x = torch.zeros(3, 2, 64, device=DEV)
    slots = ints([0, 1, 2], torch.int64)
    refused(kv.append, x.half(), x.half(), slots)
    refused(kv.append, x, x, slots[:2])
    refused(kv.append, x, x.bfloat16(), slots)
    odd = torch.zeros(3 * 2 * 64 + 1, device=DEV)[1:].view(3, 2, 64)
    refused(kv.append, odd, x, slots)                                                           # not on 16 bytes
    q = torch.zeros(1, 4, 64, device=DEV)
    table = torch.zeros(1, 2, dtype=torch.int32, device=DEV)
    refused(kv.attend, q[:, :3], ints([1]), table)
    refused(kv.attend, q, ints([1, 1]), table)                                                  # more rows than the table
    refused(kv.attend, q, ints([1]), table, window=-1)
    refused(kv.attend, q, ints([1]), table, scale=math.inf)
    refused(kv.attend, torch.zeros(0, 4, 64, device=DEV), ints([1]), table)                     # fewer tokens than requests
    refused(fb.head_norm_rope, torch.zeros(1, 1, 24, device=DEV), None, None, None, None, None)
    refused(fb.head_norm_rope, torch.zeros(1, 1, 32, device=DEV), None, None, None, rope_table(4, 64), ints([0]))
    refused(fb.head_norm_rope, torch.zeros(1, 1, 32, device=DEV), None, None, None, rope_table(4, 32), None)
    refused(fb.head_norm_rope, torch.zeros(1, 1, 32, device=DEV).half(), None, None, None, None, None)


def test_empty_calls_do_nothing():
    c, m = pools(2, 2, 16, 64)
    kv = fb.KvCache(c, m, c.clone(), m.clone(), q_heads=4)
    none = torch.zeros(0, 2, 64, device=DEV)
    kv.append(none, none, torch.zeros(0, dtype=torch.int64, device=DEV))
    out = kv.attend(torch.zeros(0, 4, 64, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV),
                    torch.zeros(0, 2, dtype=torch.int32, device=DEV))
    assert out.shape == (0, 4, 64)
    q, k = fb.head_norm_rope(torch.zeros(0, 4, 64, device=DEV), none, None, None, None, None)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    t = fb.KvTables(page_size=16, max_blocks=4)
    o = t.extend(torch.zeros(0, dtype=torch.int32, device=DEV), ints([1]), ints([1]), torch.zeros(0, 4, dtype=torch.int32, device=DEV))
    assert o.cu_tokens.tolist() == [0] and o.free_count.item() == 1
    torch.cuda.synchronize()
