"""Pages with several owners: fork, free, compact and copy_pages against a plain model of the tables (whole numbers: equal)."""
import random

import pytest
import torch

from paper_2002_02645_b200 import binding as fb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Model:
    """Tables of one layer as lists; every page is free or owned."""

    def __init__(self, rows, blocks, pages, page, seed=0):
        self.page, self.blocks, self.pages, self.rows = page, blocks, pages, rows
        self.lens = [0] * rows
        self.table = [[-1] * blocks for _ in range(rows)]
        self.free = list(range(pages))
        random.Random(seed).shuffle(self.free)
        self.shared = [0] * pages

    def used(self, row):
        return -(-self.lens[row] // self.page)

    def fill(self, row, tokens):
        want = -(-tokens // self.page)
        assert self.lens[row] == 0 and want <= self.blocks and want <= len(self.free)
        for j in range(want):
            self.table[row][j] = self.free.pop()
        self.lens[row] = tokens

    def fork(self, src, dst, n):
        granted, copies = [0] * len(src), [[-1, -1, 0] for _ in src]
        lens, stack, left = list(self.lens), list(self.free), len(self.free)
        for i in range(n):
            s, d = src[i], dst[i]
            if not (0 <= s < self.rows and 0 <= d < self.rows) or s == d or self.lens[d] or -(-self.lens[s] // self.page) > self.blocks:
                continue
            full, tail = divmod(self.lens[s], self.page)
            if tail:
                left -= 1
                if left < 0:
                    continue
                copies[i] = [self.table[s][full], stack[left], tail]
                self.table[d][full] = stack[left]
                self.free.pop()
            for j in range(full):
                self.table[d][j] = self.table[s][j]
                self.shared[self.table[s][j]] += 1
            granted[i], lens[d] = 1, self.lens[s]
        self.lens = lens
        return granted, copies

    def release(self, rows):
        gone = []
        for r in rows:
            if not 0 <= r < self.rows:
                continue
            for p in self.table[r][:self.used(r)]:
                self.shared[p] -= 1
                if self.shared[p] < 0:
                    gone.append(p)
                    self.shared[p] = 0
            self.lens[r] = 0
        self.free += sorted(gone)

    def compact(self):
        used = self.pages - len(self.free)
        holes = sorted(p for p in self.free if p < used)
        high = sorted(set(range(used, self.pages)) - set(self.free))
        assert len(holes) == len(high)
        name = dict(zip(high, holes))
        for r in range(self.rows):
            for j in range(self.used(r)):
                self.table[r][j] = name.get(self.table[r][j], self.table[r][j])
        for s, d in name.items():
            self.shared[d], self.shared[s] = self.shared[s], 0
        self.free = [self.pages - 1 - i for i in range(len(self.free))]
        return [[s, d, self.page] for s, d in zip(high, holes)]


class Device:
    def __init__(self, m, max_batch=64, table_extra=0):
        self.m = m
        self.h = fb.KvTables(page_size=m.page, max_blocks=m.blocks, max_batch=max_batch)
        self.extra = table_extra
        self.load()

    def load(self):
        m = self.m
        self.lens, self.shared = ints(m.lens), ints(m.shared)
        self.table = ints([r + [-7] * self.extra for r in m.table]).view(m.rows, m.blocks + self.extra)
        self.free, self.count = ints(m.free + [-1] * (m.pages - len(m.free))), ints([len(m.free)])

    def same(self):
        m = self.m
        assert self.lens.tolist() == m.lens and self.count.tolist() == [len(m.free)] and self.shared.tolist() == m.shared
        assert self.free[:len(m.free)].tolist() == m.free
        table = self.table.tolist()
        for r in range(m.rows):
            assert table[r][:m.used(r)] == m.table[r][:m.used(r)]
            assert table[r][m.blocks:] == [-7] * self.extra

    def fork(self, src, dst, n=None, in_place=True):
        n = len(src) if n is None else n
        out = None
        if in_place:
            out = fb.ForkOut(len(src), self.m.rows, DEV)
            out.lens, out.free_count = self.lens, self.count
        before = (self.lens.clone(), self.count.clone())
        got = self.h.fork(ints(src), ints(dst), self.lens, self.free, self.count, self.table, self.shared,
                          batch_count=None if n == len(src) else ints([n]), out=out)
        if not in_place:
            assert torch.equal(before[0], self.lens) and torch.equal(before[1], self.count)
            self.lens, self.count = got.lens.clone(), got.free_count.clone()
        granted, copies = self.m.fork(src, dst, n)
        assert got.granted.tolist() == granted and got.copies.tolist() == copies
        self.same()
        return got

    def release(self, rows, n=None, in_place=True):
        n = len(rows) if n is None else n
        got = self.h.free(ints(rows), self.lens, self.free, self.count, self.table, self.shared, batch_count=None if n == len(rows) else ints([n]),
                          out=(self.lens, self.count) if in_place else None)
        if not in_place:
            assert self.lens.tolist() == self.m.lens
            self.lens, self.count = (t.clone() for t in got)
        self.m.release(rows[:n])
        self.same()

    def compact(self):
        copies, moves = self.h.compact(self.lens, self.free, self.count, self.table, self.shared)
        want = self.m.compact()
        assert moves.tolist() == [len(want)]
        assert copies.tolist() == want + [[-1, -1, 0]] * (self.m.pages // 2 - len(want))
        self.same()
        return copies, moves


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("pages", [37, 64, 1000, 2500])
@pytest.mark.parametrize("in_place", [False, True])
def test_random_life(page, pages, in_place):
    """Prompts join, fork (also forks of forks), end in any order and are compacted, until the pool has been through a few times."""
    rng = random.Random(page + pages)
    m = Model(rows=40, blocks=9, pages=pages, page=page)
    d = Device(m, table_extra=3)
    for step in range(60):
        empty = [r for r in range(40) if m.lens[r] == 0]
        some = [r for r in range(40) if m.lens[r]]
        kind = rng.choice(("fill", "fork", "fork", "free", "compact"))
        if kind == "fill" and empty:
            row, tokens = rng.choice(empty), rng.randint(1, 9 * page)
            if -(-tokens // page) <= len(m.free):
                m.fill(row, tokens)
                d.load()
        elif kind == "fork" and len(empty) > 2 and some:
            k = rng.randint(1, len(empty))
            dst = rng.sample(empty, k)
            src = [rng.choice(some + empty[:1]) for _ in dst]
            for i in range(k):
                if rng.random() < 0.1:
                    src[i] = rng.choice((-1, 40, dst[i]))
                if rng.random() < 0.05:
                    dst[i] = rng.choice([-1, 41, rng.choice(some)])
            d.fork(src, dst, rng.randint(0, k) if rng.random() < 0.3 else None, in_place)
        elif kind == "free" and some:
            rows = rng.sample(some, rng.randint(1, len(some)))
            if rng.random() < 0.2:
                rows.append(rng.choice((-1, 40)))
            d.release(rows, rng.randint(0, len(rows)) if rng.random() < 0.3 else None, in_place)
        elif kind == "compact":
            d.compact()
    d.release([r for r in range(40) if m.lens[r]], None, in_place)
    assert len(m.free) == pages and not any(m.shared)
    d.compact()


def test_refused_forks_leave_no_trace_and_tails_are_served_in_order():
    m = Model(rows=12, blocks=4, pages=7, page=16)
    m.fill(0, 33)                   # two full pages and a tail
    m.fill(1, 32)                   # no tail
    m.lens[2] = 100                 # a length that its table cannot hold
    d = Device(m)
    #        tail  tail  no page left  needs none  dst full  too long  twice a source, empty source
    d.fork([0, 0, 0, 1, 0, 2, 11], [3, 4, 5, 6, 1, 7, 8])
    assert d.count.item() == 0 and m.shared[m.table[0][0]] == 2
    m.lens[2] = 0
    d.load()
    d.release([0, 3, 4])
    d.fork([6], [0])
    d.release([1])
    d.release([6, 0])
    assert len(m.free) == 7


def test_ended_together_in_one_call():
    """A prompt and all of its continuations in one call: their pages come back once."""
    m = Model(rows=30, blocks=8, pages=100, page=16)
    m.fill(0, 16 * 8)
    d = Device(m)
    d.fork([0] * 29, list(range(1, 30)))
    assert m.shared[m.table[0][3]] == 29 and len(m.free) == 92
    d.release(list(range(5, 30)) + [0])
    d.release([1, 2, 3, 4])
    assert len(m.free) == 100


def test_large_tables():
    """8,192 forks of 50 prompts, several CTAs; then half of them end, then a pool of many segments is compacted."""
    rng = random.Random(1)
    m = Model(rows=9000, blocks=40, pages=13001, page=16)
    for r in range(50):
        m.fill(r, rng.randint(1, 640))
    d = Device(m, max_batch=8192)
    rows = list(range(50, 8242))
    rng.shuffle(rows)
    d.fork([rng.randrange(50) for _ in rows], rows)
    ends = rng.sample(range(8242), 5000)
    d.release(ends)
    copies, moves = d.compact()
    assert moves.item() > 1000
    d.release([r for r in range(9000) if m.lens[r]][:8192])


def test_compact_of_nothing_and_everything():
    m = Model(rows=3, blocks=4, pages=12, page=16)
    d = Device(m)
    assert d.compact()[1].item() == 0               # all free
    for r in range(3):
        m.fill(r, 64)
    d.load()
    assert d.compact()[1].item() == 0               # none free
    m = Model(rows=3, blocks=4, pages=1, page=16)
    d = Device(m)
    d.compact()
    m.fill(1, 3)
    d.load()
    d.compact()


@pytest.mark.parametrize("pages", [4095, 4097, 70001, 200000])
@pytest.mark.parametrize("share", [0.02, 0.5, 0.97])
def test_compact_of_large_pools(pages, share):
    """Pools for many CTAs, a few or nearly all of their pages free, in any order."""
    rng = random.Random(pages)
    m = Model(rows=20, blocks=60, pages=pages, page=16)
    m.free = rng.sample(range(pages), int(share * pages))
    left = sorted(set(range(pages)) - set(m.free))
    for r in range(20):
        m.lens[r] = rng.randint(0, 960)
        m.table[r] = [rng.choice(left) for _ in range(60)]
    m.shared = [0 if p % 3 else p % 7 for p in range(pages)]
    for p in m.free:
        m.shared[p] = 0
    Device(m).compact()


def pools(gen, pages, heads, page, dim):
    codes = lambda: torch.randint(0, 256, (pages, heads, page, dim // 2), generator=gen, device=DEV, dtype=torch.uint8)
    meta = lambda: torch.randn(pages, heads, page, 2, generator=gen, device=DEV).bfloat16()
    return codes(), meta(), codes(), meta()


@pytest.mark.parametrize("page,heads,dim", [(16, 1, 64), (64, 8, 128), (32, 3, 192), (128, 2, 256)])
@pytest.mark.parametrize("token_major", [False, True])
def test_copy_pages(page, heads, dim, token_major):
    gen = torch.Generator(device=DEV).manual_seed(dim)
    p = pools(gen, 50, heads, page, dim)
    if token_major:                                 # tokens outermost within a page
        p = tuple(t.transpose(1, 2).contiguous().transpose(1, 2) for t in p)
    kv = fb.KvCache(*p, q_heads=heads)
    rng = random.Random(dim)
    order = rng.sample(range(50), 40)
    copies = [[order[i], order[20 + i], rng.choice((0, 1, 3, page // 2 + 1, page, page))] for i in range(20)]
    copies[4][0] = -1
    copies[6][0] = copies[5][0]                     # a source twice
    want = [t.clone() for t in p]
    for s, t, n in copies[:17]:
        for w in want:
            if s >= 0:
                w[t, :, :n] = w[s, :, :n]
    kv.copy_pages(ints(copies), count=ints([17]))
    kv.poll_status()
    assert all(torch.equal(a, b) for a, b in zip(p, want))
    # the rest of the list; pages outside of the pool are skipped and told
    for s, t, n in copies[17:]:
        for w in want:
            w[t, :, :n] = w[s, :, :n]
    kv.copy_pages(ints(copies[17:] + [[order[0], 50, 1], [50, order[1], 1], [order[2], -1, 1], [1 << 30, 0, 1]]))
    with pytest.raises(fb.FiError, match="copy_pages"):
        kv.poll_status()
    assert all(torch.equal(a, b) for a, b in zip(p, want))
    kv.copy_pages(ints([]).view(0, 3))
    kv.poll_status()


def test_forked_requests_attend_as_if_they_had_been_stored_alone():
    """A prompt is stored, forked, the copies go on with tokens of their own, one ends, the pool is compacted: attention sees for each
    what it would have seen in a store of its own."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    page, pages, heads, dim, rows = 16, 40, 2, 64, 5
    rand = lambda n: torch.randn(n, heads, dim, generator=gen, device=DEV).bfloat16()
    codes = lambda n: torch.zeros(n, heads, page, dim // 2, dtype=torch.uint8, device=DEV)
    meta = lambda n: torch.zeros(n, heads, page, 2, dtype=torch.bfloat16, device=DEV)

    def store(n_pages, n_rows):
        kv = fb.KvCache(codes(n_pages), meta(n_pages), codes(n_pages), meta(n_pages), q_heads=4)
        t = fb.KvTables(page_size=page, max_blocks=8, max_batch=8)
        state = dict(lens=torch.zeros(n_rows, dtype=torch.int32, device=DEV), free=torch.randperm(n_pages, generator=gen, device=DEV).int(),
                     count=ints([n_pages]), table=torch.full((n_rows, 8), -1, dtype=torch.int32, device=DEV),
                     shared=torch.zeros(n_pages, dtype=torch.int32, device=DEV))
        return kv, t, state

    def add(kv, t, s, row_list, k, v, new):
        out = t.extend(s["lens"], s["free"], s["count"], s["table"], new_lens=ints(new), row_idx=ints(row_list), max_tokens=sum(new))
        kv.append(k, v, out.slot_map)
        s["lens"], s["count"] = out.lens, out.free_count

    kv, t, s = store(pages, rows)
    pk, pv = rand(37), rand(37)
    add(kv, t, s, [1], pk, pv, [37])
    out = t.fork(ints([1, 1, 1]), ints([0, 2, 4]), s["lens"], s["free"], s["count"], s["table"], s["shared"])
    kv.copy_pages(out.copies)
    s["lens"], s["count"] = out.lens, out.free_count
    new = {0: 30, 1: 4, 2: 11, 4: 1}
    more = {r: (rand(n), rand(n)) for r, n in new.items()}
    add(kv, t, s, list(new), torch.cat([more[r][0] for r in new]), torch.cat([more[r][1] for r in new]), list(new.values()))
    s["lens"], s["count"] = t.free(ints([2]), s["lens"], s["free"], s["count"], s["table"], s["shared"])
    copies, moves = t.compact(s["lens"], s["free"], s["count"], s["table"], s["shared"])
    kv.copy_pages(copies, count=moves)
    live = [0, 1, 4]
    used = sorted({p for r in live for p in s["table"][r, :-(-int(s["lens"][r]) // page)].tolist()})
    assert used == list(range(pages - int(s["count"])))
    q = torch.randn(3, 4, dim, generator=gen, device=DEV).bfloat16()
    got = kv.attend(q, s["lens"], s["table"], row_idx=ints(live))
    for i, r in enumerate(live):
        kv1, t1, s1 = store(8, 1)
        add(kv1, t1, s1, [0], torch.cat([pk, more[r][0]]), torch.cat([pv, more[r][1]]), [37 + new[r]])
        assert torch.equal(kv1.attend(q[i:i + 1], s1["lens"], s1["table"]), got[i:i + 1])
    kv.poll_status()


def test_capture():
    m = Model(rows=20, blocks=6, pages=60, page=16)
    for r in range(4):
        m.fill(r, 20 * r + 13)
    d = Device(m)
    src, dst = ints([0, 1, 2, 3, 3]), ints([10, 11, 12, 13, 14])
    table, shared, free = d.table.clone(), d.shared.clone(), d.free.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        d.table.copy_(table); d.shared.copy_(shared); d.free.copy_(free)
        out = d.h.fork(src, dst, d.lens, d.free, d.count, d.table, d.shared)
        lens, count = d.h.free(src[1:4], out.lens, d.free, out.free_count, d.table, d.shared)
        copies, moves = d.h.compact(lens, d.free, count, d.table, d.shared)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    granted, cp = m.fork(src.tolist(), dst.tolist(), 5)
    m.release([1, 2, 3])
    want = m.compact()
    assert out.granted.tolist() == granted and out.copies.tolist() == cp and copies.tolist()[:len(want)] == want and moves.item() == len(want)
    d.lens, d.count = lens, count
    d.same()


def test_refusals():
    m = Model(rows=4, blocks=4, pages=8, page=16)
    d = Device(m, max_batch=4)
    rows = ints([0, 1])
    state = (d.lens, d.free, d.count, d.table)
    bad = [lambda: d.h.fork(rows, rows[:1], *state, d.shared), lambda: d.h.fork(rows.long(), rows, *state, d.shared),
           lambda: d.h.fork(rows, rows, *state, d.shared[:7]), lambda: d.h.fork(rows, rows, *state[:3], d.table[:, :3], d.shared),
           lambda: d.h.free(rows.cpu(), *state, d.shared), lambda: d.h.free(rows, *state, d.shared.float()),
           lambda: d.h.free(rows, *state, d.shared, out=(d.lens[:3], d.count)), lambda: d.h.compact(d.lens, d.free, d.count, d.table, d.shared[:3])]
    gen = torch.Generator(device=DEV).manual_seed(1)
    kv = fb.KvCache(*pools(gen, 4, 1, 16, 64), q_heads=1)
    bad += [lambda: kv.copy_pages(rows), lambda: kv.copy_pages(ints([[0, 1, 1]]).long()), lambda: kv.copy_pages(ints([[0, 1]])),
            lambda: kv.copy_pages(ints([[0, 1, 1]]), count=rows.float())]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    five, many = ints([0, 1, 2, 3, 0]), torch.zeros(1048577, dtype=torch.int32, device=DEV)
    for call in (lambda: d.h.fork(five, five, *state, d.shared), lambda: d.h.free(five, *state, d.shared),
                 lambda: d.h.free(rows, d.lens, many, d.count, d.table, many.clone()), lambda: d.h.compact(d.lens, many, d.count, d.table, many.clone())):
        with pytest.raises(fb.FiError, match="INVALID"):
            call()
