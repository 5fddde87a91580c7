"""The cache's pages against a plain simulation, and the operators run together:
sequences that grow, fork, leave and move while what they hold stays theirs."""
import random

import pytest
import torch

import paper_2609_00049_gb300 as rq
from kv_reference import gen, i32, starts_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


class Pool:
    """The bookkeeping as the header words it, and the same on the GPU."""

    def __init__(self, n_pages, n_rows, max_pages, page=16, block=1, layers=2, kv=1, D=16):
        self.page, self.n_pages, self.n_rows, self.max_pages = page, n_pages, n_rows, max_pages
        self.used = [0] * n_pages
        self.tables = [[-1] * max_pages for _ in range(n_rows)]
        self.lengths = [0] * n_rows
        shape = (layers, n_pages, kv, page, D)
        g = gen(n_pages)
        self.buffers = {n: torch.randint(0, 256, shape, generator=g, device="cuda").to(torch.uint8) for n in ("k_codes", "v_codes")}
        self.buffers |= {n: torch.rand(shape[:3] + (page // block,), generator=g, device="cuda") for n in ("k_scale", "v_scale")}
        self.cache = rq.kv_cache(**self.buffers)
        self.d_used, self.d_tables, self.d_lengths = i32(self.used), i32(self.tables), i32(self.lengths)
        self.pages = rq.kv_pages(self.d_used, self.d_tables, self.d_lengths)
        self.ws = rq.workspace(rq.realq_pages_workspace_size(n_pages, n_rows, max_pages))

    def check(self):
        assert self.d_lengths.tolist() == self.lengths
        assert self.d_tables.tolist() == self.tables
        assert self.d_used.tolist() == self.used

    def contents(self):
        return {n: t.clone() for n, t in self.buffers.items()}

    def reserve(self, adds, spare=3):
        """Returns whether there was room; checks everything, the copies of shared pages among it."""
        ps, T = self.page, sum(adds)
        before = self.contents()
        positions = torch.full((T + spare,), 99, dtype=torch.int64, device="cuda")
        rq.realq_pages_reserve(self.pages, starts_of(adds), positions, self.cache, ws=self.ws)
        takes, copies = [], []
        for s, (n, L) in enumerate(zip(adds, self.lengths)):
            first, after = -(-L // ps), -(-(L + n) // ps)
            part = self.tables[s][L // ps] if n and L % ps else -1
            copies.append(part)
            takes.append(after - first if n else 0)
        writers = {p: [s for s in range(self.n_rows) if copies[s] == p] for p in copies if p >= 0}
        for s in range(self.n_rows):
            p = copies[s]
            if p >= 0 and (self.used[p] == 1 or (len(writers[p]) >= self.used[p] and s == writers[p][-1])):
                copies[s] = -1
            takes[s] += copies[s] >= 0
        free = [p for p in range(self.n_pages) if self.used[p] == 0]
        room = sum(takes) <= len(free) and all(-(-(L + n) // ps) <= self.max_pages for n, L in zip(adds, self.lengths) if n)
        want = [-1] * (T + spare)
        moved = {}
        if room:
            at = t = 0
            for s, n in enumerate(adds):
                L = self.lengths[s]
                if n == 0:
                    continue
                if copies[s] >= 0:
                    p = free[at]
                    at += 1
                    moved[p] = copies[s]
                    self.used[copies[s]] -= 1
                    self.used[p] = 1
                    self.tables[s][L // ps] = p
                for j in range(-(-L // ps), -(-(L + n) // ps)):
                    if self.tables[s][j] >= 0:
                        self.used[self.tables[s][j]] -= 1
                    self.tables[s][j] = free[at]
                    self.used[free[at]] = 1
                    at += 1
                want[t:t + n] = range(L, L + n)
                t += n
                self.lengths[s] += n
            rq.realq_workspace_status(self.ws)
        else:
            with pytest.raises(rq.RealqError) as e:
                rq.realq_workspace_status(self.ws)
            assert e.value.status == rq.REALQ_ERR_NO_PAGES
        assert positions.tolist() == want
        for n, t in self.buffers.items():
            for p, q in moved.items():
                before[n][:, p] = before[n][:, q]
            assert torch.equal(t, before[n]), n
        self.check()
        return room

    def fork(self, src, dst):
        rq.realq_pages_fork(self.pages, i32(src), i32(dst), ws=self.ws)
        last = {d: s for s, d in zip(src, dst) if 0 <= d < self.n_rows and 0 <= s < self.n_rows}
        rows, lens = [list(r) for r in self.tables], list(self.lengths)
        for d, s in last.items():
            for p in self.tables[d]:
                if p >= 0:
                    self.used[p] -= 1
            for p in rows[s]:
                if p >= 0:
                    self.used[p] += 1
        for d, s in last.items():
            self.tables[d], self.lengths[d] = list(rows[s]), lens[s]
        self.check()

    def release(self, rows):
        rq.realq_pages_release(self.pages, i32(rows))
        for s in set(r for r in rows if 0 <= r < self.n_rows):
            for p in self.tables[s]:
                if p >= 0:
                    self.used[p] -= 1
            self.tables[s], self.lengths[s] = [-1] * self.max_pages, 0
        self.check()

    def compact(self, in_place):
        before = self.contents()
        live = [p for p in range(self.n_pages) if self.used[p] > 0]
        u = len(live)
        to = dict(zip([p for p in live if p >= u], [p for p in range(u) if self.used[p] == 0]))
        moved_to = i32([7] * self.n_pages)
        uo, to_ = (self.d_used, self.d_tables) if in_place else (torch.empty_like(self.d_used), torch.empty_like(self.d_tables))
        rq.realq_pages_compact(self.pages, self.cache, uo, to_, moved_to, ws=self.ws)
        if not in_place:
            self.check()
            self.d_used.copy_(uo)
            self.d_tables.copy_(to_)
        want = [to.get(p, p) if self.used[p] > 0 else -1 for p in range(self.n_pages)]
        assert moved_to.tolist() == want
        used = [0] * self.n_pages
        for p in live:
            used[want[p]] = self.used[p]
        self.used = used
        self.tables = [[want[p] if p >= 0 else p for p in r] for r in self.tables]
        self.check()
        assert all(n > 0 for n in used[:u]) and not any(used[u:])
        for n, t in self.buffers.items():
            for p, q in to.items():
                before[n][:, q] = before[n][:, p]
            assert torch.equal(t, before[n]), n


@pytest.mark.parametrize("n_pages,n_rows,max_pages,page,kv,D,layers", [(1, 1, 1, 16, 1, 16, 1), (40, 6, 8, 16, 1, 16, 2), (300, 40, 30, 32, 2, 48, 3),
                                                                       (9000, 1500, 20, 16, 1, 16, 1), (64, 3, 20, 256, 3, 80, 2)])
def test_pages_at_random(n_pages, n_rows, max_pages, page, kv, D, layers):
    r = random.Random(n_pages)
    p = Pool(n_pages, n_rows, max_pages, page, kv=kv, D=D, layers=layers)
    for step in range(14):
        what = r.choice(["reserve", "reserve", "fork", "release", "compact", "back"])
        some = lambda: [r.randrange(n_rows) for _ in range(r.randint(0, n_rows))]   # noqa: E731
        if what == "reserve":
            most = r.choice([1, 3, page, 4 * page])
            p.reserve([r.choice([0, 1, 1, r.randint(0, most)]) for _ in range(n_rows)])
        elif what == "fork":
            dst = some()
            p.fork([r.randrange(n_rows) for _ in dst], dst)
        elif what == "release":
            p.release(some())
        elif what == "compact":
            p.compact(r.random() < 0.5)
        else:   # sequences put back to fewer tokens: rejected drafts
            p.lengths = [n - r.randint(0, min(n, 2 * page)) if r.random() < 0.3 else n for n in p.lengths]
            p.d_lengths.copy_(i32(p.lengths))


def test_reserve_is_all_or_nothing():
    p = Pool(10, 3, 6, 16)
    assert p.reserve([40, 1, 0])            # 3 + 1 pages
    assert not p.reserve([100, 1, 0])       # a row of 6 entries is too short
    assert not p.reserve([16, 0, 96])       # 1 + 6 pages of 6
    assert p.reserve([0, 0, 96])
    assert not p.reserve([16, 0, 0])        # none left
    assert p.reserve([8, 15, 0])            # fits in the partly filled pages
    p.release([2, 2, 5, -1])                # twice, and rows that are not there
    for bad in ([0, 3, 2, 4], [1, 2, 3, 4], [0, 1, 2, 9], [-1, 1, 2, 3]):
        pos = torch.full((4,), 5, dtype=torch.int64, device="cuda")
        rq.realq_pages_reserve(p.pages, i32(bad), pos, p.cache, ws=p.ws)
        assert pos.tolist() == [-1] * 4
        p.check()
        with pytest.raises(rq.RealqError):
            rq.realq_workspace_status(p.ws)
    p.d_lengths[1] = -5                     # a length that cannot be
    pos = torch.empty(1, dtype=torch.int64, device="cuda")
    rq.realq_pages_reserve(p.pages, i32([0, 0, 1, 1]), pos, p.cache, ws=p.ws)
    assert pos.tolist() == [-1]


def test_a_shared_last_page_has_one_writer():
    """Beams that share a partly filled page: every writer but the last holder gets a copy."""
    p = Pool(30, 6, 4, 16)
    p.reserve([20, 5, 0, 0, 0, 0])
    p.fork([0, 0, 0, 1], [2, 3, 4, 5])
    p.reserve([0, 1, 1, 1, 0, 1])           # row 0 and 4 hold on: rows 2 and 3 copy; 1 and 5 share alone: 5 keeps
    assert len({p.tables[s][1] for s in (0, 2, 3)}) == 3 and p.tables[0][1] == p.tables[4][1]
    p.reserve([1, 0, 0, 0, 1, 0])           # the two that were left
    p.fork([2, 0, 1, 1], [0, 2, 1, 3])      # a beam's reordering: two rows change places, one stays, one twice
    p.reserve([1, 1, 1, 1, 1, 1])
    p.fork([0, 9, -1, 1, 2], [1, 2, 2, 8, 1])   # rows that are not there; the last of two entries for row 1 counts
    p.compact(True)


def test_copy_pages():
    p = Pool(20, 1, 1, 64, kv=3, D=48, layers=3, block=16)
    before = p.contents()
    src, dst = [0, 3, 19, 25, 2], [1, 4, 18, 2, -1]
    rq.realq_pages_copy(p.cache, i32(src), i32(dst))
    for n, t in p.buffers.items():
        for a, b in list(zip(src, dst))[:3]:
            before[n][:, b] = before[n][:, a]
        assert torch.equal(t, before[n]), n
    rq.realq_pages_copy(p.cache, i32([]), i32([]))


def test_pages_in_a_graph():
    """Fork and reserve captured once, replayed as sequences grow."""
    p = Pool(200, 4, 20, 16)
    p.reserve([37, 50, 0, 0])
    src, dst, starts = i32([0, 1]), i32([2, 3]), starts_of([1, 1, 1, 1])
    pos = torch.empty(4, dtype=torch.int64, device="cuda")

    def step():
        rq.realq_pages_fork(p.pages, src, dst, ws=p.ws)
        rq.realq_pages_reserve(p.pages, starts, pos, p.cache, ws=p.ws)
    state = [t.clone() for t in (p.d_used, p.d_tables, p.d_lengths)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            step()
    torch.cuda.synchronize()
    for t, s in zip((p.d_used, p.d_tables, p.d_lengths), state):
        t.copy_(s)
    for i in range(20):
        g.replay()
        rows, used = p.d_tables.tolist(), p.d_used.tolist()
        assert p.d_lengths.tolist() == [38 + i, 51 + i, 38 + i, 51 + i]
        assert pos.tolist() == [37 + i, 50 + i, 37 + i, 50 + i]
        held = [e for r in rows for e in r if e >= 0]
        assert all(used[e] == held.count(e) for e in range(200))
        for s in range(4):      # the page that is written is the row's own
            assert used[rows[s][p.d_lengths[s].item() - 1 >> 4]] == 1
    rq.realq_workspace_status(p.ws)


def test_cache_of_many_sequences_lives_through_everything():
    """Tokens appended to sequences that fork, leave and are compacted are read back as they were put, in every layer
    (a scale per token, so that a token's value does not depend on its neighbours)."""
    r = random.Random(5)
    n_rows, layers, kv, D = 9, 2, 2, 32
    p = Pool(120, n_rows, 12, 16, layers=layers, kv=kv, D=D)
    held = [[] for _ in range(n_rows)]      # each row's tokens: layers x kv x D of what has been appended

    def values(x):                          # what a token reads as
        s = (x.double().abs().amax(dim=-1, keepdim=True) / 127).float()   # (in fp32 torch multiplies by 1 / 127 here)
        return torch.round(x / s) * s
    for step in range(25):
        what = r.choice(["grow", "grow", "grow", "fork", "leave", "compact"])
        if what == "grow":
            adds = [r.choice([0, 1, 1, 2, 9]) if len(h) < 150 else 0 for h in held]
            if not sum(adds) or not p.reserve(adds, spare=0):
                continue
            T = sum(adds)
            x = torch.randn(layers, T, kv, D, generator=gen(step), device="cuda")
            pos = torch.tensor([q for n, h in zip(adds, held) for q in range(len(h), len(h) + n)], device="cuda")
            for la in range(layers):
                rq.realq_kv_append(p.cache, la, x[la], -x[la], starts_of(adds), pos, p.d_tables)
            t = 0
            for s, n in enumerate(adds):
                held[s] += [values(x[:, t + i]) for i in range(n)]
                t += n
        elif what == "fork":
            dst = r.sample(range(n_rows), r.randint(1, n_rows))
            src = [r.randrange(n_rows) for _ in dst]
            p.fork(src, dst)
            old = [list(h) for h in held]
            for a, b in zip(src, dst):
                held[b] = list(old[a])
        elif what == "leave":
            rows = r.sample(range(n_rows), 2)
            p.release(rows)
            for s in rows:
                held[s] = []
        else:
            p.compact(r.random() < 0.5)
        counts = [len(h) for h in held]
        if sum(counts) == 0:
            continue
        pos = torch.cat([torch.arange(n) for n in counts]).cuda()
        for la in range(layers):
            k, v = torch.empty(sum(counts), kv, D, device="cuda"), torch.empty(sum(counts), kv, D, device="cuda")
            rq.realq_kv_read(p.cache, la, starts_of(counts), pos, p.d_tables, k, v)
            want = torch.stack([t[la] for h in held for t in h])
            assert torch.equal(k, want) and torch.equal(v, -want)


def test_reserving_more_than_a_million_pages_at_once():
    """Rows that need more than 2^20 pages each: refused where the pool has fewer, whatever is left of it, and given
    what they need where it has them."""
    n, page = 2 ** 21, 16
    codes = [torch.empty(1, n, 1, page, 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = rq.kv_cache(*codes, *(torch.empty(1, n, 1, 1, device="cuda") for _ in range(2)))
    used, tables, lengths = i32([0] * n), torch.full((3, n), -1, dtype=torch.int32, device="cuda"), i32([0] * 3)
    pages = rq.kv_pages(used, tables, lengths)
    ws = rq.workspace(rq.realq_pages_workspace_size(n, 3, n))

    def reserve(need):      # pages of each row, the last but for 3 places
        adds = [max(0, page * k - 3) for k in need]
        before = [t.clone() for t in (used, tables, lengths)]
        pos = torch.full((sum(adds),), 5, dtype=torch.int64, device="cuda")
        rq.realq_pages_reserve(pages, starts_of(adds), pos, cache, ws=ws)
        free = int((before[0] == 0).sum())
        if sum(need) > free:
            with pytest.raises(rq.RealqError) as e:
                rq.realq_workspace_status(ws)
            assert e.value.status == rq.REALQ_ERR_NO_PAGES
            assert bool((pos == -1).all())
            for a, b in zip(before, (used, tables, lengths)):
                assert torch.equal(a, b)
            return False
        rq.realq_workspace_status(ws)
        at = torch.nonzero(before[0] == 0)[:, 0].to(torch.int32)
        want = before[1].clone()
        t = k0 = 0
        for s, k in enumerate(need):
            if k:
                want[s, :k] = at[k0:k0 + k]
                assert torch.equal(pos[t:t + adds[s]], torch.arange(adds[s], device="cuda"))
            k0, t = k0 + k, t + adds[s]
        assert torch.equal(tables, want) and lengths.tolist() == [b + a for b, a in zip(before[2].tolist(), adds)]
        assert torch.equal(used, before[0].index_fill(0, at[:k0].long(), 1))
        return True
    m = 2 ** 20
    assert not reserve([m + 7, m + 7, 0])
    assert not reserve([m + 7, m - 7, 1])
    assert reserve([m - 6, 0, 0])
    assert not reserve([0, m + 20, 0])          # 2^20 + 6 are left
    assert reserve([0, m + 6, 0])
    rq.realq_pages_release(pages, i32([0, 1]))
    assert int(used.sum()) == 0
    assert reserve([m + 5, 0, 3])
