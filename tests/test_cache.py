"""The paged cache (GPU): appending, forking, trimming and compacting against a
model of it that keeps lists, call after call; refusals leave it as it was."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DEV = "cuda:0"


@pytest.fixture(scope="module")
def opa():
    import paper_2609_11938_gb300 as opa
    return opa


@pytest.fixture()
def ctx(opa):
    with opa.Context(0) as c:
        yield c


class Model:
    """The cache's definition, one sequence and one page after another."""

    def __init__(self, n_pages, page, n_seqs, per):
        self.page, self.per = page, per
        self.seqs = [[] for _ in range(n_seqs)]          # pages
        self.length = [0] * n_seqs
        self.refs = [0] * n_pages
        self.slots = [[None] * page for _ in range(n_pages)]

    def take(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def append(self, seqs, counts, rows):
        # pages are chosen before any is let go: none becomes free here
        at = 0
        for s, n in zip(seqs, counts):
            part = self.length[s] % self.page
            if n and part and self.refs[self.seqs[s][-1]] > 1:
                old = self.seqs[s][-1]
                new = self.take()
                self.slots[new][:part] = self.slots[old][:part]
                self.refs[old] -= 1
                self.seqs[s][-1] = new
            for r in rows[at:at + n]:
                if self.length[s] % self.page == 0:
                    self.seqs[s].append(self.take())
                self.slots[self.seqs[s][-1]][self.length[s] % self.page] = r
                self.length[s] += 1
            at += n

    def fork(self, src, dst):
        for a, b in zip(src, dst):
            self.seqs[b], self.length[b] = list(self.seqs[a]), self.length[a]
            for p in self.seqs[a]:
                self.refs[p] += 1

    def trim(self, seqs, lengths):
        for s, n in zip(seqs, lengths):
            keep = -(-n // self.page)
            for p in self.seqs[s][keep:]:
                self.refs[p] -= 1
            self.seqs[s], self.length[s] = self.seqs[s][:keep], n

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [i for i in range(live) if self.refs[i] == 0]
        move = [i for i in range(live, len(self.refs)) if self.refs[i] > 0]
        to = dict(zip(move, holes))
        for a, b in to.items():
            self.slots[b], self.refs[b], self.refs[a] = list(self.slots[a]), self.refs[a], 0
        self.seqs = [[to.get(p, p) for p in s] for s in self.seqs]
        return live


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def same(cache, m):
    """Tables, lengths, counts, and every token that a sequence holds."""
    assert cache.refs.tolist() == m.refs
    assert cache.length.tolist() == m.length
    assert cache.table.tolist() == [s + [-1] * (m.per - len(s)) for s in m.seqs]
    low = int(cache.low)
    assert all(r > 0 for r in m.refs[:low])
    k, v = cache.k_pages.float().cpu(), cache.v_pages.float().cpu()
    for s, n in zip(m.seqs, m.length):
        for i in range(n):
            p, e = s[i // m.page], i % m.page
            want = m.slots[p][e]
            assert (k[p, :, e] == want).all() and (v[p, :, e] == -want).all()


def rows(ids, heads, dim, dtype):
    x = torch.tensor(ids, dtype=torch.float32, device=DEV)[:, None, None].expand(-1, heads, dim).to(dtype)
    return x.contiguous(), (-x).contiguous()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("seed,page,heads,dim", [(0, 16, 1, 8), (1, 16, 3, 64), (2, 32, 2, 40), (3, 128, 1, 128)])
def test_calls_in_any_order(ctx, dtype, seed, page, heads, dim):
    rng = random.Random(seed)
    n_seqs, per, n_pages = 9, 6, 40
    c = ctx.cache(n_pages, page, heads, dim, n_seqs, per, dtype)
    m = Model(n_pages, page, n_seqs, per)
    nxt = 1
    for _ in range(60):
        what = rng.choice(["append", "append", "append", "fork", "trim", "trim", "compact"])
        if what == "append":
            seqs = rng.sample(range(n_seqs), rng.randint(1, n_seqs))
            counts = [min(rng.choice([0, 1, 1, 5, page, 2 * page + 1]), per * page - m.length[s]) for s in seqs]
            need = sum(-(-(m.length[s] + n) // page) + 1 for s, n in zip(seqs, counts))
            if need > m.refs.count(0):
                continue
            ids = [(nxt + i) % 251 + 1 for i in range(sum(counts))]      # exact in either type
            nxt += len(ids)
            k, v = rows(ids, heads, dim, dtype)
            off = [0]
            for n in counts:
                off.append(off[-1] + n)
            ctx.cache_append(c, i32(seqs), i32(off), k, v)
            m.append(seqs, counts, ids)
        elif what == "fork":
            empty = [s for s in range(n_seqs) if m.length[s] == 0]
            full = [s for s in range(n_seqs) if m.length[s] > 0]
            if not empty or not full:
                continue
            dst = rng.sample(empty, rng.randint(1, len(empty)))
            src = [rng.choice(full) for _ in dst]
            ctx.cache_fork(c, i32(src), i32(dst))
            m.fork(src, dst)
        elif what == "trim":
            seqs = rng.sample(range(n_seqs), rng.randint(1, 4))
            to = [rng.choice([0, m.length[s], rng.randint(0, m.length[s])]) for s in seqs]
            if rng.random() < 0.3:
                to = [0] * len(seqs)
                ctx.cache_trim(c, i32(seqs))
            else:
                ctx.cache_trim(c, i32(seqs), i32(to))
            m.trim(seqs, to)
        else:
            _, live = ctx.cache_compact(c)
            assert int(live) == m.compact() and int(c.low) == int(live)
        ctx.check()
        same(c, m)


def test_many_pages(ctx):
    """A pool of several tiles of pages, freed with gaps and compacted, and free
    pages found past long runs of pages in use."""
    page, per, n_seqs, n_pages = 16, 64, 300, 20_001
    c = ctx.cache(n_pages, page, 1, 8, n_seqs, per)
    m = Model(n_pages, page, n_seqs, per)
    rng = random.Random(5)
    counts = [rng.randint(1, per * page) for _ in range(n_seqs)]
    ids = [i % 250 + 1 for i in range(sum(counts))]
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    k, v = rows(ids, 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32(list(range(n_seqs))), i32(off), k, v)
    # by position in the definition's terms (its list walk would be slow here)
    table, nxt = [], 0
    for n in counts:
        p = -(-n // page)
        table.append(list(range(nxt, nxt + p)))
        nxt += p
    assert c.table.tolist() == [t + [-1] * (per - len(t)) for t in table]
    gone = rng.sample(range(n_seqs), 140)
    ctx.cache_trim(c, i32(gone))
    refs = [0] * n_pages
    for s, t in enumerate(table):
        if s not in gone:
            for p in t:
                refs[p] = 1
    assert c.refs.tolist() == refs
    # scattered free pages are taken lowest first
    free = [p for p in range(n_pages) if refs[p] == 0][:per]
    k2, v2 = rows([7] * (per * page), 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32([gone[0]]), i32([0, per * page]), k2, v2)
    assert c.table[gone[0]].tolist() == free
    table[gone[0]], gone = free, gone[1:]
    before = c.k_pages.clone()
    _, live = ctx.cache_compact(c)
    ctx.check()
    held = [s for s in range(n_seqs) if s not in gone]
    old = sorted(p for s in held for p in table[s])
    assert int(live) == len(old)
    holes = sorted(set(range(len(old))) - set(old))
    to = dict(zip([p for p in old if p >= len(old)], holes))
    for s in held:
        want = [to.get(p, p) for p in table[s]]
        assert c.table[s].tolist() == want + [-1] * (per - len(want))
        assert torch.equal(c.k_pages[want], before[table[s]])
    assert c.refs.tolist() == [1] * len(old) + [0] * (n_pages - len(old))


@pytest.mark.parametrize("n_pages", [4096, 4097])
def test_compact_at_a_tile(ctx, n_pages):
    """Pools of one tile of pages and of one page more, full but for a gap, and full."""
    c = ctx.cache(n_pages, 16, 1, 8, 3, 4096)
    counts = [1600, 160, 16 * n_pages - 1760]
    k, v = rows([1] * counts[0] + [2] * counts[1] + [3] * counts[2], 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32([0, 1, 2]), i32([0, 1600, 1760, 16 * n_pages]), k, v)
    _, live = ctx.cache_compact(c)
    ctx.check()
    assert int(live) == n_pages and c.table[1].tolist()[:10] == list(range(100, 110))
    ctx.cache_trim(c, i32([1]))
    _, live = ctx.cache_compact(c)
    ctx.check()
    last = n_pages - 110
    assert int(live) == n_pages - 10
    assert c.table[2].tolist()[:last] == list(range(110, n_pages - 10)) + list(range(100, 110))
    assert (c.k_pages[100:110] == 3).all() and c.refs.tolist() == [1] * (n_pages - 10) + [0] * 10


def test_strided_rows(ctx):
    """Keys and values as parts of one projection."""
    c = ctx.cache(8, 16, 2, 64, 2, 4)
    qkv = torch.arange(20, device=DEV)[:, None].expand(20, 6 * 64).to(torch.bfloat16).contiguous()
    qkv[:, 4 * 64:] *= -1
    k, v = qkv[:, 2 * 64:4 * 64].view(20, 2, 64), qkv[:, 4 * 64:].view(20, 2, 64)
    ctx.cache_append(c, i32([1]), i32([0, 20]), k, v)
    ctx.check()
    assert c.table[1].tolist() == [0, 1, -1, -1]
    assert (c.k_pages[0, :, :, 0].float().cpu() == torch.arange(16.0)).all()
    assert (c.v_pages[1, 1, :4, 63].float().cpu() == -torch.arange(16.0, 20.0)).all()


def snapshot(c):
    return [t.clone() for t in (c.k_pages, c.v_pages, c.table, c.length, c.refs, c.low)]


def test_refusals_change_nothing(opa, ctx):
    c = ctx.cache(6, 16, 1, 8, 4, 3)
    k, v = rows(list(range(1, 41)), 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32([0, 1]), i32([0, 20, 40]), k, v)
    ctx.check()
    before = snapshot(c)

    def refused(status, call, *a):
        call(c, *a)
        with pytest.raises(opa.OpattrError) as e:
            ctx.check()
        assert e.value.status == status
        for x, y in zip(snapshot(c), before):
            assert torch.equal(x, y)
        ctx.check()

    bad = opa.E_INVALID_ARG
    few = lambda n: rows([9] * n, 1, 8, torch.bfloat16)  # noqa: E731
    refused(bad, ctx.cache_append, i32([4]), i32([0, 1]), *few(1))              # no such sequence
    refused(bad, ctx.cache_append, i32([-1]), i32([0, 1]), *few(1))
    refused(bad, ctx.cache_append, i32([2, 2]), i32([0, 1, 2]), *few(2))        # one twice
    refused(bad, ctx.cache_append, i32([2, 3]), i32([0, 2, 1]), *few(1))        # offsets
    refused(bad, ctx.cache_append, i32([2, 3]), i32([0, 1, 1]), *few(2))
    refused(bad, ctx.cache_append, i32([0]), i32([0, 29]), *few(29))            # longer than the table
    refused(opa.E_PAGES, ctx.cache_append, i32([2, 3]), i32([0, 17, 34]), *few(34))   # four pages of two
    refused(bad, ctx.cache_fork, i32([0]), i32([1]))                            # not empty
    refused(bad, ctx.cache_fork, i32([0, 1]), i32([2, 2]))
    refused(bad, ctx.cache_fork, i32([0, 2]), i32([2, 3]))                      # a source that is a destination
    refused(bad, ctx.cache_fork, i32([7]), i32([2]))
    refused(bad, ctx.cache_trim, i32([0]), i32([21]))                           # longer than it is
    refused(bad, ctx.cache_trim, i32([0]), i32([-1]))
    refused(bad, ctx.cache_trim, i32([0, 0]), i32([1, 1]))
    # the last two pages, and then none
    ctx.cache_append(c, i32([2, 3]), i32([0, 16, 32]), *few(32))
    ctx.check()
    assert c.refs.tolist() == [1] * 6
    ctx.cache_fork(c, i32([]), i32([]))
    ctx.cache_trim(c, i32([]))
    ctx.cache_append(c, i32([]), i32([0]), *few(0))
    ctx.check()


def test_shared_page_without_room_for_its_copy(opa, ctx):
    c = ctx.cache(2, 16, 1, 8, 3, 2)
    k, v = rows([1] * 20, 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32([0]), i32([0, 20]), k, v)
    ctx.cache_fork(c, i32([0]), i32([2]))
    ctx.check()
    k1, v1 = rows([2], 1, 8, torch.bfloat16)
    ctx.cache_append(c, i32([2]), i32([0, 1]), k1, v1)
    with pytest.raises(opa.OpattrError) as e:
        ctx.check()
    assert e.value.status == opa.E_PAGES
    assert c.refs.tolist() == [2, 2] and c.length.tolist() == [20, 0, 20]


@pytest.mark.parametrize("page,heads,dim,n", [(16, 1, 8, 5), (128, 3, 128, 40), (64, 2, 40, 2), (16, 1, 8, 2600)])
def test_sharers_of_unlike_lengths(ctx, page, heads, dim, n):
    """Sequences share pages and go on from unlike places in them, all in one call.
    The last one keeps the page and writes over what the others take along."""
    per = 3
    c = ctx.cache(n + 2 * n + 8, page, heads, dim, n, per)
    m = Model(n + 2 * n + 8, page, n, per)
    first = list(range(1, 2 * page))
    k, v = rows(first, heads, dim, torch.bfloat16)
    ctx.cache_append(c, i32([0]), i32([0, len(first)]), k, v)
    m.append([0], [len(first)], first)
    others = list(range(1, n))
    ctx.cache_fork(c, i32([0] * (n - 1)), i32(others))
    m.fork([0] * (n - 1), others)
    lengths = [page + 1 + (page - 2) * (n - 1 - s) // (n - 1) for s in range(n)]      # the last is the shortest
    ctx.cache_trim(c, i32(list(range(n))), i32(lengths))
    m.trim(list(range(n)), lengths)
    counts = [min(page + 3, per * page - x) for x in lengths]
    if n > 1000:
        counts = [1 + s % 3 if s < n - 1 else page + 3 for s in range(n)]
    ids = [i % 251 + 1 for i in range(sum(counts))]
    off = [0]
    for x in counts:
        off.append(off[-1] + x)
    k, v = rows(ids, heads, dim, torch.bfloat16)
    ctx.cache_append(c, i32(list(range(n))), i32(off), k, v)
    m.append(list(range(n)), counts, ids)
    ctx.check()
    assert m.refs[c.table[n - 1].tolist()[1]] == 1
    same(c, m)
