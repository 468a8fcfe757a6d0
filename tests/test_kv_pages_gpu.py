"""The bookkeeping of the cache's pages against the same rules written out on the host, number by number and byte by byte."""
import random

import pytest
import torch

from gpu_util import announce
from paper_2203_05016_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def dev(values, shape=None):
    t = torch.tensor(values, dtype=torch.int32)
    return (t if shape is None else t.view(shape)).to(DEV)


class Book:
    """The rules: tables, lengths and uses as lists, pages' contents as one tag each."""

    def __init__(self, pages, page, width, rows, uses=None):
        self.pages, self.page, self.width = pages, page, width
        self.rows, self.lengths = [list(r) for r, _ in rows], [n for _, n in rows]
        self.uses = [0] * pages if uses is None else list(uses)
        if uses is None:
            for b, r in enumerate(self.rows):
                for p in r[:self.held(self.lengths[b])]:
                    if 0 <= p < pages:
                        self.uses[p] += 1
        self.copies = []

    def held(self, n):
        return min(self.width, -(-max(n, 0) // self.page))

    def table(self):
        return [r + [-1] * (self.width - len(r)) for r in self.rows]

    def take(self):
        free = [p for p in range(self.pages) if self.uses[p] == 0]
        if not free:
            return -1
        self.uses[free[0]] = 1
        return free[0]

    def extend(self, counts, tokens):
        slots, starts = [], [0]
        for b, c in enumerate(counts):
            n, c = max(self.lengths[b], 0), max(c, 0)
            row = self.rows[b][:self.held(n)]
            row += [self.take() for _ in range(self.held(n + c) - len(row))]
            self.rows[b], self.lengths[b] = row, min(n + c, 2 ** 31 - 1)
            starts.append(min(starts[-1] + c, 2 ** 31 - 1))
            for at in range(n, n + min(c, tokens)):
                p = row[at // self.page] if at // self.page < len(row) else -1
                slots.append(p * self.page + at % self.page if 0 <= p < self.pages else -1)
        return (slots + [-1] * tokens)[:tokens], starts

    def fork(self, parents):
        old = [r[:self.held(n)] for r, n in zip(self.rows, self.lengths)]
        for r in old:
            for p in r:
                if 0 <= p < self.pages:
                    self.uses[p] -= 1
        rows, lengths, seen, wanting = [], [], set(), []
        for i, b in enumerate(parents):
            if not 0 <= b < len(old):
                rows.append([])
                lengths.append(0)
                continue
            n = max(self.lengths[b], 0)
            rows.append(list(old[b]))
            lengths.append(n)
            at = n // self.page
            named = list(old[b])
            if b in seen and n % self.page and at < self.width and 0 <= old[b][at] < self.pages:
                wanting.append((i, at))
                named[at] = -1
            seen.add(b)
            for p in named:
                if 0 <= p < self.pages:
                    self.uses[p] += 1
        for i, at in wanting:
            p = self.take()
            if p >= 0:
                self.copies.append((rows[i][at], p))
            rows[i][at] = p
        self.rows, self.lengths = rows, lengths

    def compact(self):
        live = [p for p in range(self.pages) if self.uses[p]]
        n = len(live)
        holes = [p for p in range(n) if not self.uses[p]]
        moves = dict(zip([p for p in live if p >= n], holes))
        for p, to in moves.items():
            self.copies.append((p, to))
            self.uses[to], self.uses[p] = self.uses[p], 0
        self.rows = [[moves.get(p, p) for p in r] for r in self.table()]


def cache_of(pages, page=32, heads=1, D=64, seed=0):
    c = binding.KVCache(pages, page, heads, D, torch.float16, DEV)
    g = torch.Generator().manual_seed(seed)
    c.data.copy_(torch.randint(0, 256, tuple(c.data.shape), generator=g, dtype=torch.uint8))
    return c


def strided(values, width, ld):
    """A table in memory of another pitch, whose filling must stay."""
    t = torch.full((max(len(values), 1), ld), 77, dtype=torch.int32)
    for b, r in enumerate(values):
        t[b, :width] = torch.tensor(r, dtype=torch.int32)
    return t.to(DEV)[:len(values), :width]


def moved(data, copies):
    want = data.clone()
    for source, to in copies:
        want[to] = data[source]
    return want


def book_of(rng, pages, page, width, rows, fill=0.5, shared=True):
    """Random sequences that name distinct pages, or share full ones."""
    free = list(range(pages))
    rng.shuffle(free)
    out = []
    for _ in range(rows):
        n = rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, width * page), width * page])
        need = -(-n // page)
        row = []
        if shared and out and rng.random() < 0.5:
            r, m = rng.choice(out)
            row = r[:min(m // page, n // page)]
        take = need - len(row)
        if take > len(free) * fill:
            n, take = len(row) * page, 0
        row = row + [free.pop() for _ in range(take)]
        out.append((row, n))
    return Book(pages, page, width, out)


@pytest.mark.parametrize("pages,page,width,rows", [(1, 32, 1, 1), (40, 32, 5, 9), (300, 64, 7, 33), (4097, 32, 40, 130), (9000, 128, 3, 1500),
                                                   (16385, 32, 4, 60), (16384, 32, 30, 1100), (20000, 64, 2, 2500)])
@pytest.mark.parametrize("seed", [0, 1])
def test_extend(pages, page, width, rows, seed):
    announce("extend", pages, page, width, rows, seed)
    rng = random.Random("%d %d %d" % (pages, rows, seed))
    c, book = cache_of(pages, page), book_of(rng, pages, page, width, rows)
    before = c.data.clone()
    for ld, in_place in ((width, False), (width + 3, True)):
        counts = [rng.choice([0, 1, 1, page, -3, rng.randint(0, 3 * page)]) for _ in range(rows)]
        tokens = max(0, sum(max(x, 0) for x in counts) + rng.choice([-5, 0, 7]))
        table, lengths, uses = strided(book.table(), width, ld), dev(book.lengths), dev(book.uses)
        slots, starts = book.extend(counts, tokens)
        got = c.extend(table, lengths, uses, dev(counts), tokens, out=(table, lengths, uses) if in_place else None)
        assert [x.shape for x in got] == [(rows, width), (rows,), (pages,), (tokens,), (rows + 1,)]
        assert got[0].tolist() == book.table() and got[1].tolist() == book.lengths and got[2].tolist() == book.uses
        assert got[3].tolist() == slots and got[4].tolist() == starts
        if in_place:
            assert got[0] is table and (table._base.view(rows, ld)[:, width:] == 77).all()
    assert torch.equal(c.data, before)


def test_extend_at_the_end_of_things():
    """No page left, a row that is full, numbers that 32 bits do not hold, entries that name no page, no sequence at all."""
    announce("extend limits")
    c = cache_of(3)
    book = Book(3, 32, 4, [([2], 32), ([], 0), ([-1, 99], 40), ([], 2 ** 31 - 2)])
    counts = [40, 200, 5, 7]
    want = Book(3, 32, 4, [([2], 32), ([], 0), ([-1, 99], 40), ([], 2 ** 31 - 2)])
    want.rows[3] = [-1] * 4                                        # held, but by no page
    book.rows[3] = [-1] * 4
    slots, starts = want.extend(counts, 260)
    got = c.extend(dev(book.table()), dev(book.lengths), dev(book.uses), dev(counts), 260)
    assert got[0].tolist() == want.table() and got[1].tolist() == want.lengths and got[2].tolist() == want.uses
    assert got[3].tolist() == slots and got[4].tolist() == starts and want.lengths[3] == 2 ** 31 - 1
    many = [2 ** 31 - 1, 2 ** 31 - 1, 1]
    book = Book(3, 32, 2, [([], 0)] * 3)
    got = c.extend(dev(book.table()), dev(book.lengths), dev(book.uses), dev(many), 70)
    slots, starts = book.extend(many, 70)
    assert got[0].tolist() == book.table() and got[3].tolist() == slots and got[4].tolist() == starts == [0] + [2 ** 31 - 1] * 3
    empty = torch.zeros(0, 2, dtype=torch.int32, device=DEV)
    got = c.extend(empty, dev([]), dev([0, 1, 0]), dev([]), 3)
    assert got[2].tolist() == [0, 1, 0] and got[3].tolist() == [-1] * 3 and got[4].tolist() == [0]


@pytest.mark.parametrize("pages,page,width,rows,children,heads,D", [(1, 32, 1, 1, 1, 1, 64), (40, 32, 5, 9, 12, 3, 96), (300, 64, 7, 33, 20, 5, 128),
                                                                    (4097, 32, 40, 130, 257, 1, 64), (9000, 32, 3, 1500, 1400, 1, 64),
                                                                    (16385, 32, 4, 60, 70, 1, 64), (16384, 32, 30, 700, 800, 1, 64), (9000, 32, 2, 2500, 2049, 1, 64)])
@pytest.mark.parametrize("seed", [0, 1])
def test_fork(pages, page, width, rows, children, heads, D, seed):
    announce("fork", pages, page, width, rows, children, seed)
    rng = random.Random("%d %d %d" % (pages, rows, seed))
    c, book = cache_of(pages, page, heads, D), book_of(rng, pages, page, width, rows)
    for ld, same_uses in ((width, False), (width + 5, True)):
        parents = [rng.choice([rng.randrange(rows), rng.randrange(rows), 0, -1, rows]) for _ in range(children)]
        table, lengths, uses = strided(book.table(), width, ld), dev(book.lengths), dev(book.uses)
        before, old = c.data.clone(), table.clone()
        out = None
        if same_uses:
            out = (strided([[5] * width] * children, width, ld), torch.empty(children, dtype=torch.int32, device=DEV), uses)
        book.copies = []
        book.fork(parents)
        got = c.fork(table, lengths, uses, dev(parents), out=out)
        assert got[0].tolist() == book.table() and got[1].tolist() == book.lengths and got[2].tolist() == book.uses
        assert torch.equal(c.data, moved(before, book.copies)) and torch.equal(table, old)
        if same_uses:
            assert (got[0]._base.view(children, ld)[:, width:] == 77).all()
        rows, children = children, rows


def test_fork_at_the_end_of_things():
    announce("fork limits")
    c = cache_of(3)
    # one page left for two that want one; another table's page stays; entries that name no page, lengths past the table
    book = Book(3, 32, 3, [([0], 20), ([99, -4], 40), ([], -5), ([-1, -1, -1], 1000)], uses=[1, 1, 0])
    before = c.data.clone()
    parents = [0, 0, 0, 1, 1, 2, 3, 3]
    args = dev(book.table()), dev(book.lengths), dev(book.uses)
    book.fork(parents)
    got = c.fork(*args, dev(parents))
    assert got[0].tolist() == book.table() and got[1].tolist() == book.lengths and got[2].tolist() == book.uses
    assert got[0][2, 0] == -1 and torch.equal(c.data, moved(before, book.copies))
    # given up as a whole: free at once, and taken by nobody
    got = c.fork(*args, dev([]))
    assert got[0].shape == (0, 3) and got[2].tolist() == [0, 1, 0]
    got = c.fork(torch.zeros(0, 3, dtype=torch.int32, device=DEV), dev([]), dev([0, 1, 0]), dev([0, -1]))
    assert got[0].tolist() == [[-1] * 3] * 2 and got[1].tolist() == [0, 0] and got[2].tolist() == [0, 1, 0]
    # a page that is given up by this very call is taken by its copies
    book = Book(2, 32, 1, [([0], 9), ([1], 3)])
    before = c2 = cache_of(2)
    before, args = c2.data.clone(), (dev(book.table()), dev(book.lengths), dev(book.uses))
    book.fork([0, 0])
    got = c2.fork(*args, dev([0, 0]))
    assert got[0].tolist() == book.table() == [[0], [1]] and got[2].tolist() == [1, 1] and torch.equal(c2.data[1], before[0])


@pytest.mark.parametrize("pages,page,width,rows,heads,D", [(1, 32, 1, 1, 1, 64), (40, 32, 5, 9, 3, 96), (300, 64, 7, 33, 5, 128), (4096, 32, 40, 130, 1, 64), (16384, 32, 3, 5, 1, 64), (20481, 32, 40, 900, 1, 64),
                                                           (9001, 32, 6, 1500, 2, 64)])
@pytest.mark.parametrize("share", [0.0, 0.1, 0.6, 1.0])
def test_compact(pages, page, width, rows, heads, D, share):
    announce("compact", pages, page, width, rows, share)
    rng = random.Random("%d %d %f" % (pages, rows, share))
    c = cache_of(pages, page, heads, D)
    named = rng.sample(range(pages), int(pages * share))
    table = [[rng.choice(named + [-1, pages, 2 ** 31 - 1]) for _ in range(width)] for _ in range(rows)]
    uses = [0] * pages
    for p in named:
        uses[p] = rng.choice([1, 2, 1000000])
    for ld, in_place in ((width, False), (width + 3, True)):
        book = Book(pages, page, width, [(r, 0) for r in table], uses)
        t, u, before = strided(table, width, ld), dev(uses), c.data.clone()
        got = c.compact(t, u, out=(t, u) if in_place else None)
        book.compact()
        assert got[0].tolist() == book.rows and got[1].tolist() == book.uses
        assert torch.equal(c.data, moved(before, book.copies))
        if in_place:
            assert (t._base.view(rows, ld)[:, width:] == 77).all()


def test_pages_past_four_gigabytes():
    announce("pages, far")
    c = binding.KVCache(40000, 64, 16, 128, torch.float16, DEV)     # 5.6 GB
    g = torch.Generator().manual_seed(5)
    some = torch.randint(0, 256, (3, c.data.shape[1]), generator=g, dtype=torch.uint8).to(DEV)
    for i, p in enumerate((39999, 39998, 35001)):
        c.data[p].copy_(some[i])
    uses = torch.zeros(40000, dtype=torch.int32, device=DEV)
    uses[[39999, 39998, 35001]] = 1
    uses[:35000] = 3                                                # other tables' pages
    table, lengths = dev([[39999, 39998], [35001, -1]]), dev([100, 64])
    got = c.fork(table, lengths, uses, dev([0, 0, 1]))
    assert got[0].tolist() == [[39999, 39998], [39999, 35000], [35001, -1]] and torch.equal(c.data[35000], some[1])
    small, now = c.compact(got[0], got[2])
    assert small.tolist() == [[35003, 35002], [35003, 35000], [35001, -1]]
    assert torch.equal(c.data[35003], some[0]) and torch.equal(c.data[35002], some[1]) and torch.equal(c.data[35001], some[2])
    assert now[35000:35005].tolist() == [1, 1, 1, 2, 0] and int((now > 0).sum()) == 35004


def test_page_that_no_count_knows_stays():
    announce("compact stale")
    c = cache_of(8)
    got = c.compact(dev([[7, 3]]), dev([0, 0, 0, 2, 0, 0, 0, 0]))          # 7 is named, but by no count
    assert got[0].tolist() == [[7, 0]] and got[1].tolist() == [2] + [0] * 7


def test_graph():
    """A step that hands out pages, captured and replayed: in place, against the rules at every replay."""
    announce("pages graph")
    c = cache_of(50)
    book = Book(50, 32, 6, [([3, 9], 40), ([], 0), ([11], 31)])
    table, lengths, uses, counts = dev(book.table()), dev(book.lengths), dev(book.uses), dev([1, 1, 1])
    parents = dev([0, 1, 2])
    held = (table, lengths, uses)
    def step():
        new = c.fork(*held, parents)
        for a, b in zip(held, new):
            a.copy_(b)
        c.extend(*held, counts, 40, out=held, slots=slots, starts=starts)
    slots, starts = torch.zeros(40, dtype=torch.int32, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    keep = [x.clone() for x in held]
    step()                                                          # warm
    for a, b in zip(held, keep):
        a.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    data = c.data.clone()
    for i in range(6):
        who, n = [[0, 0, 2], [0, 1, 1], [2, 1, 0], [0, 1, 2], [1, 1, 1], [2, -1, 0]][i], [i, 1, 7 * i]
        parents.copy_(dev(who))
        counts.copy_(dev(n))
        graph.replay()
        torch.cuda.synchronize()
        book.copies = []
        book.fork(who)
        data = moved(data, book.copies)
        want = book.extend(n, 40)
        assert table.tolist() == book.table() and lengths.tolist() == book.lengths and uses.tolist() == book.uses
        assert slots.tolist() == want[0] and starts.tolist() == want[1] and torch.equal(c.data, data)


def test_streams():
    announce("pages streams")
    c, side = cache_of(64), torch.cuda.Stream()
    book = Book(64, 32, 4, [([5, 8], 50), ([60], 10)])
    args = dev(book.table()), dev(book.lengths), dev(book.uses)
    torch.cuda.synchronize()
    got = c.fork(*args, dev([0, 0, 1]), stream=side)
    again = c.extend(*got, dev([30, 30, 30]), 90, stream=side)
    last = c.compact(again[0], again[2], stream=side)
    side.synchronize()
    book.fork([0, 0, 1])
    book.extend([30, 30, 30], 90)
    assert again[0].tolist() == book.table()
    book.compact()
    assert last[0].tolist() == book.rows and last[1].tolist() == book.uses
