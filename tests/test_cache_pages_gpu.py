"""The cache's page operations against plain Python bookkeeping: pages, counts and tables agree exactly, and what no call names stays."""
import random

import pytest
import torch

from layer_utils import compact_ref, fork_ref, release

pytestmark = pytest.mark.gpu


def gdn():
    import paper_2608_30310_b200 as m
    return m


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Cache:
    """A cache on the device and its double in plain Python: what each page holds is a number."""

    def __init__(self, pages, rows, row_pages, pool_bytes=(64, 48, 4112), page_tokens=16, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.pools = [torch.randint(-100, 100, (pages, b), generator=g, dtype=torch.int8).cuda() for b in pool_bytes]
        self.want = [p.clone() for p in self.pools]
        self.count, self.table, self.page_tokens = [0] * pages, [[-1] * row_pages for _ in range(rows)], page_tokens
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = gdn().Workspace()

    def fill(self, lengths, rng):
        """Rows of these many pages, of random free pages."""
        free = [p for p, c in enumerate(self.count) if c == 0]
        rng.shuffle(free)
        for r, n in enumerate(lengths):
            for j in range(n):
                self.table[r][j] = free.pop()
                self.count[self.table[r][j]] = 1
        self.upload()

    def upload(self):
        self.refcounts, self.tables = ints(self.count), ints(self.table)

    def moved(self, moves):
        for pool in self.want:
            src = pool[[s for s, _ in moves]].clone()
            pool[[d for _, d in moves]] = src

    def agrees(self, status=0):
        torch.cuda.synchronize()
        assert self.refcounts.tolist() == self.count
        assert self.tables.tolist() == self.table
        for got, want in zip(self.pools, self.want):
            assert torch.equal(got, want)
        assert int(self.status) == status, int(self.status)

    def fork(self, parents, children, tokens, status=0):
        moves, bad, short = fork_ref(self.count, self.table, parents, children, tokens, self.page_tokens)
        assert (-7 if bad else -8 if short else 0) == status
        self.moved(moves)
        self.status.zero_()
        gdn().gdn_cache_fork(self.pools, self.page_tokens, self.refcounts, self.tables, ints(parents), ints(children), ints(tokens),
                             workspace=self.ws, status_word=self.status)
        assert gdn().last_launch_count() >= 2
        self.agrees(status)

    def free(self, rows, status=0):
        for r in dict.fromkeys(rows):
            if 0 <= r < len(self.table):
                release(self.count, self.table, r)
        self.status.zero_()
        gdn().gdn_cache_free(self.refcounts, self.tables, ints(rows), status_word=self.status)
        self.agrees(status)

    def compact(self, in_place=True, status=0):
        moves, count, table, to, M = compact_ref(self.count, self.table)
        self.moved(moves)
        self.status.zero_()
        oc, ot = (self.refcounts, self.tables) if in_place else (torch.full_like(self.refcounts, 77), torch.full_like(self.tables, 77))
        page_map, live = torch.full_like(self.refcounts, 77), ints([77])
        gdn().gdn_cache_compact(self.pools, self.refcounts, self.tables, oc, ot, page_map, live, workspace=self.ws, status_word=self.status)
        torch.cuda.synchronize()
        assert page_map.tolist() == to and live.tolist() == [M]
        if not in_place:
            assert self.refcounts.tolist() == self.count and self.tables.tolist() == self.table
        self.count, self.table, self.refcounts, self.tables = count, table, oc, ot
        self.agrees(status)
        return M


@pytest.mark.parametrize("bytes_", [(16,), (64, 48, 4096), (4112, 8192 + 16, 3 * 4096), tuple(16 * (i + 1) for i in range(150))], ids=lambda b: "%d pools" % len(b))
@pytest.mark.parametrize("n", [1, 2, 37])
def test_copy(bytes_, n):
    c = Cache(100, 1, 1, bytes_)
    ids = random.Random(n).sample(range(100), 2 * n)
    c.moved(list(zip(ids[:n], ids[n:])))
    gdn().gdn_cache_copy(c.pools, ints(ids[:n]), ints(ids[n:]))
    assert gdn().last_launch_count() == -(-len(bytes_) // 64)
    c.upload()
    c.agrees()


def test_copy_of_one_page_to_many_and_bad_pairs():
    c = Cache(40, 1, 1)
    src, dst = [3, 3, 3, 40, -1, 5, 6], [7, 8, 9, 10, 11, 40, -1]
    c.moved([(3, 7), (3, 8), (3, 9)])
    gdn().gdn_cache_copy(c.pools, ints(src), ints(dst), status_word=c.status)
    c.upload()
    c.agrees(-7)
    gdn().gdn_cache_copy(c.pools, ints([]), ints([]))
    c.agrees(-7)


@pytest.mark.parametrize("page_tokens", [1, 7, 16])
@pytest.mark.parametrize("pages,parents,children,row", [(8, 1, 1, 3), (300, 3, 20, 40), (9000, 5, 60, 700), (3000, 2, 1500, 9)])
def test_fork(page_tokens, pages, parents, children, row):
    rng = random.Random(pages + page_tokens)
    rows = list(range(parents + children + 1))
    c = Cache(pages, len(rows), row, page_tokens=page_tokens, pool_bytes=(64, 80) if pages > 1000 else (64, 48, 4112))
    c.fill([rng.randint(row // 2, row) for _ in range(parents)] + [0] * (children + 1), rng)
    held = [sum(e >= 0 for e in r) * page_tokens for r in c.table]
    who = [rng.randrange(parents) for _ in range(children)]
    kids = rows[parents:parents + children]
    rng.shuffle(kids)
    tokens = [rng.choice([0, 1, held[p], rng.randint(0, held[p]), held[p] - 1]) for p in who]
    c.fork(who, kids, tokens)
    # again: the children give back what they hold, and take from other parents, some from a child that stays
    stay, again = kids[0], kids[1:]
    who = [rng.choice(list(range(parents)) + [stay]) for _ in again]
    held = [sum(e >= 0 for e in r) * page_tokens for r in c.table]
    if again:
        c.fork(who, again, [rng.randint(0, held[p]) for p in who])
    c.free([rng.choice(rows) for _ in range(children + 3)])
    c.compact(in_place=bool(pages % 2))
    c.free(rows)
    assert not any(c.count)


def test_fork_leaves_out_what_is_wrong():
    rng = random.Random(1)
    c = Cache(60, 12, 6)
    c.fill([6, 3, 2] + [0] * 9, rng)
    c.table[9] = c.table[0][:2] + [-1] * 4                                  # a child that holds pages already
    for p in c.table[9][:2]:
        c.count[p] += 1
    c.table[8][:2] = [60, 2]                                                # a parent whose table is broken
    c.upload()
    #            good  same child twice  onto itself  no such rows      too long  none held  negative  a parent that is a child  broken table
    parents = [0, 1, 1, 2, 12, -1, 0, 0, 1, 0, 9, 8]
    children = [9, 3, 3, 2, 4, 5, -2, 6, 7, 10, 11, 1]
    tokens = [37, 5, 9, 4, 4, 4, 4, 97, 70, -3, 4, 20]
    c.fork(parents, children, tokens, status=-7)
    assert c.table[9][:3] != [-1] * 3 and c.table[3] == [-1] * 6


def test_fork_without_pages_for_all():
    c = Cache(8, 6, 3)
    c.fill([3, 2, 0, 0, 0, 0], random.Random(2))                            # three free pages, four forks that want one
    c.fork([0, 0, 1, 0], [2, 3, 4, 5], [33, 40, 17, 35], status=-8)
    assert c.table[5] == [-1] * 3 and all(c.table[r][0] >= 0 for r in (2, 3, 4))
    c.free([2, 3, 4, 5])
    c.fork([0], [2], [33])


def test_children_give_back_before_any_takes():
    """The one page that the fork needs is the one that its child, or another fork's, holds."""
    c = Cache(4, 4, 3)
    c.fill([2, 1, 1, 0], random.Random(3))
    c.fork([0, 0], [2, 1], [17, 5])
    c.fork([0, 0], [1, 2], [30, 3])


def test_free():
    rng = random.Random(4)
    c = Cache(500, 9, 50)
    c.fill([50, 20, 0, 33, 50, 1, 0, 0, 0], rng)
    c.fork([0, 0, 3], [6, 7, 8], [100, 800, 33])
    c.free([0, 0, 2, 5, 0])
    c.free([7, 9, -1, 7], status=-7)
    c.free([])
    c.status.zero_()
    c.table[1][2], before = 600, c.table[1][2]                              # no such page; and one whose count is zero already
    c.count[c.table[1][0]] = 0
    c.upload()
    zero = c.table[1][0]
    gdn().gdn_cache_free(c.refcounts, c.tables, ints([1]), status_word=c.status)
    for j, p in enumerate(c.table[1]):
        if p >= 0 and p < 500 and p != zero:
            c.count[p] -= 1
        c.table[1][j] = -1
    c.agrees(-7)
    assert c.count[before] == 1


@pytest.mark.parametrize("pages,live", [(1, 0), (1, 1), (5, 0), (5, 5), (64, 1), (1000, 300), (1000, 999), (33000, 20000), (70001, 100)])
@pytest.mark.parametrize("in_place", [True, False])
def test_compact(pages, live, in_place):
    rng = random.Random(pages + live)
    width = max(1, -(-live // 7))
    c = Cache(pages, 8, width, (64,) if pages > 2000 else (64, 48, 4112))
    left = live
    lengths = []
    for _ in range(7):
        lengths.append(min(width, left))
        left -= lengths[-1]
    c.fill(lengths + [0], rng)
    if live:
        c.table[7] = list(c.table[0])
        for p in c.table[0]:
            c.count[p] += p >= 0
        c.upload()
    assert c.compact(in_place) == live
    assert c.compact(not in_place) == live                                  # nothing moves any more


def test_compact_names_that_are_not_there():
    c = Cache(30, 3, 5)
    c.fill([5, 4, 0], random.Random(5))
    dead = c.count.index(0)
    c.table[2][:4] = [30, dead, -5, c.table[0][0]]
    c.upload()
    c.compact(status=-7)


def test_many_pools_and_far_pages():
    """150 pools take three launches; offsets in a pool pass 32 bits."""
    rng = random.Random(6)
    c = Cache(20, 5, 4, tuple(16 * (1 + i % 5) for i in range(150)))
    c.fill([4, 3, 0, 0, 0], rng)
    c.fork([0, 1], [2, 3], [50, 40])
    c.free([0])
    c.compact()
    big = torch.zeros((2200, 1 << 20), dtype=torch.int8, device="cuda")
    big[2199], big[1] = 5, 6
    counts, tables = torch.zeros(2200, dtype=torch.int32, device="cuda"), ints([[2199, 1, -1], [-1, -1, -1]])
    counts[2199] = counts[1] = 1
    page_map, live = torch.zeros_like(counts), ints([0])
    gdn().gdn_cache_compact([big], counts, tables, counts, tables, page_map, live)
    torch.cuda.synchronize()
    assert tables.tolist()[0] == [0, 1, -1] and bool((big[0] == 5).all()) and bool((big[1] == 6).all())
    gdn().gdn_cache_copy([big], ints([0]), ints([2198]))
    assert bool((big[2198] == 5).all()) and bool((big[2197] == 0).all()) and bool((big[2199] == 5).all())


def test_captured():
    """A branch made, and given up, in a graph that is replayed; its workspace grows afterwards."""
    rng = random.Random(7)
    c = Cache(200, 8, 20)
    c.fill([20, 11, 0, 0, 0, 0, 0, 0], rng)
    parents, children, tokens = ints([0, 1, 0]), ints([4, 5, 6]), ints([300, 170, 16])
    side = torch.cuda.Stream()

    def call():
        gdn().gdn_cache_fork(c.pools, 16, c.refcounts, c.tables, parents, children, tokens, workspace=c.ws, stream=side)
    torch.cuda.synchronize()
    call()
    side.synchronize()
    moves, _, _ = fork_ref(c.count, c.table, [0, 1, 0], [4, 5, 6], [300, 170, 16], 16)
    c.moved(moves)
    c.agrees()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call()
        gdn().gdn_cache_free(c.refcounts, c.tables, children[:2], stream=side)
    c.ws.ensure(20 << 20, side)
    tokens.copy_(ints([250, 100, 320]))
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        moves, _, _ = fork_ref(c.count, c.table, [0, 1, 0], [4, 5, 6], [250, 100, 320], 16)
        c.moved(moves)
        release(c.count, c.table, 4)
        release(c.count, c.table, 5)
        c.agrees()


@pytest.mark.parametrize("children,row", [(40, 30), (40, 600)])
def test_forks_left_out_among_many(children, row):
    """The same rules where the rows are long, and a kernel of its own gives them back, as where they are short."""
    rng = random.Random(row)
    c = Cache(children * row // 2, children + 8, row, (64,))
    c.fill([row, row // 2, row] + [0] * 5 + [rng.randint(0, row // 8) for _ in range(children)], rng)
    c.table[2][row // 3] = len(c.count) + 5                                 # a broken parent
    c.upload()
    who = [rng.randrange(3) for _ in range(children)]
    kids = list(range(8, 8 + children))
    tokens = [rng.randint(0, row * 16) for _ in range(children)]
    kids[5], kids[6], who[7], who[9], tokens[11], kids[13] = kids[4], 8 + children + 3, kids[1], -1, row * 16 + 1, -7
    c.fork(who, kids, tokens, status=-7)


def test_refused_tensors():
    c = Cache(16, 3, 4)
    c.upload()
    one = ints([1])
    g = gdn()
    for call, name in ((lambda: g.gdn_cache_copy(c.pools, one, ints([1, 2])), "dst"),
                       (lambda: g.gdn_cache_copy([c.pools[0], c.pools[1][:8]], one, one), "pool 1"),
                       (lambda: g.gdn_cache_copy([c.pools[2][:, :64]], one, one), "pool 0"),
                       (lambda: g.gdn_cache_copy([one], one, one), "pages"),
                       (lambda: g.gdn_cache_fork(c.pools, 16, c.refcounts[:8], c.tables, one, one, one), "refcounts"),
                       (lambda: g.gdn_cache_fork(c.pools, 16, c.refcounts, c.tables[:, ::2], one, one, one), "tables"),
                       (lambda: g.gdn_cache_fork(c.pools, 16, c.refcounts, c.tables, one, one, ints([1, 2])), "tokens"),
                       (lambda: g.gdn_cache_free(c.refcounts, c.tables[0], one), "tables"),
                       (lambda: g.gdn_cache_compact(c.pools, c.refcounts, c.tables, c.refcounts, c.tables[:2], c.refcounts, one), "out_tables")):
        with pytest.raises(ValueError, match=name):
            call()
    with pytest.raises(TypeError, match="src"):
        g.gdn_cache_copy(c.pools, one.long(), one)
    with pytest.raises(g.GdnError, match="invalid argument"):
        g.gdn_cache_copy([torch.zeros(16, 24, dtype=torch.int8, device="cuda")], one, one)
    with pytest.raises(g.GdnError, match="invalid argument"):
        g.gdn_cache_fork(c.pools, 0, c.refcounts, c.tables, one, one, one)
    many = [torch.zeros(16, 16, dtype=torch.int8, device="cuda") for _ in range(300)]
    many[7][3] = 5
    g.gdn_cache_copy(many, ints([3]), ints([4]))                            # more pools than the native argument path holds
    assert bool((many[7][4] == 5).all())
