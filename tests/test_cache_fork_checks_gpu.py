"""Forks whose parents name free pages, in each form of the call, and forks at the documented limits."""
import random

import pytest
import torch

from layer_utils import fork_ref
from test_cache_pages_gpu import Cache, gdn, ints

pytestmark = pytest.mark.gpu

# rows' entries and forks: one planning kernel; a CTA that gives back for each fork; a cluster for each
FORMS = [(12, 5), (600, 40), (5000, 6)]


def call(c, parents, children, tokens, left_out, status):
    """The forks but for those of ``left_out`` by the reference, all of them by the call."""
    keep = [i for i in range(len(parents)) if i not in left_out]
    moves, bad, short = fork_ref(c.count, c.table, *([v[i] for i in keep] for v in (parents, children, tokens)), c.page_tokens)
    assert not bad and not short
    c.moved(moves)
    c.status.zero_()
    gdn().gdn_cache_fork(c.pools, c.page_tokens, c.refcounts, c.tables, ints(parents), ints(children), ints(tokens), workspace=c.ws, status_word=c.status)
    c.agrees(status)


@pytest.mark.parametrize("row,forks", FORMS)
@pytest.mark.parametrize("where", ["first", "middle", "last whole", "partial", "behind"])
def test_a_parent_that_names_a_free_page(row, forks, where):
    """The page is the lowest free one, which the next fork that needs one takes; behind the forks' tokens it does not matter."""
    rng = random.Random(row)
    c = Cache(4 * row + 300, 2 + forks, row, (64, 48))
    c.fill([row, row] + [row // 20] * forks, rng)
    tokens = [(row - 2) * 16 + 5] * forks                                    # pages 0 to row - 3 whole, row - 2 in part
    at = {"first": 0, "middle": row // 2, "last whole": row - 3, "partial": row - 2, "behind": row - 1}[where]
    held = c.table[0][at]
    c.count[held] = 0
    free = c.count.index(0)
    c.table[0][at] = free
    c.upload()
    parents = [i % 2 for i in range(forks)]
    children = list(range(2, 2 + forks))
    out = set() if where == "behind" else {i for i in range(forks) if parents[i] == 0}
    if where == "behind":
        # (the reference gives pages by count alone, too)
        call(c, parents, children, tokens, out, 0)
        return
    before = [list(c.table[children[i]]) for i in out]
    call(c, parents, children, tokens, out, -7)
    assert [c.table[children[i]] for i in out] == before


@pytest.mark.parametrize("row,forks", FORMS)
def test_a_parents_own_hold_is_enough(row, forks):
    """Children that share the parent's pages give theirs back while the parent's row is checked: its pages stay held."""
    c = Cache(2 * row + forks + 10, 1 + forks, row, (64,))
    c.fill([row] + [0] * forks, random.Random(3))
    kids = list(range(1, 1 + forks))
    for tokens in ([row * 16] * forks, [row * 16 - 3] * forks, [0] * forks):
        call(c, [0] * forks, kids, tokens, set(), 0)
        assert all(c.count[p] >= 1 for p in c.table[0])


@pytest.mark.parametrize("row", [4, 5])
def test_forks_at_the_limits(row):
    """4,096 forks of 262,144 rows: in one planning kernel (4 entries a row), and with the giving back in a kernel of its own (5)."""
    rng = random.Random(row)
    rows, forks, parents = 262144, 4096, 700
    c = Cache(14000, rows, row, (16,))
    c.fill([rng.randint(1, row) for _ in range(parents)], rng)
    held = [sum(e >= 0 for e in c.table[r]) * 16 for r in range(parents)]
    children = rng.sample(range(rows - 2 * forks, rows), forks)
    children[0] = rows - 1 if rows - 1 not in children else children[0]
    for _ in range(2):
        who = [rng.randrange(parents) for _ in range(forks)]
        call(c, who, children, [rng.randint(0, held[p]) for p in who], set(), 0)
