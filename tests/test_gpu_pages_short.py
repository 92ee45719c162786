"""Pools that run out while requests share a half-filled block and hold different numbers of its rows (forks that were cut): what a request
kept stays its own, whatever the others are allowed to write."""
import random

import pytest

from tests.test_gpu_pages import pool, update

pytestmark = pytest.mark.gpu


def kept_rows(lens, parent, new_lens, cap):
    B = len(lens)
    p = [b if parent is None else parent[b] for b in range(B)]
    want = [min(max(n, 0), cap) if 0 <= x < B else 0 for x, n in zip(p, new_lens)]
    return [min(lens[x], w) if 0 <= x < B else 0 for x, w in zip(p, want)], want


def check_rows(table, lens, parent, new_lens, got, page, cap, held):
    """Every row of the pool is a name; the copies are carried out, then every request writes the rows that it was granted.  What it kept of
    its parent has to be there before and after, what it wrote too, and held blocks as they were.  -> some request got fewer rows"""
    out, out_lens, copies, full = got
    B = len(lens)
    mem = {}
    at = lambda t, b, i: (t[b][i // page], i % page)  # noqa: E731
    kept, want = kept_rows(lens, parent, new_lens, cap)
    read = lambda cell: mem.get(cell, ("old",) + cell)  # noqa: E731
    mine = [[("old",) + at(table, b if parent is None else parent[b], i) for i in range(kept[b])] for b in range(B)]
    taken = {}
    for a, b, m in copies:
        taken.update({(b, r): read((a, r)) for r in range(m)})
    mem.update(taken)
    for b in range(B):
        assert kept[b] <= out_lens[b] <= want[b], b
        assert [read(at(out, b, i)) for i in range(kept[b])] == mine[b], b
        assert all(e >= 0 for e in out[b][:-(-out_lens[b] // page)]) and all(e == -1 for e in out[b][-(-out_lens[b] // page):]), b
    for b in range(B):
        for i in range(kept[b], out_lens[b]):
            mem[at(out, b, i)] = ("new", b, i)
            mine[b].append(("new", b, i))
    for b in range(B):
        assert [read(at(out, b, i)) for i in range(out_lens[b])] == mine[b], (b, kept, out_lens)
    assert not any(held and held[x] for x, _ in mem)
    short = out_lens != want
    assert full or not short
    return short


@pytest.mark.parametrize("lens", [[5, 9], [9, 5], [5, 9, 9, 2]])
def test_the_request_with_the_most_rows_of_a_shared_block_keeps_it(lens):
    """One block, nothing free, all want to grow: one does, the others keep what they have."""
    page, cap, B = 16, 32, len(lens)
    c = pool(B, page, cap, 1, 1)
    table, grown = [[0, -1]] * B, [n + 1 for n in lens]
    got = update(c, table, lens, list(range(B)), grown, None)
    assert check_rows(table, lens, None, grown, got, page, cap, None)
    most = lens.index(max(lens))
    assert got[1] == [n + (b == most) for b, n in enumerate(lens)] and got[3]
    assert got[0] == table and got[2] == [[-1, -1, 0]] * B
    c.ctx.close()


def test_with_blocks_left_the_shorter_ones_are_copied():
    page, cap = 16, 32
    c = pool(3, page, cap, 8, 1)
    table, lens, grown = [[4, -1]] * 3, [5, 9, 9], [7, 10, 30]
    got = update(c, table, lens, None, grown, None)
    assert got == ([[0, -1], [4, -1], [1, 2]], grown, [[4, 0, 5], [-1, -1, 0], [4, 1, 9]], False)
    assert not check_rows(table, lens, None, grown, got, page, cap, None)
    c.ctx.close()


@pytest.mark.parametrize("page", [2, 16, 64])
@pytest.mark.parametrize("seed", [0, 1, 2, 3])
def test_kept_rows_outlive_a_pool_that_runs_out(page, seed):
    """Steps of cut forks and of growth over a pool of few blocks, some of them held."""
    r = random.Random(1000 * page + seed)
    B, cap = 8, 4 * page
    n_blocks = 9
    c = pool(B, page, cap, n_blocks, seed)
    table, lens = [[-1] * 4 for _ in range(B)], [0] * B
    held = [0] * n_blocks
    if seed % 2:
        held[r.randrange(n_blocks)] = 1
    short = 0
    for step in range(40):
        parent, new_lens = list(range(B)), [n + r.choice([0, 1, 1, 2]) for n in lens]
        if step % 4 == 0:                                         # one is continued by others, cut somewhere
            p = max(range(B), key=lambda b: (lens[b], r.random()))
            for b in r.sample([x for x in range(B) if x != p], r.randint(2, 6)):
                parent[b], new_lens[b] = p, r.randint(max(0, lens[p] - page), lens[p])
            if step == 0:
                new_lens[p] = 2 * page - 1
        got = update(c, table, lens, parent, new_lens, held)
        short += check_rows(table, lens, parent, new_lens, got, page, cap, held)
        table, lens = got[0], got[1]
    assert short > 3
    c.ctx.close()


def test_many_requests_over_one_block_of_the_largest_page():
    """65535 rows in a block and the ranks of 300 requests beside them; the one with the most rows comes late."""
    page, B = 65536, 300
    c = pool(B, page, page, 1, 2, Hkv=1)
    lens = [65000 + b % 7 for b in range(B)]
    lens[271] = lens[299] = page - 1
    got = update(c, [[0]] * B, lens, None, [page] * B, None)
    assert got[1] == [page if b == 271 else n for b, n in enumerate(lens)] and got[3] and got[0] == [[0]] * B
    c.ctx.close()
