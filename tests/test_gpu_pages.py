"""Pages: forks, growth, ends, compaction and the copies they ask for, against a bookkeeping written out in Python."""
import random

import pytest
import torch

from tests.cache_case import CacheCase, ints, raw
from tests.harness import DEV

pytestmark = pytest.mark.gpu


def plan(table, lens, parent, new_lens, held, n_blocks, page, cap):
    """The rules of lfps_pages_update, one request after the other.  -> (table, lens, copies, ran out)"""
    B, per = len(table), len(table[0])
    clip = lambda e: min(max(e, 0), n_blocks - 1)  # noqa: E731
    blocks = lambda rows: -(-rows // page)  # noqa: E731
    lens = [min(max(n, 0), cap) for n in lens]
    live = {clip(table[b][j]) for b in range(B) for j in range(blocks(lens[b]))} | {x for x in range(n_blocks) if held and held[x]}
    free = [x for x in range(n_blocks) if x not in live]
    keep, want = [], []
    for b in range(B):
        p = b if parent is None else parent[b]
        if not 0 <= p < B:
            keep.append([]), want.append((0, 0))
            continue
        length = min(max(new_lens[b], 0), cap)
        rows = min(lens[p], length)
        keep.append([clip(table[p][j]) for j in range(blocks(rows))])
        want.append((rows, length))
    writes = [w[1] > w[0] and w[0] % page != 0 for w in want]
    out, out_lens, copies, short, taken = [], [], [], False, 0
    for b in range(B):
        rows, length = want[b]
        mine, copy = list(keep[b]), [-1, -1, 0]
        needs_copy = False
        if writes[b]:
            x = mine[-1]
            writers = [i for i in range(B) if writes[i] and keep[i][-1] == x]
            others = sum(k.count(x) for k in keep) > len(writers)
            needs_copy = others or writers[0] != b or bool(held and held[x])
        need = int(needs_copy) + blocks(length) - len(mine)
        got = free[taken:taken + need]
        taken += need
        if len(got) < need:
            short = True
        if needs_copy and not got:
            length = rows
        else:
            if needs_copy:
                copy = [mine[-1], got[0], rows % page]
                mine[-1] = got[0]
                got = got[1:]
            mine += got
            length = min(length, len(mine) * page)
        out.append(mine + [-1] * (per - len(mine)))
        out_lens.append(length)
        copies.append(copy)
    return out, out_lens, copies, short


def pool(B, page, cap, n_blocks, seed, dtype="bf16", Hkv=2):
    c = CacheCase(dtype, Hkv, Hkv, [0] * B, page, cap=cap, spare=0, seed=seed)
    c.n_blocks = n_blocks
    shape = (n_blocks, Hkv, page, 128)
    c.K = c.randn(*shape).clamp(-448, 448).to(c.kd)
    c.V = c.randn(*shape).clamp(-448, 448).to(c.vd)
    return c


def update(c, table, lens, parent, new_lens, held):
    c.table, c.seq = ints(table), ints(lens)
    c.view()
    out, out_lens, copies = torch.zeros_like(c.table), torch.zeros_like(c.seq), torch.zeros((c.B, 3), dtype=torch.int32, device=DEV)
    work = c.ctx.pages_workspace(c.n_blocks)
    work.fill_(0xA5)                                          # nothing is kept in it
    c.ctx.lfps_pages_update(c.kv, None if parent is None else ints(parent), ints(new_lens), out, out_lens, copies, work,
                            None if held is None else ints(held))
    full = bool(c.ctx.lfps_poll_status() & 8)
    return out.tolist(), out_lens.tolist(), copies.tolist(), full


@pytest.mark.parametrize("page", [1, 2, 16, 64])
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_update_against_the_written_out_rules(page, seed):
    """Twenty steps of a pool in which requests fork, grow, are cut and end, some blocks held, sometimes none left."""
    r = random.Random(100 * page + seed)
    B, cap = 9, 8 * page + 3
    per = -(-cap // page)
    n_blocks = r.choice([B * per, B * per // 2, 9000])
    c = pool(B, page, cap, n_blocks, seed)
    table, lens = [[-1] * per for _ in range(B)], [0] * B
    held = [1 if r.random() < 0.05 else 0 for _ in range(n_blocks)] if seed else None
    ran_out = 0
    for _ in range(20):
        parent = None if r.random() < 0.2 else [r.choice([-1, B + 3]) if r.random() < 0.15 else (r.randrange(B) if r.random() < 0.5 else b) for b in range(B)]
        base = [lens[b if parent is None else parent[b]] if parent is None or 0 <= parent[b] < B else 0 for b in range(B)]
        new_lens = [n + r.choice([0, 1, 1, 3, page, -2, cap]) for n in base]
        want = plan(table, lens, parent, new_lens, held, n_blocks, page, cap)
        got = update(c, table, lens, parent, new_lens, held)
        for a, b in zip(got, want):
            assert a == b
        table, lens, ran_out = got[0], got[1], ran_out + got[3]
    assert ran_out > 0 or n_blocks != B * per // 2          # (the pool that cannot hold all requests at full length runs out)
    c.ctx.close()


def test_update_of_tables_and_lengths_that_make_no_sense():
    B, page, cap = 4, 16, 60
    c = pool(B, page, cap, 20, 5)
    table, lens = [[3, -7, 900, 3], [19, 19, 19, 19], [2 ** 31 - 1, 0, 0, 1], [5, 6, 7, 8]], [61, -4, 50, 33]
    parent, new_lens = [3, 0, -2 ** 31, 2 ** 31 - 1], [2 ** 31 - 1, 59, 5, 5]
    got = update(c, table, lens, parent, new_lens, None)
    assert list(got) == list(plan(table, lens, parent, new_lens, None, 20, page, cap))
    parent = [3, 2, 1, 0]
    got = update(c, table, lens, parent, new_lens, None)
    assert list(got) == list(plan(table, lens, parent, new_lens, None, 20, page, cap))
    c.ctx.close()


def test_update_of_many_requests_and_long_tables():
    r = random.Random(4)
    B, page, cap = 300, 4, 5000
    per, n_blocks = 1250, 20000
    c = pool(B, page, cap, n_blocks, 6, Hkv=1)
    free = list(range(n_blocks))
    r.shuffle(free)
    lens = [r.choice([0, 1, 7, 130, 301]) for _ in range(B)]
    lens[7] = 4999
    table = [[free.pop() if j < -(-n // page) else -1 for j in range(per)] for n in lens]
    parent = [r.choice([7, b, b, 0, -1]) for b in range(B)]
    new_lens = [(lens[p] if p >= 0 else 0) + r.choice([0, 1, 2, 9]) for p in parent]
    got = update(c, table, lens, parent, new_lens, None)
    assert list(got) == list(plan(table, lens, parent, new_lens, None, n_blocks, page, cap))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8k", "fp8kv"])
@pytest.mark.parametrize("page,rows_first", [(16, False), (16, True), (1, False), (64, False)])
def test_copies_move_the_leading_rows_only(dtype, page, rows_first):
    c = pool(2, page, 4 * page, 40, 7, dtype)
    if rows_first:
        c.K, c.V = (raw(x).transpose(1, 2).contiguous().transpose(1, 2).view(x.dtype) for x in (c.K, c.V))
    c.table, c.seq = ints([[0, 1, 2, 3]] * 2), ints([0, 0])
    c.view()
    moves = [[3, 20, page], [-1, -1, 0], [5, 21, max(1, page // 3)], [6, 99, page], [7, 22, -1], [8, 8, page], [9, 23, 10 ** 6], [-4, 24, page]]
    want = [raw(x).clone() for x in (c.K, c.V)]
    for w in want:
        for a, b, m in moves:
            if 0 <= a < 40 and 0 <= b < 40 and m > 0:
                w[b, :, :min(m, page)] = w[a, :, :min(m, page)]
    c.ctx.lfps_pages_copy(c.kv, ints(moves))
    for x, w in zip((c.K, c.V), want):
        assert torch.equal(raw(x), w)
    c.ctx.close()


@pytest.mark.parametrize("n_blocks,share", [(1, 1.0), (2, 0.5), (37, 0.3), (4096, 0.5), (4097, 0.9), (12345, 0.2), (9000, 0.0)])
@pytest.mark.parametrize("with_held", [False, True])
def test_compaction(n_blocks, share, with_held):
    r = random.Random(n_blocks)
    page, B = 2, 5
    live = sorted(r.sample(range(n_blocks), int(share * n_blocks)))
    r.shuffle(live)
    held = [0] * n_blocks
    if with_held:
        for x in r.sample(range(n_blocks), max(1, n_blocks // 10)):
            held[x] = 1
    per = max(1, -(-len(live) // B))
    c = pool(B, page, per * page, n_blocks, 8, Hkv=1)
    table = [live[b * per:(b + 1) * per] for b in range(B)]
    lens = [max(0, len(t) * page - r.randint(0, 1)) for t in table]
    used = [-(-n // page) for n in lens]
    table = [t + [r.randrange(-5, n_blocks + 5) for _ in range(per - len(t))] for t in table]
    if used[0] and used[1]:
        table[1][0] = table[0][0]                              # shared by two requests
    c.table, c.seq = ints(table), ints(lens)
    c.view()
    before = [raw(x).clone() for x in (c.K, c.V)]
    out, n_live = torch.zeros_like(c.table), ints([0])
    moves, block_map = torch.zeros((n_blocks // 2, 3), dtype=torch.int32, device=DEV), torch.zeros(n_blocks, dtype=torch.int32, device=DEV)
    work = c.ctx.pages_workspace(n_blocks)
    work.fill_(0x5A)
    c.ctx.lfps_pages_compact(c.kv, out, moves, block_map, n_live, work, ints(held) if with_held else None)
    c.ctx.lfps_pages_copy(c.kv, moves)
    alive = {table[b][j] for b in range(B) for j in range(used[b])} | {x for x in range(n_blocks) if held[x]}
    m = len(alive)
    holes = [x for x in range(m) if x not in alive]
    movers = sorted(x for x in alive if x >= m)
    want_map = [x if x in alive else -1 for x in range(n_blocks)]
    for a, b in zip(movers, holes):
        want_map[a] = b
    assert n_live.item() == m and block_map.tolist() == want_map
    want = [[a, b, page] for a, b in zip(movers, holes)]
    assert moves.tolist() == want + [[-1, -1, 0]] * (n_blocks // 2 - len(want))
    assert out.tolist() == [[want_map[table[b][j]] if j < used[b] else -1 for j in range(per)] for b in range(B)]
    for x, y in zip((c.K, c.V), before):
        for a in alive:
            assert torch.equal(raw(x)[want_map[a]], y[a])
    c.ctx.close()


def test_pages_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError, pages_workspace_bytes
    c = CacheCase("bf16", 2, 2, [30, 30], 16)
    lens, out, copies = torch.zeros_like(c.seq), torch.zeros_like(c.table), torch.zeros((2, 3), dtype=torch.int32, device=DEV)
    work = c.ctx.pages_workspace(c.n_blocks)
    ok = dict(kv=c.kv, parent=None, new_lens=c.seq, table_out=out, lens_out=lens, copies=copies, work=work)
    slab = CacheCase("bf16", 2, 2, [30, 30])
    no_pages = slab.kv
    no_pages.block_table_stride, no_pages.n_blocks = out.shape[1], c.n_blocks      # (so that the shapes pass: there is no table)
    for bad, err in ((dict(table_out=c.table), LfpsError), (dict(lens_out=c.seq), LfpsError), (dict(work=work[:-16]), LfpsError),
                     (dict(work=torch.empty(work.numel() + 4, dtype=torch.uint8, device=DEV)[4:]), LfpsError), (dict(kv=no_pages), LfpsError),
                     (dict(copies=copies[:1]), ValueError), (dict(new_lens=c.seq.long()), TypeError), (dict(held=ints([0])), ValueError)):
        with pytest.raises(err):
            c.ctx.lfps_pages_update(**{**ok, **bad})
    with pytest.raises(LfpsError) as e:
        c.ctx.lfps_pages_copy(no_pages, copies)
    assert e.value.code == LFPS_EINVAL
    with pytest.raises(ValueError):
        c.ctx.lfps_pages_copy(c.kv, copies.view(3, 2))
    assert pages_workspace_bytes(1) > 0
    c.ctx.close()
    slab.ctx.close()
