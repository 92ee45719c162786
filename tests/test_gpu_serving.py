"""Prompts, forks, decode steps and a compaction over one paged cache, as a serving loop makes them, against the same rows in a
contiguous cache and in 64 bits; and the same loop's launches captured into a graph."""
import pytest
import torch

from tests.cache_case import D, attend64, ints, packed
from tests.harness import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
def test_a_prompt_its_forks_and_their_steps(fp8):
    from paper_2506_15704_amd.binding import Lfps
    g = torch.Generator(device=DEV)
    g.manual_seed(11)
    B, Hq, Hkv, page, cap, n_blocks, steps = 6, 8, 2, 16, 700, 300, 6
    per, k = -(-cap // page), 64
    ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, max_seq_len=cap, max_k=k, radius=2, k_fp8=fp8, v_fp8=fp8)
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    K, V = (torch.full((n_blocks, Hkv, page, D), float("nan"), device=DEV).to(dt) for _ in range(2))
    rows = [[] for _ in range(B)]                                # every request's (k, v) rows as appended, [t, Hkv, D] each
    tables, lens = [torch.full((B, per), -1, dtype=torch.int32, device=DEV) for _ in range(2)], [ints([0] * B) for _ in range(2)]
    work, copies, at = ctx.pages_workspace(n_blocks), torch.zeros((B, 3), dtype=torch.int32, device=DEV), 0

    def next_pages(parent, new_lens):
        nonlocal at
        kv = ctx.paged_kv_view(K, V, tables[at], lens[at])
        ctx.lfps_pages_update(kv, ints(parent), ints(new_lens), tables[1 - at], lens[1 - at], copies, work)
        ctx.lfps_pages_copy(kv, copies)
        at = 1 - at
        assert lens[at].tolist() == new_lens and ctx.lfps_poll_status() == 0
        return ctx.paged_kv_view(K, V, tables[at], lens[at])

    def new_rows(news):
        T = sum(news)
        qkv = torch.randn((T, Hq + 2 * Hkv, D), device=DEV, generator=g).to(torch.bfloat16)
        q, kn, vn = qkv.split([Hq, Hkv, Hkv], dim=1)
        cut = packed(news)
        for b in range(B):
            rows[b] = rows[b] + [(kn[cut[b]:cut[b + 1]], vn[cut[b]:cut[b + 1]])]
        return q, kn, vn, ints(cut)

    def cache(b):
        kb, vb = (torch.cat([r[i] for r in rows[b]]).float() for i in (0, 1))
        return [x.to(dt).float().double().transpose(0, 1) for x in (kb, vb)]

    # two prompts, the second in two chunks
    for news, new_lens in (([333, 120, 0, 0, 0, 0], [333, 120, 0, 0, 0, 0]), ([0, 77, 0, 0, 0, 0], [333, 197, 0, 0, 0, 0])):
        kv = next_pages(list(range(B)), new_lens)
        q, kn, vn, cu = new_rows(news)
        ctx.lfps_append(kn, vn, cu, kv)
        out = torch.zeros(q.shape, dtype=q.dtype, device=DEV)
        ctx.lfps_prompt_attn(q, cu, kv, out)
        cut = packed(news)
        for b in range(B):
            if news[b]:
                kb, vb = cache(b)
                for h in range(Hq):
                    i = news[b] - 1
                    ref, weighted, _ = attend64(q[cut[b] + i, h:h + 1].double(), kb[h // 4], vb[h // 4])
                    assert bool(((out[cut[b] + i, h].double() - ref[0]).abs() <= 2.0 ** -8 * 1.01 * (ref.abs() + weighted)[0] + 1e-3 * weighted[0]).all())
    # the first is continued four times, the second twice (slots 0 and 5 swap ancestors: 1 ends there)
    parent = [0, 0, 0, 0, 1, 1]
    have = [333, 333, 333, 333, 197, 197]
    rows = [list(rows[p]) for p in parent]
    kv = next_pages(parent, [n + 1 for n in have])
    group_start, prefix = ints([0, 4, 6]), ints([333, 197])
    budget = ints([k] * B)
    topk, nxt = (torch.full((B, Hq, k), -1, dtype=torch.int32, device=DEV) for _ in range(2))
    for step in range(steps):
        have = [n + 1 for n in have]
        if step:
            kv = next_pages(list(range(B)), have)
        q, kn, vn, cu = new_rows([1] * B)
        ctx.lfps_append(kn, vn, cu, kv)
        qf, out, full, sparse = q.float().contiguous(), *(torch.zeros((B, Hq, D), device=DEV) for _ in range(3))
        ctx.lfps_prefix_attn_decode(qf, kv, group_start, prefix, out)
        ctx.lfps_full_attn_decode(qf, kv, full)
        for b in range(B):
            kb, vb = cache(b)
            assert kb.shape[1] == have[b]
            for h in range(Hq):
                ref, weighted, dots = attend64(qf[b, h:h + 1].double(), kb[h // 4], vb[h // 4])
                tol = (2.0 ** -16 * (1 + dots) * weighted + 1e-6)[0]
                assert bool(((out[b, h].double() - ref[0]).abs() <= tol).all()) and bool(((full[b, h].double() - ref[0]).abs() <= tol).all())
        if step == 0:
            ctx.lfps_exact_topk(qf, kv, budget, topk)
        else:
            ctx.lfps_step(qf, kv, topk, budget, nxt, sparse)
            topk, nxt = nxt, topk
            assert bool((topk >= 0).all())
    # two end, the pool is compacted, and the others go on as if nothing had happened
    kv = next_pages([0, -1, 2, 3, -1, 5], [have[0], 0, have[2], have[3], 0, have[5]])
    before = torch.zeros((B, Hq, D), device=DEV)
    ctx.lfps_full_attn_decode(qf, kv, before)
    moves, block_map, n_live = torch.zeros((n_blocks // 2, 3), dtype=torch.int32, device=DEV), torch.zeros(n_blocks, dtype=torch.int32, device=DEV), ints([0])
    ctx.lfps_pages_compact(kv, tables[1 - at], moves, block_map, n_live, work)
    ctx.lfps_pages_copy(kv, moves)
    lens[1 - at].copy_(lens[at])
    at = 1 - at
    kv = ctx.paged_kv_view(K, V, tables[at], lens[at])
    assert int(tables[at].max()) < n_live.item() < n_blocks
    after = torch.zeros_like(before)
    ctx.lfps_full_attn_decode(qf, kv, after)
    assert torch.equal(before, after)
    ctx.close()


def test_a_captured_step_replays_like_the_eager_one():
    """Pages, copies, append, prompt attention and prefix attention in one graph; every replay, with eager work between them, against
    the eager calls on a cache of its own."""
    from paper_2506_15704_amd.binding import Lfps
    B, Hq, Hkv, page, cap, n_blocks = 5, 4, 2, 16, 400, 200
    per = -(-cap // page)

    class Side:
        def __init__(self):
            g = torch.Generator(device=DEV)
            g.manual_seed(3)
            self.ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, max_seq_len=cap, max_k=1, radius=1)
            self.K, self.V = (torch.randn((n_blocks, Hkv, page, D), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
            self.table = torch.randperm(n_blocks, device=DEV, generator=g)[:B * per].view(B, per).to(torch.int32).contiguous()
            self.lens, self.new_lens = ints([300, 17, 33, 0, 250]), ints([310, 301, 301, 4, 250])
            self.parent = ints([0, 0, 0, 3, 4])
            self.table2, self.lens2, self.copies = torch.zeros_like(self.table), torch.zeros_like(self.lens), torch.zeros((B, 3), dtype=torch.int32, device=DEV)
            self.work = self.ctx.pages_workspace(n_blocks)
            self.cu, self.T = ints([0, 10, 11, 12, 16, 16]), 16
            self.q = torch.zeros((self.T, Hq, D), dtype=torch.bfloat16, device=DEV)
            self.k, self.v = (torch.zeros((self.T, Hkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
            self.qd, self.outd, self.out = torch.zeros((B, Hq, D), device=DEV), torch.zeros((B, Hq, D), device=DEV), torch.zeros_like(self.q)
            self.start, self.prefix = ints([0, 3, 5]), ints([280, 3])
            self.kv, self.kv2 = (self.ctx.paged_kv_view(self.K, self.V, t, n) for t, n in ((self.table, self.lens), (self.table2, self.lens2)))

        def fill(self, seed):
            g = torch.Generator(device=DEV)
            g.manual_seed(seed)
            for x in (self.q, self.k, self.v, self.qd):
                x.copy_(torch.randn(x.shape, device=DEV, generator=g))

        def run(self):
            c = self.ctx
            c.lfps_pages_update(self.kv, self.parent, self.new_lens, self.table2, self.lens2, self.copies, self.work)
            c.lfps_pages_copy(self.kv, self.copies)
            c.lfps_append(self.k, self.v, self.cu, self.kv2)
            c.lfps_prompt_attn(self.q, self.cu, self.kv2, self.out)
            c.lfps_prefix_attn_decode(self.qd, self.kv2, self.start, self.prefix, self.outd)

    a, e = Side(), Side()
    a.fill(1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):                                # another stream than the tensors' own
        a.run()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.run()
    for seed in (5, 6, 7):
        a.fill(seed)
        e.fill(seed)
        e.run()
        torch.cuda.synchronize()
        graph.replay()
        for x, y in ((a.out, e.out), (a.outd, e.outd), (a.table2, e.table2), (a.lens2, e.lens2), (a.copies, e.copies), (a.K, e.K), (a.V, e.V)):
            assert torch.equal(x, y)
    a.ctx.close()
    e.ctx.close()
