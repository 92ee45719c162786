"""A cache of bounded length as a serving loop keeps it: tokens turned into the cache, layers with a window and layers with all rows, weights
added up, rows evicted, pages freed; and the launches of a step captured into a graph."""
import pytest
import torch

from tests.cache_case import D, attend64, ints, packed
from tests.harness import DEV

pytestmark = pytest.mark.gpu


def _turned(x, pos, freq):
    x, half = x.double(), freq.shape[0]
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
    angle = (pos.double().view(-1, 1) * freq.double()).unsqueeze(1)
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()], -1)


@pytest.mark.parametrize("page", [0, 16])
def test_prompts_steps_and_evictions(page):
    """fp32, so that what the steps select can be followed in 64 bits; positions go on where the rows are fewer."""
    from paper_2506_15704_amd.binding import Lfps
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    B, Hq, Hkv, cap, budget, sink, recent, window = 3, 8, 2, 160, 60, 4, 16, 33
    G = Hq // Hkv
    ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, kv_dtype="f32", max_seq_len=cap, max_k=8, radius=1)
    freq, one = torch.tensor([1e4 ** (-i / 64) for i in range(64)], device=DEV), torch.ones(D, device=DEV)
    rot = ctx.rotary(inv_freq=freq, q_weight=one, k_weight=one, eps=1e-6)
    n_blocks = 64
    shape = (n_blocks, Hkv, page, D) if page else (B, Hkv, cap, D)
    K, V = torch.full(shape, float("nan"), device=DEV), torch.full(shape, float("nan"), device=DEV)
    per = cap // 16
    tables, lens, at = [torch.full((B, per), -1, dtype=torch.int32, device=DEV) for _ in range(2)], [ints([0] * B) for _ in range(2)], 0
    copies, work = torch.zeros((B, 3), dtype=torch.int32, device=DEV), ctx.pages_workspace(n_blocks)
    masses = [torch.full((B, Hkv, cap), float("nan"), device=DEV) for _ in range(2)]
    held, place = ints([0] * B), [0] * B                          # rows with a weight; positions used so far
    rows = [[torch.zeros((0, D), dtype=torch.float64, device=DEV) for _ in range(Hkv)] for _ in range(B)]
    values = [[torch.zeros((0, D), dtype=torch.float64, device=DEV) for _ in range(Hkv)] for _ in range(B)]
    weight = [[torch.zeros(0, dtype=torch.float64, device=DEV) for _ in range(Hkv)] for _ in range(B)]

    def resize(new_lens):
        nonlocal at
        if page:
            kv = ctx.paged_kv_view(K, V, tables[at], lens[at])
            ctx.lfps_pages_update(kv, None, ints(new_lens), tables[1 - at], lens[1 - at], copies, work)
            ctx.lfps_pages_copy(kv, copies)
        else:
            lens[1 - at].copy_(ints(new_lens))
        at = 1 - at
        assert lens[at].tolist() == new_lens
        return ctx.paged_kv_view(K, V, tables[at], lens[at]) if page else ctx.kv_view(K, V, lens[at])

    for news in ([100, 30, 1], [1, 1, 1], [20, 70, 120], [1, 1, 1], [1, 1, 1]):
        before = lens[at].tolist()
        kv = resize([n + t for n, t in zip(before, news)])
        T = sum(news)
        qkv = torch.randn((T, Hq + 2 * Hkv, D), device=DEV, generator=g)
        q, kn, vn = qkv.split([Hq, Hkv, Hkv], dim=1)
        pos = torch.cat([torch.arange(p, p + t) for p, t in zip(place, news)]).to(torch.int32).to(DEV)
        cu, cut = ints(packed(news)), packed(news)
        q_out = torch.zeros((T, Hq, D), device=DEV)
        ctx.lfps_rotate_append(rot, q, kn, vn, pos, cu, kv, q_out)
        win, full = torch.zeros_like(q_out), torch.zeros_like(q_out)
        if max(news) == 1:
            ctx.lfps_window_attn_decode(q_out, kv, window, sink, win)
            ctx.lfps_full_attn_mass_decode(q_out, kv, masses[0], full, held=held)
        else:
            ctx.lfps_window_attn(q_out, cu, kv, window, sink, win)
            ctx.lfps_prompt_attn(q_out, cu, kv, full)
            ctx.lfps_attn_mass(q_out, cu, kv, masses[0], held=held)
        qr, kr = _turned(q, pos, freq), _turned(kn, pos, freq)
        for b, t in enumerate(news):
            for h in range(Hkv):
                rows[b][h] = torch.cat([rows[b][h], kr[cut[b]:cut[b + 1], h]])
                values[b][h] = torch.cat([values[b][h], vn[cut[b]:cut[b + 1], h].double()])
                weight[b][h] = torch.cat([weight[b][h], torch.zeros(t, dtype=torch.float64, device=DEV)])
                n = rows[b][h].shape[0]
                for i in range(t):
                    p = n - t + i
                    for x in range(h * G, h * G + G):
                        w = torch.softmax(rows[b][h][:p + 1] @ qr[cut[b] + i, x] / D ** 0.5, 0)
                        weight[b][h][:p + 1] += w
                        if i in (0, t - 1):
                            j = torch.arange(p + 1, device=DEV)
                            j = j[(j > p - window) | (j < sink)]
                            ref = attend64(qr[cut[b] + i, x].view(1, D), rows[b][h][j], values[b][h][j])[0][0]
                            assert float((win[cut[b] + i, x].double() - ref).abs().max()) < 1e-5
                            assert float((full[cut[b] + i, x].double() - w @ values[b][h][:p + 1]).abs().max()) < 1e-5
                assert float((masses[0][b, h, :n].double() - weight[b][h]).abs().max()) < 1e-4
        place = [p + t for p, t in zip(place, news)]
        # what is over the budget goes; the survivors are followed by the library's own choice, which the weights in 64 bits bear out
        kept = torch.full((B, Hkv, cap), -1, dtype=torch.int32, device=DEV)
        lens_out = ints([0] * B)
        ctx.lfps_evict(kv, masses[0], ints([budget] * B), sink, recent, masses[1], kept, lens_out)
        masses.reverse()
        for b in range(B):
            n = rows[b][0].shape[0]
            m = min(n, budget)
            assert int(lens_out[b]) == m
            for h in range(Hkv):
                i = kept[b, h, :m].long()
                if m < n:
                    gone = torch.ones(n, dtype=torch.bool, device=DEV)
                    gone[i] = False
                    between = i[sink:m - recent]
                    assert i[:sink].tolist() == list(range(sink)) and i[m - recent:].tolist() == list(range(n - recent, n))
                    assert float(weight[b][h][gone].max()) <= float(weight[b][h][between].min()) + 1e-4
                rows[b][h], values[b][h], weight[b][h] = rows[b][h][i], values[b][h][i], weight[b][h][i]
        held = lens_out.clone()
        if page:
            resize([r[0].shape[0] for r in rows])
        else:
            lens[at].copy_(lens_out)
    ctx.close()


@pytest.mark.parametrize("page", [0, 16])
def test_a_captured_step_gives_what_eager_calls_give(page):
    """Rotation, both attentions, the weights and an eviction into another cache, replayed with other inputs between eager work."""
    from paper_2506_15704_amd.binding import Lfps
    g = torch.Generator(device=DEV)
    g.manual_seed(6)
    B, Hq, Hkv, cap = 4, 8, 2, 300
    ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, max_seq_len=cap, max_k=8, radius=1)
    other = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, max_seq_len=cap, max_k=8, radius=1)      # eager work has a workspace of its own
    rot = ctx.rotary(inv_freq=torch.tensor([1e4 ** (-i / 32) for i in range(32)], device=DEV), q_weight=torch.ones(D, device=DEV))
    shape = (B * 19 + 2, Hkv, 16, D) if page else (B, Hkv, cap, D)
    randn = lambda *s: torch.randn(s, device=DEV, generator=g)  # noqa: E731
    caches = [[randn(*shape).to(torch.bfloat16) for _ in range(2)] for _ in range(2)]
    table = torch.randperm(B * 19 + 2, device=DEV, generator=g)[:B * 19].view(B, 19).to(torch.int32).contiguous()
    lens, cu, budget = ints([300, 41, 1, 170]), ints([0, 2, 4, 5, 10]), ints([100, 41, 5, 60])
    view = lambda c, x: c.paged_kv_view(x[0], x[1], table, lens) if page else c.kv_view(x[0], x[1], lens)  # noqa: E731
    qkv, qd, pos = randn(10, Hq + 2 * Hkv, D).to(torch.bfloat16), randn(B, Hq, D), ints(list(range(10)))
    q, kn, vn = qkv.split([Hq, Hkv, Hkv], dim=1)

    def state():
        z = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device=DEV)  # noqa: E731
        return dict(q_out=z(10, Hq, D, dt=torch.bfloat16), win=z(10, Hq, D, dt=torch.bfloat16), step=z(B, Hq, D), full=z(B, Hq, D), mass=z(B, Hkv, cap),
                    sums=z(B, Hkv, cap), mass_out=z(B, Hkv, cap), kept=z(B, Hkv, cap, dt=torch.int32), lens_out=ints([0] * B))

    def work(c, s, to):
        kv = view(c, caches[0])
        c.lfps_rotate_append(rot, q, kn, vn, pos, cu, kv, s["q_out"])
        c.lfps_window_attn(s["q_out"], cu, kv, 50, 3, s["win"])
        c.lfps_window_attn_decode(qd, kv, 50, 3, s["step"])
        c.lfps_full_attn_mass_decode(qd, kv, s["mass"], s["full"], held=lens, decay=0.5)
        c.lfps_attn_mass(s["q_out"], cu, kv, s["sums"])
        c.lfps_evict(kv, s["sums"], budget, 4, 10, s["mass_out"], s["kept"], s["lens_out"], to=view(c, to))

    captured, eager, spare = state(), state(), [x.clone() for x in caches[1]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(ctx, captured, caches[1])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work(ctx, captured, caches[1])
    for x in captured.values():
        x.zero_()
    for x, y in zip(spare, caches[1]):
        x.copy_(y)
    for turn in range(4):
        qkv.copy_(randn(10, Hq + 2 * Hkv, D).to(torch.bfloat16))
        qd.copy_(randn(B, Hq, D))
        pos.copy_(ints([1000 * turn + i for i in range(10)]))
        lens.copy_(ints([300 - turn, 41 + turn, 1 + 3 * turn, 170]))
        graph.replay()
        if turn % 2:
            torch.cuda.synchronize()
        work(other, eager, spare)
        for name in captured:
            assert torch.equal(captured[name], eager[name]), (turn, name)
        for x, y in zip(spare, caches[1]):
            assert torch.equal(x, y)
    ctx.close()
    other.close()


def test_another_stream_than_the_default():
    """Everything is enqueued on the current stream: inputs that a slow kernel on it makes are waited for."""
    from paper_2506_15704_amd.binding import Lfps
    B, Hq, Hkv, n = 2, 4, 1, 500
    ctx = Lfps(batch=B, n_q_heads=Hq, n_kv_heads=Hkv, max_seq_len=n, max_k=8, radius=1)
    stream = torch.cuda.Stream()
    outs = []
    for s in (torch.cuda.current_stream(), stream):
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g = torch.Generator(device=DEV)
            g.manual_seed(7)
            slow = torch.randn((4096, 4096), device=DEV, generator=g)
            for _ in range(10):
                slow = slow @ slow * 1e-2
            K, V = (torch.randn((B, Hkv, n, D), device=DEV, generator=g).to(torch.bfloat16) for _ in range(2))
            q, lens = torch.randn((B, Hq, D), device=DEV, generator=g), ints([n, 200])
            kv = ctx.kv_view(K, V, lens)
            out, full, mass = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((B, Hkv, n), device=DEV)
            ctx.lfps_window_attn_decode(q, kv, 90, 2, out)
            ctx.lfps_full_attn_mass_decode(q, kv, mass, full)
            kept, lens_out, mass_out = torch.zeros((B, Hkv, n), dtype=torch.int32, device=DEV), ints([0, 0]), torch.zeros_like(mass)
            ctx.lfps_evict(kv, mass, ints([100, 100]), 2, 5, mass_out, kept, lens_out)
            outs.append([x.clone() for x in (out, full, mass, K, V, kept, lens_out)])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    ctx.close()
