"""Appends, prompts, shared prefixes and copies of pages where the cache is pinned host memory, and in contexts whose partial results
need more room than the least."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints, raw
from tests.harness import DEV, stored_values

pytestmark = pytest.mark.gpu


def pinned(x):
    h = torch.empty(raw(x).shape, dtype=raw(x).dtype, pin_memory=True)
    h.copy_(raw(x))
    return h.view(x.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv", "fp8v"])
def test_a_cache_in_host_memory_gives_the_same_results(dtype):
    """Bit for bit, and the appended rows are the same ones: few tokens in parts, a prompt, a prefix that small and large groups share."""
    lens, news = [900, 310, 40] + [300 + i for i in range(37)], [5, 300, 7] + [1] * 37
    c = CacheCase(dtype, 4, 1, lens, seed=1)
    T = sum(news)
    q = c.randn(T, 4, D).to(c.q_dtype)
    k, v = (c.randn(T, 1, D).to(c.q_dtype) for _ in range(2))
    cu, qd = ints([sum(news[:b]) for b in range(c.B + 1)]), c.randn(c.B, 4, D)
    runs = []
    for K, V in ((raw(c.K).clone().view(c.kd), raw(c.V).clone().view(c.vd)), (pinned(c.K), pinned(c.V))):
        kv = c.ctx.kv_view(K, V, c.seq)
        c.ctx.lfps_append(k, v, cu, kv)
        outs = [torch.zeros_like(q)]
        c.ctx.lfps_prompt_attn(q, cu, kv, outs[0])
        for starts, prefixes in (([0, 3, 40], [30, 256]), ([0, 1, 2], [700, 300])):
            outs.append(torch.zeros((c.B, 4, D), device=DEV))
            c.ctx.lfps_prefix_attn_decode(qd, kv, ints(starts), ints(prefixes), outs[-1])
        torch.cuda.synchronize()
        runs.append(outs + [raw(x).to(DEV) for x in (K, V)])
    for a, b in zip(*runs):
        assert torch.equal(a.nan_to_num(7) if a.is_floating_point() else a, b.nan_to_num(7) if b.is_floating_point() else b)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8k"])
def test_pages_in_host_memory(dtype):
    from paper_2506_15704_amd import binding
    lens = [70, 33, 90]
    c = CacheCase(dtype, 2, 2, lens, 16, seed=2)
    K, V = pinned(c.K), pinned(c.V)
    kv = binding.lfps_kv(binding._cache_ptr(K), binding._cache_ptr(V), K.stride(0), K.stride(1), K.stride(2), c.seq.data_ptr(),
                         c.table.data_ptr(), 16, c.table.stride(0), c.n_blocks)
    moves = ints([[int(c.table[0, 1]), int(c.table[1, 4]), 16], [int(c.table[2, 0]), int(c.table[1, 5]), 9], [-1, -1, 0]])
    q, cu = c.randn(6, 2, D).to(torch.bfloat16), ints([0, 1, 3, 6])
    outs = [torch.zeros_like(q), torch.zeros_like(q)]
    for view, out in ((c.kv, outs[0]), (kv, outs[1])):
        c.ctx.lfps_pages_copy(view, moves)
        c.ctx.lfps_append(q, q, cu, view)
        c.ctx.lfps_prompt_attn(q, cu, view, out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    for x, y in ((c.K, K), (c.V, V)):
        same = raw(x).cpu(), raw(y)
        assert torch.equal(*(t.nan_to_num(7) if t.is_floating_point() else t for t in same))
    c.ctx.close()


def _attend(c, q, lead, shared):
    """[B, Hq, D] in 64 bits, all requests at once, rows below `shared` those of request `lead`; and the weighted |v|."""
    i = torch.arange(c.cap, device=DEV)
    from_ = torch.where(i < shared.view(-1, 1), lead.view(-1, 1), torch.arange(c.B, device=DEV).view(-1, 1))
    k, v = (stored_values(x).double().nan_to_num(0)[from_, :, i.expand_as(from_)].permute(0, 2, 3, 1).contiguous() for x in (c.K, c.V))
    x = torch.matmul(q.double().view(c.B, c.Hkv, c.G, D), k) / D ** 0.5
    p = torch.softmax(x.masked_fill(i >= c.seq.view(-1, 1, 1, 1), float("-inf")), -1)
    v = v.transpose(2, 3).contiguous()
    dots = torch.matmul(q.double().abs().view(c.B, c.Hkv, c.G, D), k.abs()).amax(-1, keepdim=True) / D ** 0.5
    return [t.view(c.B, c.Hq, -1) for t in (torch.matmul(p, v), torch.matmul(p, v.abs()), dots)]


# Query and weights as sums of 16-bit terms, 2^-18 (bf16) or 2^-22 (fp16) left of each; fp32 products and sums, 2^-24 of the absolute sum a
# term, the scores' errors twice; the exponential 2^-21.
def _tolerance(dtype, weighted, dots, n):
    left = {"f16": 2.0 ** -22, "f32": 0.0}.get(dtype, 2.0 ** -18)
    return (2 * (left + 260 * 2.0 ** -24) * dots + 2 * left + 2.0 ** -21 + (n + 80) * 2.0 ** -24) * weighted + 1e-7


@pytest.mark.parametrize("dtype,group", [("bf16", 4), ("f32", 4), ("fp8kv", 50), ("bf16", 50)])
def test_prefix_of_more_heads_than_the_least_room_has_rows(dtype, group):
    """1100 requests of 32 heads: 70400 partial rows for two parts."""
    B = 1100
    c = CacheCase(dtype, 32, 8, [60 + (b * 7) % 41 for b in range(B)], seed=3)
    starts = list(range(0, B, group)) + [B]
    prefixes = [20 + (i * 5) % 40 for i in range(len(starts) - 1)]
    q, out = c.randn(B, 32, D), torch.zeros((B, 32, D), device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints(starts), ints(prefixes), out)
    lead = torch.arange(B, device=DEV) // group * group
    shared = torch.minimum(torch.tensor(prefixes, device=DEV)[lead // group], c.seq[lead].long())
    ref, weighted, dots = _attend(c, q, lead, shared)
    assert bool(((out.double() - ref).abs() <= _tolerance(dtype, weighted, dots, 100)).all())
    c.ctx.close()


def test_prompt_of_more_heads_than_the_least_room_has_rows():
    """One token of each of 1100 requests, 32 heads; and a few tokens of a few of them."""
    B = 1100
    c = CacheCase("bf16", 32, 8, [60 + (b * 7) % 41 for b in range(B)], seed=4)
    q, out = c.randn(B, 32, D).to(torch.bfloat16), torch.zeros((B, 32, D), dtype=torch.bfloat16, device=DEV)
    none = torch.zeros(B, dtype=torch.long, device=DEV)
    ref, weighted, dots = _attend(c, q.float(), none, none)
    # 16-bit weights and output, half a step each; fp32 scores and sums
    tol = 2.0 ** -8 * 1.01 * (ref.abs() + weighted) + (2 * 130 * 2.0 ** -24 * dots + 2.0 ** -21 + 110 * 2.0 ** -24) * weighted + 1e-7
    c.ctx.lfps_prompt_attn(q, ints(list(range(B + 1))), c.kv, out)
    assert bool(((out.double() - ref).abs() <= tol).all())
    few = [3, 500, 501, 1099]                                    # only these bring a token
    cu = ints([sum(x < b for x in few) for b in range(B + 1)])
    got = torch.zeros((4, 32, D), dtype=torch.bfloat16, device=DEV)
    c.ctx.lfps_prompt_attn(q[few].contiguous(), cu, c.kv, got)
    assert bool(((got.double() - ref[few]).abs() <= tol[few]).all())
    c.ctx.close()


def test_fp16_prompts_keep_the_sum_of_many_small_weights():
    """One key 2^22.1 above 65535 others, which together weigh 1.4%: weights below the normal fp16 numbers count in sum and output alike."""
    T, n = 32768, 65536
    c = CacheCase("f16", 2, 1, [n], seed=5, scale=0.0)
    c.V.fill_(1.0)
    c.K[0, 0, 0, 0], c.V[0, 0, 0] = 10.83, 0.0
    q = torch.zeros((T, 2, D), dtype=torch.float16, device=DEV)
    q[..., 0] = 16.0
    out = torch.zeros_like(q)
    c.ctx.lfps_prompt_attn(q, ints([0, T]), c.kv, out)
    w = torch.exp(-16.0 * c.K[0, 0, 0, 0].double() / D ** 0.5)
    others = n - T + torch.arange(T, device=DEV).double()
    ref = (others * w / (1 + others * w)).view(T, 1, 1)
    # 2^-15 < weight * 2^8 < 2^-14: a step of 2^-24 there, half of it 2^-10 of a weight (sum and output hold the same rounded one); output 2^-11
    assert bool(((out.double() - ref).abs() <= (2.0 ** -10 + 2.0 ** -11 + 2.0 ** -14) * ref).all())
    c.ctx.close()


def _far_apart(x, stride_b, stride_n, dtype):
    """[n, Hkv, rows, D] with the given strides in a buffer of its own, most of which nothing touches."""
    n, Hkv, rows, _ = x.shape
    size = (n - 1) * stride_b + (rows - 1) * stride_n + Hkv * D
    y = torch.empty(size, dtype=raw(x).dtype, device=DEV).as_strided(x.shape, (stride_b, D, stride_n, 1))
    y.copy_(raw(x))
    return y.view(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv", "f32"])
@pytest.mark.parametrize("layout,stride_b,stride_n", [(0, (1 << 30) + 64, 256), (0, 256, 3 << 20), (16, 80_000_000, 256), (16, 256, (9 << 24) + 32)])
def test_rows_more_than_2_to_the_31_elements_apart(dtype, layout, stride_b, stride_n):
    """Requests, rows, blocks, and rows of a block: the same results as close together, and the same rows appended and copied."""
    lens, news = [700, 200, 333], [3, 150, 0]
    c = CacheCase(dtype, 4, 2, lens, layout, cap=700, seed=6)
    if layout == 0 and stride_n > stride_b:
        stride_b = 2 * D                                       # (rows of the requests side by side: three of them in one stride)
    far = [_far_apart(x, stride_b, stride_n, x.dtype) for x in (c.K, c.V)]
    assert (far[0].shape[0] - 1) * stride_b + (far[0].shape[2] - 1) * stride_n > 1 << 31
    q, qd = c.randn(153, 4, D).to(c.q_dtype), c.randn(3, 4, D)
    k, v = (c.randn(153, 2, D).to(c.q_dtype) for _ in range(2))
    cu, runs = ints([0, 3, 153, 153]), []
    for K, V in ((c.K, c.V), far):
        kv = c.ctx.paged_kv_view(K, V, c.table, c.seq) if layout else c.ctx.kv_view(K, V, c.seq)
        if layout:
            spare = sorted(set(range(c.n_blocks)) - set(c.table.flatten().tolist()))
            c.ctx.lfps_pages_copy(kv, ints([[int(c.table[0, 2]), spare[-1], 16], [int(c.table[2, 1]), spare[0], 5]]))
        c.ctx.lfps_append(k, v, cu, kv)
        outs = [torch.zeros_like(q), torch.zeros_like(qd)]
        c.ctx.lfps_prompt_attn(q, cu, kv, outs[0])
        c.ctx.lfps_prefix_attn_decode(qd, kv, ints([0, 2, 3]), ints([150, 40]), outs[1])
        runs.append(outs + [raw(x).contiguous().view(torch.uint8 if x.element_size() == 1 else torch.int16 if x.element_size() == 2 else torch.int32) for x in (K, V)])
    for a, b in zip(*runs):
        assert torch.equal(a, b)
    c.ctx.close()
