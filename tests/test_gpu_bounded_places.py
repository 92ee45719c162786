"""Rotation, windows, accumulated weights and eviction where the cache is pinned host memory, where it is spread over more than 2^31 elements, and
where a context has more heads, rows or requests than the usual ones."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints, raw
from tests.harness import DEV
from tests.test_gpu_cache_places import _far_apart, pinned
from tests.test_gpu_evict import _evict_and_check, _mass
from tests.test_gpu_mass import _check as check_mass, _check_step as check_mass_step
from tests.test_gpu_window import _check as check_window, _check_step as check_window_step

pytestmark = pytest.mark.gpu


def _bits(x):
    x = x.contiguous()
    return raw(x).view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()])


def _everything(c, kv, news, seed):
    """Every call once, in the order of their use; a second cache of the same kind receives nothing: the eviction is in place."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    T = sum(news)
    qkv = torch.randn((T, c.Hq + 2 * c.Hkv, D), device=DEV, generator=g).to(c.q_dtype)
    q, k, v = qkv[:, :c.Hq], qkv[:, c.Hq:c.Hq + c.Hkv], qkv[:, c.Hq + c.Hkv:]
    cu = ints([sum(news[:b]) for b in range(c.B + 1)])
    rot = c.ctx.rotary(inv_freq=1e4 ** (-torch.arange(64, device=DEV) / 64), q_weight=1 + 0.1 * torch.randn(D, device=DEV, generator=g), eps=1e-6)
    turned, out = torch.empty_like(q.contiguous()), torch.zeros((T, c.Hq, D), dtype=c.q_dtype, device=DEV)
    c.ctx.lfps_rotate_append(rot, q, k, v, None, cu, kv, turned)
    c.ctx.lfps_window_attn(turned, cu, kv, 100, 5, out)
    mass = torch.zeros((c.B, c.Hkv, c.cap), device=DEV)
    c.ctx.lfps_attn_mass(turned, cu, kv, mass)
    step, rows = torch.randn((c.B, c.Hq, D), device=DEV, generator=g), [torch.zeros((c.B, c.Hq, D), device=DEV) for _ in range(2)]
    c.ctx.lfps_window_attn_decode(step, kv, 150, 3, rows[0])
    c.ctx.lfps_full_attn_mass_decode(step, kv, mass, rows[1], held=c.seq, decay=0.5)
    weights = mass.clone()
    mass_out, kept, lens = torch.zeros_like(mass), torch.zeros_like(mass, dtype=torch.int32), torch.zeros_like(c.seq)
    c.ctx.lfps_evict(kv, mass, ints([n * 2 // 3 for n in c.lens]), 4, 20, mass_out, kept, lens)
    torch.cuda.synchronize()
    return [turned, out, weights, *rows, mass_out, kept, lens]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv", "fp8v"])
@pytest.mark.parametrize("layout", [0, 16])
def test_a_cache_in_host_memory_gives_the_same_results(dtype, layout):
    from paper_2506_15704_amd import binding
    lens, news = [500, 310, 40], [5, 300, 7]
    c = CacheCase(dtype, 4, 1, lens, layout, seed=1)
    K, V = pinned(c.K), pinned(c.V)
    page = (c.table.data_ptr(), layout, c.table.stride(0), c.n_blocks) if layout else ()
    host = binding.lfps_kv(binding._cache_ptr(K), binding._cache_ptr(V), K.stride(0), K.stride(1), K.stride(2), c.seq.data_ptr(), *page)
    runs = [_everything(c, kv, news, 5) for kv in (c.kv, host)]
    for a, b in zip(runs[0] + [c.K, c.V], runs[1] + [raw(x).to(DEV).view(x.dtype) for x in (K, V)]):
        assert torch.equal(_bits(a), _bits(b))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv", "f32"])
@pytest.mark.parametrize("layout,stride_b,stride_n", [(0, (1 << 30) + 64, 256), (0, 256, 3 << 20), (16, 80_000_000, 256), (16, 256, (9 << 24) + 32)])
def test_rows_more_than_2_to_the_31_elements_apart(dtype, layout, stride_b, stride_n):
    lens, news = [700, 200, 333], [3, 150, 0]
    c = CacheCase(dtype, 4, 2, lens, layout, cap=700, seed=6)
    if layout == 0 and stride_n > stride_b:
        stride_b = 2 * D                                       # (rows of the requests side by side: three of them in one stride)
    far = [_far_apart(x, stride_b, stride_n, x.dtype) for x in (c.K, c.V)]
    assert (far[0].shape[0] - 1) * stride_b + (far[0].shape[2] - 1) * stride_n > 1 << 31
    near, runs = [x.clone() if x.element_size() > 1 else raw(x).clone().view(x.dtype) for x in (c.K, c.V)], []
    for K, V in (near, far):
        kv = c.ctx.paged_kv_view(K, V, c.table, c.seq) if layout else c.ctx.kv_view(K, V, c.seq)
        runs.append(_everything(c, kv, news, 7) + [K, V])
        if K is far[0]:                                        # and from there into rows that lie together
            to = c.ctx.paged_kv_view(c.K, c.V, c.table, c.seq) if layout else c.ctx.kv_view(c.K, c.V, c.seq)
            w, lens_out = torch.rand((3, 2, 700), device=DEV), ints([0, 0, 0])
            kept, mass_out = torch.zeros(w.shape, dtype=torch.int32, device=DEV), torch.zeros_like(w)
            c.ctx.lfps_evict(kv, w, ints([90, 90, 90]), 1, 1, mass_out, kept, lens_out, to=to)
            for b in range(3):
                for g in range(2):
                    i = kept[b, g, :90].long()
                    at, block = (i % 16, c.table[b].long()[i // 16]) if layout else (i, torch.full_like(i, b))
                    for x, y in ((far[0], c.K), (far[1], c.V)):
                        assert torch.equal(raw(x)[block, g, at], raw(c.get(y, b, 0, 90))[:, g])
    for a, b in zip(*runs):
        assert torch.equal(_bits(a), _bits(b))
    c.ctx.close()


@pytest.mark.parametrize("lens,Hkv", [([70001, 33000, 32768, 32769], 1), ([40000], 2), ([35000] * 9 + [3], 16)])
def test_evictions_of_more_rows_than_registers_hold(lens, Hkv):
    """More than 32768: a request's rows are read again by every pass, and what is kept of the parts before counts on."""
    c = CacheCase("fp8kv", Hkv, Hkv, lens, 64, seed=2)
    budget = [n // 3 for n in lens]
    _evict_and_check(c, _mass(c), budget, 4, 500)
    c.ctx.close()


def test_evictions_of_many_equal_weights_over_many_rows():
    c = CacheCase("fp8kv", 1, 1, [66000, 66000], 64, seed=3)
    w = torch.zeros((2, 1, 66000), device=DEV)
    w[0, 0, 65000:] = 1.0
    w[1, 0] = (torch.arange(66000, device=DEV) % 7 < 2).float()
    for budget in ([33000, 33000], [32768, 18858], [65999, 1], [40000, 65999]):
        _evict_and_check(c, w, budget, 10, 10)
        for b in range(2):                                     # (in place: the rows behind have to be numbers that differ again)
            for x in (c.K, c.V):
                c.put(x, b, 0, c.randn(66000, 1, D).to(x.dtype))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv"])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 2048, 1024), (600, 4, 1), (5, 3, 3)])
def test_many_heads_or_requests(dtype, B, Hq, Hkv):
    lens = [70 - 13 * i % 70 for i in range(B)]
    news = [min(n, i % 3) for i, n in enumerate(lens)] if B > 1 else [1]
    c = CacheCase(dtype, Hq, Hkv, lens, 16, seed=B)
    check_window(c, news, 20, 3)
    check_window_step(c, 20, 3)
    check_mass(c, news, [n - t for t, n in zip(news, lens)], 0.75)
    check_mass_step(c, [n - 1 for n in lens], 0.75)
    _evict_and_check(c, _mass(c), [n // 2 for n in lens], 1, 2)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8kv"])
@pytest.mark.parametrize("news", [[900] + [1] * 31, [0] * 31 + [1024], [1025] + [0] * 31, [0] * 31 + [33], [32] * 32, [33] + [32] * 31])
def test_weights_of_one_prompt_among_single_tokens(dtype, news):
    """The batch has few tokens a request, and one request all of them; and the numbers at which the kernel's blocks change."""
    c = CacheCase(dtype, 4, 1, [max(t, 1) + 100 * (b % 3) for b, t in enumerate(news)], 16, seed=4)
    check_mass(c, news)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8kv", "fp8k"])
@pytest.mark.parametrize("layout", [0, 16])
@pytest.mark.parametrize("G", [1, 2, 4])
def test_steps_over_more_rows_than_the_caches_keep(dtype, layout, G):
    """Rows that are read past the caches: windows that take most of them, and all of them with their weights."""
    Hkv, n = 8, 20000
    B = -(-(300 << 20) // (Hkv * n * 128 * (2 if dtype == "fp8kv" else 3)))
    lens = [n - 37 * b for b in range(B)]
    c = CacheCase(dtype, Hkv * G, Hkv, lens, layout, seed=G)
    assert sum(min(m, 19900) for m in lens) * Hkv * 128 * sum(x.element_size() for x in (c.K, c.V)) > 288 << 20
    check_window_step(c, 19850, 50)
    check_mass_step(c, [m - 1 for m in lens], 0.5)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8kv"])
@pytest.mark.parametrize("layout", [0, 16])
def test_lengths_outside_the_cache_are_the_nearest_inside(dtype, layout):
    cap, news = 150, [4, 60, 3, 0]
    c = CacheCase(dtype, 4, 2, [cap] * 4, layout, seed=9)
    clean, runs = [raw(c.K).clone(), raw(c.V).clone()], []
    for lens in ([-5, cap + 1000, 2 ** 31 - 1, -2 ** 31], [0, cap, cap, 0]):
        c.seq.copy_(ints(lens))
        for x, y in zip((c.K, c.V), clean):
            raw(x).copy_(y)
        c.lens = [0, cap, cap, 0]
        runs.append(_everything(c, c.kv, news, 3)[:-1] + [raw(c.K).clone(), raw(c.V).clone()])
        held, mass = c.seq.clone(), torch.ones((4, 2, cap), device=DEV)
        c.ctx.lfps_attn_mass(torch.zeros((0, 4, D), dtype=c.q_dtype, device=DEV), ints([0] * 5), c.kv, mass, held=held, decay=0.5)
        runs[-1].append(mass)
    for a, b in zip(*runs):
        assert torch.equal(_bits(a), _bits(b))
    c.ctx.close()


def test_written_arrays_that_overlap_read_ones():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64], 16)
    T = 8
    room = torch.zeros(1 << 16, device=DEV)
    q, cu = torch.zeros((T, 4, D), dtype=torch.bfloat16, device=DEV), ints([0, T])
    k = torch.zeros((T, 4, D), dtype=torch.bfloat16, device=DEV)[:, :2]
    mass = room[:128].view(1, 2, 64)
    step, out = torch.zeros((1, 4, D), device=DEV), torch.zeros((1, 4, D), device=DEV)
    inside = lambda x: room[:256].view(torch.int32)[x:x + 1]  # noqa: E731
    seq = inside(127)
    seq.fill_(64)
    table = room.view(torch.int32)[120:124].view(1, 4)
    table.zero_()
    bad_kv = [c.ctx.paged_kv_view(c.K, c.V, c.table, seq), c.ctx.paged_kv_view(c.K, c.V, table, c.seq)]
    calls = [lambda: c.ctx.lfps_attn_mass(room.view(torch.bfloat16)[:T * 4 * D].view(T, 4, D), cu, c.kv, mass),
             lambda: c.ctx.lfps_attn_mass(q, room[126:128].view(torch.int32), c.kv, mass),
             lambda: c.ctx.lfps_attn_mass(q, cu, c.kv, mass, held=inside(0)),
             lambda: c.ctx.lfps_full_attn_mass_decode(step, c.kv, mass, out, held=inside(127))]
    for kv in bad_kv:
        calls += [lambda kv=kv: c.ctx.lfps_attn_mass(q, cu, kv, mass), lambda kv=kv: c.ctx.lfps_full_attn_mass_decode(step, kv, mass, out)]
    freq, weight = room[64:128], room[128:256]
    turned = room.view(torch.bfloat16)[:T * 4 * D].view(T, 4, D)
    fine = c.ctx.rotary(inv_freq=torch.ones(64, device=DEV))
    for rot, pos, at, kv in ((c.ctx.rotary(inv_freq=freq), None, cu, c.kv), (c.ctx.rotary(q_weight=weight), None, cu, c.kv), (c.ctx.rotary(k_weight=weight), None, cu, c.kv),
                             (fine, room.view(torch.int32)[2040:2048], cu, c.kv), (fine, None, room.view(torch.int32)[2046:2048], c.kv),
                             (c.ctx.rotary(inv_freq=torch.ones(64, device=DEV), pair_axis=room.view(torch.int32)[:64]), None, cu, c.kv),
                             (fine, None, cu, bad_kv[0]), (fine, None, cu, bad_kv[1])):
        calls.append(lambda rot=rot, pos=pos, at=at, kv=kv: c.ctx.lfps_rotate_append(rot, q, k, k, pos, at, kv, turned))
    other = CacheCase("bf16", 4, 2, [64], 16)
    i32 = lambda: torch.zeros((1, 2, 64), dtype=torch.int32, device=DEV)  # noqa: E731
    calls.append(lambda: c.ctx.lfps_evict(c.kv, torch.zeros_like(mass), ints([9]), 1, 1, mass, i32(), ints([0]),
                                          to=c.ctx.paged_kv_view(other.K, other.V, table, other.seq)))
    for i, call in enumerate(calls):
        with pytest.raises(LfpsError) as e:
            call()
        assert e.value.code == LFPS_EINVAL and "overlap" in str(e.value), i
    assert int(room.view(torch.int32).count_nonzero()) == 1    # (the length)
    c.ctx.close()
    other.ctx.close()
