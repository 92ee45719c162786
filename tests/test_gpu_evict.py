"""Eviction by accumulated weight: which rows stay, and every byte of the cache behind it."""
import pytest
import torch

from tests.cache_case import CacheCase, ints, raw
from tests.harness import DEV

pytestmark = pytest.mark.gpu

LAYOUTS = [0, 16, "rows", ("rows", 64)]


def _rows_to_keep(w, n, budget, n_sink, n_recent):
    """By the definition, one head: w a list of n weights."""
    m = min(n, max(0, budget))
    sinks = min(n_sink, m)
    recent = min(n_recent, m - sinks)
    between = sorted(range(sinks, n - recent), key=lambda j: (-(w[j] if w[j] == w[j] else float("-inf")), w[j] != w[j], j))
    return sorted(list(range(sinks)) + between[:m - sinks - recent] + list(range(n - recent, n)))


def _evict_and_check(c, mass, budget, n_sink, n_recent, to=None):
    """to: a second CacheCase of the same shapes that receives the rows."""
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
    shape = (c.B, c.Hkv, c.cap)
    mass_out, kept = torch.full(shape, 7.0, device=DEV), torch.full(shape, -7, dtype=torch.int32, device=DEV)
    lens_out = ints([-7] * c.B)
    target = to or c
    want = [raw(x).clone() for x in (target.K, target.V)]
    source = [raw(x).clone() for x in (c.K, c.V)]
    c.ctx.lfps_evict(c.kv, mass, ints(budget), n_sink, n_recent, mass_out, kept, lens_out, to=to.kv if to else None)
    w = mass.cpu()
    for b, n in enumerate(c.lens):
        for g in range(c.Hkv):
            keep = _rows_to_keep(w[b, g, :n].tolist(), n, budget[b], n_sink, n_recent)
            m = len(keep)
            assert int(lens_out[b]) == m
            assert kept[b, g, :m].tolist() == keep and bool((kept[b, g, m:] == -7).all()), (b, g)
            i = torch.tensor(keep, dtype=torch.long, device=DEV)
            assert torch.equal(mass_out[b, g, :m].view(torch.int32), mass[b, g][i].view(torch.int32)) and bool((mass_out[b, g, m:] == 7).all())
            if m:
                j = torch.arange(m, device=DEV)
                block, at = (c.table[b].long()[i // c.page], i % c.page) if c.page else (torch.full_like(i, b), i)
                block_to, at_to = (target.table[b].long()[j // c.page], j % c.page) if c.page else (torch.full_like(j, b), j)
                for x, old in zip(want, source):
                    x[block_to, g, at_to] = old[block, g, at]
    for x, y in zip((target.K, target.V), want):
        t = bits[x.element_size()]
        assert torch.equal(raw(x).contiguous().view(t), y.contiguous().view(t))
    if to:
        for x, y in zip((c.K, c.V), source):
            t = bits[x.element_size()]
            assert torch.equal(raw(x).contiguous().view(t), y.contiguous().view(t))


def _mass(c, ties=0.2):
    w = torch.exp(2 * c.randn(c.B, c.Hkv, c.cap))
    return (w * (torch.rand(w.shape, device=DEV, generator=c.gen) > ties)).contiguous()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_formats_and_layouts(dtype, layout):
    lens, budget = [70, 7, 0, 165, 433, 16], [30, 2, 4, 165, 200, 100]
    c, other = CacheCase(dtype, 4, 2, lens, layout, seed=1), CacheCase(dtype, 4, 2, lens, layout, seed=2)
    w = _mass(c)
    _evict_and_check(c, w, budget, 3, 10, to=other)
    _evict_and_check(c, w, budget, 3, 10)
    c.ctx.close()
    other.ctx.close()


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 127, 1023, 1024, 1025, 4096, 5003, 20011])
def test_lengths(n):
    c = CacheCase("bf16", 2, 2, [n], 16, seed=n)
    for budget, n_sink, n_recent in ((n // 2, 4, n // 8), (1, 0, 0), (n - 1, 1, 1), (max(1, n // 3), 0, n), (n, 2, 2)):
        _evict_and_check(c, _mass(c), [budget], n_sink, n_recent)
    c.ctx.close()


@pytest.mark.parametrize("budget,n_sink,n_recent", [(0, 4, 4), (-3, 0, 0), (3, 4, 4), (4, 4, 4), (6, 4, 4), (8, 4, 4), (9, 4, 4), (50, 0, 0), (50, 100, 100),
                                                    (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), (40, 2 ** 31 - 1, 3), (40, 3, 2 ** 31 - 1)])
def test_budgets_first_rows_and_newest_rows(budget, n_sink, n_recent):
    c = CacheCase("f32", 1, 1, [100], seed=3)
    _evict_and_check(c, _mass(c), [budget], n_sink, n_recent)
    c.ctx.close()


def test_weights_that_are_equal_or_no_numbers():
    n = 300
    c = CacheCase("bf16", 8, 8, [n], 16, seed=4)
    w = torch.zeros((1, 8, n), device=DEV)
    w[0, 1] = 1.0                                                        # all the same
    w[0, 2, ::2] = -0.0                                                  # zeros of both signs are equal
    w[0, 3] = float("nan")
    w[0, 4] = c.randn(n)                                                 # negative ones
    w[0, 4, ::7], w[0, 4, 1::7], w[0, 4, 2::7] = float("nan"), float("-inf"), float("inf")
    w[0, 5] = torch.arange(n, device=DEV) % 5
    w[0, 6] = 1.0 + (torch.arange(n, device=DEV) % 3) * 2.0 ** -23       # neighbours in the last bit
    w[0, 7] = (torch.arange(n, device=DEV) % 11) * 2.0 ** -149           # below the normal numbers
    for budget in (1, 100, 150, 299):
        c.lens = [n]
        _evict_and_check(c, w, [budget], 2, 5)
    c.ctx.close()


def test_many_requests_and_heads():
    lens = [1 + 37 * i % 500 for i in range(60)]
    c = CacheCase("fp8kv", 6, 3, lens, 16, seed=9)
    _evict_and_check(c, _mass(c), [max(1, n * (i % 9) // 7) for i, n in enumerate(lens)], 4, 20)
    c.ctx.close()


def test_blocks_of_the_same_pool_receive_the_rows():
    """A prefix that two requests share stays as it is; each gets its rows in blocks of its own."""
    c = CacheCase("bf16", 2, 1, [100, 100], 16, seed=10, spare=20)
    c.table[1] = c.table[0]
    free = [i for i in range(c.n_blocks) if i not in c.table[0].tolist()]
    table = ints(free[:14]).view(2, 7)
    to = c.ctx.paged_kv_view(c.K, c.V, table, c.seq)
    w = _mass(c)
    w[1] = w[0].flip(-1)
    old = [c.get(x, 0, 0, 100) for x in (c.K, c.V)]
    mass_out, kept, lens_out = torch.zeros_like(w), torch.zeros((2, 1, 100), dtype=torch.int32, device=DEV), ints([0, 0])
    c.ctx.lfps_evict(c.kv, w, ints([40, 50]), 4, 8, mass_out, kept, lens_out, to=to)
    shared = c.table
    for x, y in zip((c.K, c.V), old):
        assert torch.equal(c.get(x, 0, 0, 100), y)
    c.table = table
    for b, m in ((0, 40), (1, 50)):
        i = torch.tensor(_rows_to_keep(w[b, 0].tolist(), 100, m, 4, 8), device=DEV)
        for x, y in zip((c.K, c.V), old):
            assert torch.equal(c.get(x, b, 0, m), y[i])
    assert lens_out.tolist() == [40, 50] and shared is not table
    c.ctx.close()


def test_rows_whose_table_entry_is_no_block_are_dropped():
    c, other = CacheCase("bf16", 2, 1, [100], 16, seed=11), CacheCase("bf16", 2, 1, [100], 16, seed=12)
    other.table[0, 1], other.table[0, 0] = -1, other.n_blocks
    before = other.K.clone()
    w = _mass(c)
    mass_out, kept, lens_out = torch.zeros_like(w), torch.zeros((1, 1, 100), dtype=torch.int32, device=DEV), ints([0])
    c.ctx.lfps_evict(c.kv, w, ints([40]), 4, 8, mass_out, kept, lens_out, to=other.view())
    mine = int(other.table[0, 2])
    rest = [i for i in range(other.n_blocks) if i != mine]
    assert torch.equal(other.K[rest].view(torch.int16), before[rest].view(torch.int16))
    assert torch.equal(other.K[mine, 0, :8], c.get(c.K, 0, 0, 100)[kept[0, 0, 32:40].long(), 0])
    c.ctx.close()
    other.ctx.close()


def test_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64])
    f, i = (lambda: torch.zeros((1, 2, 64), device=DEV)), (lambda: torch.zeros((1, 2, 64), dtype=torch.int32, device=DEV))
    ok = dict(kv=c.kv, mass=f(), budget=ints([10]), n_sink=1, n_recent=1, mass_out=f(), kept=i(), lens_out=ints([0]))
    call = lambda **bad: c.ctx.lfps_evict(**{**ok, **bad})  # noqa: E731
    call()
    for bad in (dict(mass=i()), dict(kept=f()), dict(budget=f().view(-1)[:1])):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(mass=f()[:, :1]), dict(lens_out=ints([0, 0])), dict(kept=i()[..., :32])):
        with pytest.raises(ValueError):
            call(**bad)
    m = ok["mass"]
    for bad, word in ((dict(n_sink=-1), "n_sink"), (dict(n_recent=-1), "n_recent"), (dict(mass_out=m), "overlap"), (dict(kept=m.view(torch.int32)), "overlap"),
                      (dict(lens_out=c.seq), "overlap"), (dict(lens_out=ok["budget"]), "overlap"), (dict(lens_out=ok["kept"].view(-1)[3:4]), "overlap"),
                      (dict(kept=ok["mass_out"].view(torch.int32)), "overlap"), (dict(kv=c.ctx.kv_view(c.K, None, c.seq)), "kv->v"),
                      (dict(to=c.ctx.kv_view(c.K, c.V, c.seq)), "in place"), (dict(to=c.ctx.kv_view(c.K.clone(), c.V, c.seq)), "in place")):
        with pytest.raises(LfpsError) as e:
            call(**bad)
        assert e.value.code == LFPS_EINVAL and word in str(e.value), bad.keys()
    c.ctx.close()
