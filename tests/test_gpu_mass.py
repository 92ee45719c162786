"""Accumulated attention weights, of packed tokens and of a decode step, against plain forms in 64 bits."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints, packed, raw
from tests.harness import DEV

pytestmark = pytest.mark.gpu

LAYOUTS = [0, 16, "rows", ("rows", 64)]


def _weights(x, rows, K):
    """x [M, D] at cache rows `rows`: softmax over the rows up to them, and per query the largest sum of |q||k| / sqrt(D)."""
    end = int(rows.max()) + 1
    seen = torch.arange(end, device=DEV) <= rows.view(-1, 1)
    s = (x @ K[:end].T.contiguous() / D ** 0.5).masked_fill(~seen, float("-inf"))
    dots = (x.abs() @ K[:end].abs().T.contiguous() / D ** 0.5).masked_fill(~seen, 0).amax(1, keepdim=True)
    return torch.softmax(s, 1), dots


def _relative(dots, n):
    """Of a weight: its score and that of the largest, sums of 128 exact products in fp32 (twice: the row's sum has them too), the factor to powers of
    two, the exponential 2^-21, and the row's sum over n keys."""
    return 2 * 132 * 2.0 ** -24 * dots + 2.0 ** -21 + (n + 8) * 2.0 ** -24


def _check_mass(c, got, before, held, decay, terms):
    """terms(b, g) -> (sum of weights [n], what it may be off by [n], how many weights)."""
    for b, n in enumerate(c.lens):
        assert torch.equal(got[b, :, n:], before[b, :, n:])
        for g in range(c.Hkv):
            if n == 0:
                continue
            total, off, count = terms(b, g)
            h = min(n, max(0, held[b])) if held is not None else 0
            old = torch.zeros(n, dtype=torch.float64, device=DEV)
            old[:h] = before[b, g, :h].double() * float(torch.tensor(decay, dtype=torch.float32))
            tol = off + (count + 4) * 2.0 ** -24 * total + 2.0 ** -23 * old.abs() + 1e-30
            err = (got[b, g, :n].double() - (old + total)).abs()
            assert bool((err <= tol).all()), (b, g, float((err / tol).max()), float(err.max()))


def _tokens(c, news, held=None, decay=1.0, lead=0, extra=0, q=None):
    at = [lead + x for x in packed(news)]
    T = at[-1] + extra
    wide = c.randn(T, c.Hq + 3, D).to(c.q_dtype)
    if q is not None:
        wide[:, :c.Hq] = q
    q = wide[:, :c.Hq]
    mass = c.randn(c.B, c.Hkv, c.cap).abs()
    before = mass.clone()
    c.ctx.lfps_attn_mass(q, ints(at), c.kv, mass, held=None if held is None else ints(held), decay=decay)
    return at, q, mass, before


def _check(c, news, held=None, decay=1.0, **kw):
    at, q, mass, before = _tokens(c, news, held, decay, **kw)

    def terms(b, g):
        n, t = c.lens[b], news[b]
        K = c.values(c.K, b, 0, n)[g]
        total, off = (torch.zeros(n, dtype=torch.float64, device=DEV) for _ in range(2))
        for i0 in range(max(0, t - n), t, 512):
            i1 = min(t, i0 + 512)
            for h in range(g * c.G, g * c.G + c.G):
                w, dots = _weights(q[at[b] + i0:at[b] + i1, h].double(), torch.arange(n - t + i0, n - t + i1, device=DEV), K)
                total[:w.shape[1]] += w.sum(0)
                off[:w.shape[1]] += (w * _relative(dots, n)).sum(0)
        return total, off, t * c.G

    _check_mass(c, mass, before, held, decay, terms)


def _check_step(c, held=None, decay=1.0, q=None):
    q = c.randn(c.B, c.Hq, D) if q is None else q
    out, mass = torch.full((c.B, c.Hq, D), 7.0, device=DEV), c.randn(c.B, c.Hkv, c.cap).abs()
    before = mass.clone()
    c.ctx.lfps_full_attn_mass_decode(q, c.kv, mass, out, held=None if held is None else ints(held), decay=decay)

    def terms(b, g):
        n = c.lens[b]
        K, V = (c.values(x, b, 0, n)[g] for x in (c.K, c.V))
        w, dots = _weights(q[b, g * c.G:g * c.G + c.G].double(), torch.full((c.G,), n - 1, device=DEV), K)
        ref, weighted = w @ V, w @ V.abs()
        err = (out[b, g * c.G:g * c.G + c.G].double() - ref).abs()
        assert bool((err <= (_relative(dots, n) + (n + 8) * 2.0 ** -24) * weighted + 1e-7).all()), (b, g, float(err.max()))
        return w.sum(0), (w * _relative(dots, n)).sum(0), c.G

    _check_mass(c, mass, before, held, decay, terms)
    for b, n in enumerate(c.lens):
        assert n or not bool(out[b].any())


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_formats_and_layouts(dtype, layout):
    c = CacheCase(dtype, 8, 2, [70, 91, 5, 97, 300, 0], layout, seed=1)
    _check(c, [70, 1, 0, 33, 129, 0], [0, 90, 5, 64, 171, 0], 0.5, lead=3, extra=5)
    _check_step(c, [69, 90, 5, 0, 1000, 3], 0.5)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,news,lens", [
    (1, 1, [1], [1]), (4, 1, [8], [8]), (4, 1, [9], [9]), (2, 2, [31, 32, 33], [31, 32, 33]), (2, 1, [63, 64, 65, 16, 17], [63, 64, 65, 1000, 1000]),
    (8, 8, [127, 128, 129], [127, 128, 200]), (12, 3, [257], [700]), (4, 4, [1, 1, 1], [1, 64, 65]), (4, 1, [0, 3], [400, 3])])
def test_edges_of_tiles_and_heads(dtype, Hq, Hkv, news, lens):
    c = CacheCase(dtype, Hq, Hkv, lens, seed=Hq + len(news))
    _check(c, news)
    _check(c, news, [n - t for t, n in zip(news, lens)], 0.9)
    _check_step(c)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("news,lens", [([5], [5003]), ([1, 8, 3], [4000, 129, 2111]), ([40, 2], [3001, 1500]), ([200, 1, 0, 7], [2500, 1, 0, 3000])])
def test_few_tokens_over_long_caches(dtype, news, lens):
    c = CacheCase(dtype, 4, 1, lens, 16, seed=5)
    _check(c, news, [n - t for t, n in zip(news, lens)])
    _check_step(c, [n - 1 for n in lens])
    c.ctx.close()


def test_thousands_of_tokens():
    c = CacheCase("bf16", 4, 1, [2100, 900, 4097], 64, seed=2)
    _check(c, [2100, 777, 1500])
    c.ctx.close()


def test_many_requests():
    lens = [1 + 37 * i % 900 for i in range(60)]
    c = CacheCase("bf16", 4, 2, lens, 16, seed=9)
    _check(c, [min(n, 1 + i % 5) for i, n in enumerate(lens)])
    _check_step(c, [n - 1 for n in lens])
    c.ctx.close()


def test_tokens_without_a_row_count_nowhere():
    c = CacheCase("bf16", 4, 2, [3, 150, 0], seed=3)
    _check(c, [9, 200, 6], [1, 2, 0])
    c.ctx.close()


def test_more_query_rows_than_the_workspace_has_room_for():
    """The tokens are taken in several turns, each of which adds to the ones before."""
    n, Hq = 1500, 4096
    c = CacheCase("bf16", Hq, Hq, [n], seed=13)
    q = c.randn(n, 1, D).to(torch.bfloat16).expand(n, Hq, D).contiguous()
    c.K.copy_(c.K[:, :1].expand_as(c.K).clone())
    mass = torch.full((1, Hq, n), 7.0, device=DEV)
    c.ctx.lfps_attn_mass(q, ints([0, n]), c.kv, mass)
    K = c.values(c.K, 0, 0, n)[0]
    w, dots = _weights(q[:, 0].double(), torch.arange(n, device=DEV), K)
    tol = (w * _relative(dots, n)).sum(0) + (n + 4) * 2.0 ** -24 * w.sum(0)
    assert bool(((mass[0].double() - w.sum(0)).abs() <= tol).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_far_apart(dtype):
    n = 700
    c = CacheCase(dtype, 2, 1, [n], seed=4)
    for i in range(0, n, 50):
        c.K[0, 0, i] *= 1 + i / 25
    _check(c, [n], q=(4 * c.randn(n, 2, D)).to(c.q_dtype))
    _check_step(c, q=4 * c.randn(1, 2, D))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8kv"])
def test_the_weights_of_a_token_make_one(dtype):
    """All rows' masses together: a token's weights add up to 1 for every head."""
    c = CacheCase(dtype, 8, 2, [513, 200], 16, seed=15)
    _, _, mass, _ = _tokens(c, [300, 7])
    step, out = torch.zeros_like(mass), torch.zeros((2, 8, D), device=DEV)
    c.ctx.lfps_full_attn_mass_decode(c.randn(2, 8, D), c.kv, step, out)
    for b, (t, n) in enumerate(((300, 513), (7, 200))):
        # (the rounded sum in the weights' place is off as they are; what is added up here, by a rounding each)
        assert bool(((mass[b, :, :n].double().sum(1) - 4 * t).abs() <= 4 * t * (2.0 ** -19 + 3 * (n + 4 * t) * 2.0 ** -24)).all())
        assert bool(((step[b, :, :n].double().sum(1) - 4).abs() <= 4 * (2.0 ** -19 + 3 * n * 2.0 ** -24)).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
def test_what_is_not_finite_counts_where_it_is_seen(dtype):
    """A NaN key makes the weights of the tokens behind it NaN, and with them the masses of all rows that these see; the heads' groups and the
    requests stay apart.  Values do not matter."""
    c = CacheCase(dtype, 4, 2, [200, 90], 16, seed=16)
    q = c.randn(150, 4, D).to(c.q_dtype)
    raw(c.V).fill_(float("nan") if c.vd.itemsize > 1 else 127)
    runs = []
    for spoilt in (False, True):
        if spoilt:
            k = c.get(c.K, 0, 180, 181).to(torch.float32)
            k[0, 1, 5] = float("nan")
            c.put(c.K, 0, 180, k.to(c.kd))
        runs.append(torch.zeros((2, 2, 200), device=DEV))
        c.ctx.lfps_attn_mass(q, ints([0, 100, 150]), c.kv, runs[-1])
    assert torch.equal(runs[0][:, 0], runs[1][:, 0]) and torch.equal(runs[0][1], runs[1][1]) and bool(runs[0].isfinite().all())
    assert bool(runs[1][0, 1].isnan().all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("G,t,n", [(4, 20, 300), (4, 32, 32), (1, 100, 500), (2, 300, 700), (4, 600, 600)])
def test_a_query_of_nan_counts_for_the_rows_it_sees(dtype, G, t, n):
    """Few tokens, which a kernel of their own takes, and many: the rows behind the token's have what they have without it, to the last bit."""
    c = CacheCase(dtype, 2 * G, 2, [n, 50], 16, seed=G)
    q = c.randn(t + 3, 2 * G, D).to(c.q_dtype)
    at, runs = t // 2, []
    for spoilt in (False, True):
        if spoilt:
            q[at, G:] = float("nan")                                     # (the second KV head's)
        runs.append(torch.zeros((2, 2, c.cap), device=DEV))
        c.ctx.lfps_attn_mass(q, ints([0, t, t + 3]), c.kv, runs[-1])
    sees = n - t + at + 1
    assert bool(runs[0].isfinite().all()) and torch.equal(runs[0][:, 0], runs[1][:, 0]) and torch.equal(runs[0][1], runs[1][1])
    assert bool(runs[1][0, 1, :sees].isnan().all()) and torch.equal(runs[0][0, 1, sees:], runs[1][0, 1, sees:])
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8k", "f32"])
@pytest.mark.parametrize("Hq,news,lens,held", [(4, [9, 5, 3, 0], [3, 20, 0, 8], [1, 17, 0, 8]), (1, [128, 1], [200, 1], [72, 0]), (2, [64, 65], [64, 300], [0, 235]),
                                               (4, [32, 33, 1], [32, 129, 5000], [0, 96, 4999]), (4, [64, 65, 1], [3000, 70, 1], [2936, 5, 0]), (2, [128], [128], [0])])
def test_few_tokens_of_some_requests(dtype, Hq, news, lens, held):
    """Tokens at no row, one block of queries and a row more, requests of few tokens beside others."""
    c = CacheCase(dtype, Hq, 1, lens, 16, seed=len(news) + Hq)
    _check(c, news, held, 0.5, lead=1, extra=2)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_of_minus_infinity_weigh_nothing_to_few_tokens(dtype):
    n = 100
    c = CacheCase(dtype, 1, 1, [n], seed=6)
    c.K[..., 5] = 0
    c.K[0, 0, :40, 5] = float("-inf")
    q = c.randn(n, 1, D).to(c.q_dtype)
    q[..., 5] = 1.0
    mass = torch.full((1, 1, n), 7.0, device=DEV)
    c.ctx.lfps_attn_mass(q, ints([0, n]), c.kv, mass)
    assert not bool(mass[0, 0, :40].any()) and bool((mass[0, 0, 40:] > 0).all())
    assert abs(float(mass.double().sum()) - 60) <= 60 * (2.0 ** -19 + 3 * 2 * n * 2.0 ** -24)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("G,t", [(1, 3), (1, 33), (1, 100), (2, 50), (4, 1), (4, 3), (4, 8), (4, 40), (4, 59)])
def test_infinite_keys_weigh_nothing_to_few_tokens_far_behind_them(dtype, sign, G, t):
    """All tokens see all of these keys; the last block of 32 query rows is full, or is not."""
    n = 500
    c = CacheCase(dtype, 2 * G, 2, [n, 9], seed=t)
    c.K[..., 5] = 0
    hidden = torch.zeros(n, dtype=torch.bool, device=DEV)
    hidden[:40] = hidden[100:131] = hidden[300] = True
    c.K[0, :, :n, 5] = torch.where(hidden, -sign * float("inf"), 0.0).to(c.kd)
    q = c.randn(t + 9, 2 * G, D).to(c.q_dtype)
    q[..., 5] = sign
    mass = torch.full((2, 2, n), 7.0, device=DEV)
    c.ctx.lfps_attn_mass(q, ints([0, t, t + 9]), c.kv, mass)
    j = torch.arange(n, device=DEV)[~hidden]
    for g in range(2):
        assert not bool(mass[0, g, hidden].any())
        K = c.values(c.K, 0, 0, n)[g][j]
        x = q[:t, g * G:g * G + G].double().reshape(t * G, D)
        unseen = j > torch.arange(n - t, n, device=DEV).repeat_interleave(G).view(-1, 1)
        w = torch.softmax((x @ K.T.contiguous() / D ** 0.5).masked_fill(unseen, float("-inf")), 1)
        dots = (x.abs() @ K.abs().T.contiguous() / D ** 0.5).masked_fill(unseen, 0).amax(1, keepdim=True)
        tol = (w * _relative(dots, n)).sum(0) + (t * G + 4) * 2.0 ** -24 * w.sum(0) + 1e-30
        assert bool(((mass[0, g, j].double() - w.sum(0)).abs() <= tol).all())
    assert bool(mass[1, :, :9].isfinite().all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_of_minus_infinity_weigh_nothing(dtype):
    n = 150
    c = CacheCase(dtype, 1, 1, [n], seed=6)
    c.K[..., 5] = 0
    c.K[0, 0, :90, 5] = float("-inf")
    q = c.randn(n, 1, D).to(c.q_dtype)
    q[..., 5] = 1.0
    mass = torch.full((1, 1, n), 7.0, device=DEV)
    c.ctx.lfps_attn_mass(q, ints([0, n]), c.kv, mass)
    assert not bool(mass[0, 0, :90].any()) and bool((mass[0, 0, 90:] > 0).all())      # (tokens that see no other row weigh nothing anywhere)
    assert abs(float(mass.double().sum()) - 60) <= 60 * (2.0 ** -19 + 3 * 2 * n * 2.0 ** -24)
    c.ctx.close()


def test_no_tokens_at_all():
    """What is held decays, the rest is zero."""
    c = CacheCase("bf16", 4, 2, [40, 0, 7], 16)
    mass = torch.full((3, 2, 40), 8.0, device=DEV)
    c.ctx.lfps_attn_mass(torch.zeros((0, 4, D), dtype=torch.bfloat16, device=DEV), ints([0, 0, 0, 0]), c.kv, mass, held=ints([30, 0, 100]), decay=0.25)
    want = torch.full((3, 2, 40), 8.0, device=DEV)
    want[0, :, :30], want[0, :, 30:], want[2, :, :7] = 2.0, 0.0, 2.0
    assert torch.equal(mass, want)
    c.ctx.close()


def test_the_same_sums_every_time():
    c = CacheCase("bf16", 8, 2, [900, 333], 16, seed=17)
    q, qs = c.randn(700, 8, D).to(torch.bfloat16), c.randn(2, 8, D)
    runs = []
    for _ in range(3):
        mass, step, out = torch.zeros((2, 2, 900), device=DEV), torch.zeros((2, 2, 900), device=DEV), torch.zeros((2, 8, D), device=DEV)
        c.ctx.lfps_attn_mass(q, ints([0, 500, 700]), c.kv, mass)
        c.ctx.lfps_full_attn_mass_decode(qs, c.kv, step, out)
        runs.append((mass, step, out))
    for r in runs[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, runs[0]))
    c.ctx.close()


def test_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64])
    q, cu, mass = torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV), ints([0, 8]), torch.zeros((1, 2, 64), device=DEV)
    ok, step = dict(q=q, cu=cu, kv=c.kv, mass=mass), dict(q=q[:1].float(), kv=c.kv, mass=mass, out=torch.zeros((1, 4, D), device=DEV))
    for bad in (dict(q=q.float()), dict(mass=mass.half()), dict(held=mass.view(-1)[:1])):
        with pytest.raises(TypeError):
            c.ctx.lfps_attn_mass(**{**ok, **bad})
    for bad in (dict(mass=mass[:, :1]), dict(cu=ints([0, 4, 8])), dict(held=ints([0, 0]))):
        with pytest.raises(ValueError):
            c.ctx.lfps_attn_mass(**{**ok, **bad})
    for bad in (dict(decay=1.5), dict(decay=-0.1), dict(decay=float("nan"))):
        for call, good in ((c.ctx.lfps_attn_mass, ok), (c.ctx.lfps_full_attn_mass_decode, step)):
            with pytest.raises(LfpsError) as e:
                call(**{**good, **bad})
            assert e.value.code == LFPS_EINVAL and "decay" in str(e.value)
    odd = torch.zeros(129, device=DEV)[1:].view(1, 2, 64)
    for call, good in ((c.ctx.lfps_attn_mass, ok), (c.ctx.lfps_full_attn_mass_decode, step)):
        with pytest.raises(LfpsError) as e:
            call(**{**good, "mass": odd})
        assert "aligned" in str(e.value)
    for bad in (dict(out=step["q"]), dict(mass=step["q"].view(-1)[:128].view(1, 2, 64)), dict(mass=step["out"].view(-1)[:128].view(1, 2, 64))):
        with pytest.raises(LfpsError) as e:
            c.ctx.lfps_full_attn_mass_decode(**{**step, **bad})
        assert "overlap" in str(e.value)
    no_v = c.ctx.kv_view(c.K, None, c.seq)
    c.ctx.lfps_attn_mass(**{**ok, "kv": no_v})                     # keys are enough
    with pytest.raises(LfpsError):
        c.ctx.lfps_full_attn_mass_decode(**{**step, "kv": no_v})
    c.ctx.close()


def test_arrays_that_make_no_sense():
    c = CacheCase("bf16", 4, 2, [64, 64, 64, 64], 16)
    q = torch.zeros((40, 4, D), dtype=torch.bfloat16, device=DEV)
    guard = torch.full((4 * 2 * 64 + 128,), 7.0, device=DEV)
    for cu in ([0, 500, -3, 10, 40], [40, 30, 20, 10, 0], [-100, -50, 2000000000, 5, 7]):
        c.ctx.lfps_attn_mass(q, ints(cu), c.kv, guard[64:-64].view(4, 2, 64), held=ints([-2 ** 31, 2 ** 31 - 1, -1, 65]))
        assert bool((guard[:64] == 7).all()) and bool((guard[-64:] == 7).all())
    c.ctx.close()
