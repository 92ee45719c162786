"""Attention over a sliding window and the first rows, of packed tokens and of a decode step, against plain forms in 64 bits."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints, packed, raw, to_cache
from tests.harness import DEV

pytestmark = pytest.mark.gpu

LAYOUTS = [0, 16, "rows", ("rows", 64)]


def _tolerance(dtype, ref, weighted, dots, n):
    """Scores are sums of 128 exact products in fp32 (2^-24 of the absolute sum each), weights and their sum follow them (twice); 16-bit
    weights are off by half a step each, and so is the output; sums over n keys in fp32; the exponential 2^-21.  dtype None: fp32 results."""
    half = {"f16": 2.0 ** -11, "f32": 0.0, None: 0.0}.get(dtype, 2.0 ** -8)
    return half * 1.01 * (ref.abs() + weighted) + (2 * 130 * 2.0 ** -24 * dots + 2.0 ** -21 + (n + 8) * 2.0 ** -24) * weighted + 1e-7


def _reference(x, rows, K, V, window, n_sink):
    """x [M, D] at cache rows `rows`: output, weighted |V| and the largest sum of |q||k| / sqrt(D) over the seen keys."""
    end = int(rows.max()) + 1
    j, p = torch.arange(end, device=DEV), rows.view(-1, 1)
    seen = (j <= p) & ((j > p - window) | (j < n_sink))
    s = (x @ K[:end].T.contiguous() / D ** 0.5).masked_fill(~seen, float("-inf"))
    w = torch.softmax(s, 1)
    dots = (x.abs() @ K[:end].abs().T.contiguous() / D ** 0.5).masked_fill(~seen, 0).amax(1, keepdim=True)
    return w @ V[:end], w @ V[:end].abs(), dots


def _tokens(c, news, window, n_sink, q=None, lead=0, extra=0):
    at = [lead + x for x in packed(news)]
    T = at[-1] + extra
    wide = c.randn(T, c.Hq + 3, D).to(c.q_dtype)          # q as a slice of something wider
    if q is not None:
        wide[:, :c.Hq] = q
    q = wide[:, :c.Hq]
    out = torch.full((T, c.Hq, D), 7.0, dtype=c.q_dtype, device=DEV)
    c.ctx.lfps_window_attn(q, ints(at), c.kv, window, n_sink, out)
    return at, q, out


def _check(c, news, window, n_sink, **kw):
    at, q, out = _tokens(c, news, window, n_sink, **kw)
    assert bool((out[:at[0]] == 7).all()) and bool((out[at[-1]:] == 7).all())
    for b, t in enumerate(news):
        n = c.lens[b]
        first = max(0, t - n)                              # tokens at no row: zeros
        if t == 0:
            continue
        assert not bool(out[at[b]:at[b] + first].any())
        K, V = (c.values(x, b, 0, n) for x in (c.K, c.V))
        for h in range(c.Hq):
            for i0 in range(first, t, 512):
                i1 = min(t, i0 + 512)
                rows = torch.arange(n - t + i0, n - t + i1, device=DEV)
                ref, weighted, dots = _reference(q[at[b] + i0:at[b] + i1, h].double(), rows, K[h // c.G], V[h // c.G], window, n_sink)
                err = (out[at[b] + i0:at[b] + i1, h].double() - ref).abs()
                assert bool((err <= _tolerance(c.dtype, ref, weighted, dots, min(n, window + n_sink))).all()), (b, h, i0, float(err.max()))


def _check_step(c, window, n_sink, q=None):
    q = c.randn(c.B, c.Hq, D) if q is None else q
    out = torch.full((c.B, c.Hq, D), 7.0, device=DEV)
    c.ctx.lfps_window_attn_decode(q, c.kv, window, n_sink, out)
    for b, n in enumerate(c.lens):
        if n == 0:
            assert not bool(out[b].any())
            continue
        K, V = (c.values(x, b, 0, n) for x in (c.K, c.V))
        for h in range(c.Hq):
            ref, weighted, dots = _reference(q[b, h].double().view(1, D), torch.tensor([n - 1], device=DEV), K[h // c.G], V[h // c.G], window, n_sink)
            err = (out[b, h].double() - ref[0]).abs()
            assert bool((err <= _tolerance(None, ref, weighted, dots, min(n, window + n_sink))[0]).all()), (b, h, float(err.max()))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_formats_and_layouts(dtype, layout):
    c = CacheCase(dtype, 8, 2, [70, 91, 5, 97, 300], layout, seed=1)
    _check(c, [70, 1, 0, 33, 129], 50, 3, lead=3, extra=5)
    _check_step(c, 50, 3)
    c.ctx.close()


WINDOWS = [(1, 0), (1, 1), (2, 0), (63, 0), (64, 5), (65, 64), (100, 200), (128, 1), (129, 70), (1000, 4), (5000, 0), (2 ** 31 - 1, 2 ** 31 - 1)]


@pytest.mark.parametrize("window,n_sink", WINDOWS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_and_sinks(dtype, window, n_sink):
    c = CacheCase(dtype, 4, 1, [700, 64, 333], 16, seed=window % 1000)
    _check(c, [700, 64, 130], window, n_sink)
    _check_step(c, window, n_sink)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,news,lens", [
    (1, 1, [1], [1]), (4, 1, [8], [8]), (4, 1, [9], [9]), (2, 2, [31, 32, 33], [31, 32, 33]), (2, 1, [63, 64, 65, 16, 17], [63, 64, 65, 1000, 1000]),
    (8, 8, [127, 128, 129], [127, 128, 200]), (12, 3, [257], [700]), (4, 4, [1, 1, 1], [1, 64, 65])])
def test_edges_of_tiles_and_heads(dtype, Hq, Hkv, news, lens):
    c = CacheCase(dtype, Hq, Hkv, lens, seed=Hq + len(news))
    _check(c, news, 40, 2)
    _check_step(c, 40, 2)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("news,lens", [([5], [5003]), ([1, 8, 3], [4000, 129, 2111]), ([40, 2], [3001, 1500]), ([200, 1, 0, 7], [2500, 1, 0, 3000])])
def test_few_tokens_over_long_caches(dtype, news, lens):
    c = CacheCase(dtype, 4, 1, lens, 16, seed=5)
    _check(c, news, 1500, 33)
    _check_step(c, 1500, 33)
    c.ctx.close()


@pytest.mark.parametrize("layout", [0, 16, 64])
def test_thousands_of_tokens(layout):
    c = CacheCase("bf16", 4, 1, [2100, 900, 4097], layout, seed=2)
    _check(c, [2100, 777, 1500], 517, 37)
    c.ctx.close()


def test_many_requests_of_few_tokens():
    lens = [1 + 37 * i % 900 for i in range(60)]
    news = [min(n, 1 + i % 5) for i, n in enumerate(lens)]
    c = CacheCase("bf16", 4, 2, lens, 16, seed=9)
    _check(c, news, 100, 4)
    _check_step(c, 100, 4)
    c.ctx.close()


def test_tokens_without_a_row_get_zeros():
    c = CacheCase("bf16", 4, 2, [3, 150, 0], seed=3)
    _check(c, [9, 200, 6], 20, 1)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_scores_far_apart(dtype):
    n = 700
    c = CacheCase(dtype, 2, 1, [n], seed=4)
    for i in range(0, n, 50):
        c.K[0, 0, i] *= 1 + i / 25
    _check(c, [n], 120, 4, q=(4 * c.randn(n, 2, D)).to(c.q_dtype))
    _check_step(c, 120, 4, q=4 * c.randn(1, 2, D))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_wide_window_is_all_rows(dtype):
    """Close to what lfps_prompt_attn and lfps_full_attn_decode give; a window of one row: that row's values."""
    c = CacheCase(dtype, 4, 2, [300, 41], 16, seed=12)
    at, q, out = _tokens(c, [120, 41], 300, 0)
    same = torch.zeros_like(out)
    c.ctx.lfps_prompt_attn(q, ints(at), c.kv, same)
    half = {"f16": 2.0 ** -11, "f32": 2.0 ** -20}.get(dtype, 2.0 ** -8)
    assert bool(((out - same).abs().float() <= 4.2 * half * max(float(c.values(c.V, b, 0, n).abs().max()) for b, n in enumerate(c.lens))).all())
    one = _tokens(c, [120, 41], 1, 0)[2]
    for b in range(2):
        v = c.values(c.V, b, c.lens[b] - [120, 41][b], c.lens[b]).transpose(0, 1).repeat_interleave(2, 1)
        assert torch.equal(one[at[b]:at[b + 1]].double(), v)
    c.ctx.close()


def _same_where_not_finite(got, ref, tol):
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
    assert torch.equal(got[ref.isinf()].sign(), ref[ref.isinf()].sign())
    fine = ref.isfinite()
    assert bool(((got - ref).abs()[fine] <= tol.expand_as(ref)[fine]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8v", "fp8kv"])
@pytest.mark.parametrize("Hq,news,lens", [(1, [200], [200]), (4, [300], [333]), (4, [5], [400]), (2, [1, 70], [64, 129])])
@pytest.mark.parametrize("window,n_sink", [(20, 0), (70, 3)])
def test_values_that_are_not_finite_reach_only_the_tokens_that_see_them(dtype, Hq, news, lens, window, n_sink):
    c = CacheCase(dtype, Hq, 1, lens, seed=8)
    bad = float("nan") if c.vd.itemsize == 1 else float("inf")
    for b, n in enumerate(lens):
        for row, ch, x in ((n - 1, 3, bad), (n - 2, 77, float("nan")), (n // 2, 64, bad), (n // 2 + 1, 127, -bad), (1, 9, bad), (4, 10, bad),
                           (max(0, n - 30), 50, bad), (max(0, n - 75), 51, float("nan"))):
            v = c.V[b, 0].to(torch.float32)
            v[row, ch] = x
            raw(c.V)[b, 0] = raw(to_cache(v, c.vd) if x == x or c.vd.itemsize > 1 else v.to(c.vd))
    at, q, out = _tokens(c, news, window, n_sink)
    qs, outs = c.randn(c.B, Hq, D), torch.zeros((c.B, Hq, D), device=DEV)
    c.ctx.lfps_window_attn_decode(qs, c.kv, window, n_sink, outs)
    for b, t in enumerate(news):
        n = lens[b]
        K, V = c.values(c.K, b, 0, n)[0], c.V[b, 0].to(torch.float32).double()
        for h in range(Hq):
            todo = [(q[at[b] + i, h], n - t + i, out[at[b] + i, h], dtype) for i in range(0, t, 1 + t // 60)] + [(qs[b, h], n - 1, outs[b, h], None)]
            for x, row, got, kind in todo:
                j = torch.arange(row + 1, device=DEV)
                j = j[(j > row - window) | (j < n_sink)]
                k, v = K[j], V[j]
                p = torch.softmax(k @ x.double() / D ** 0.5, 0)
                clean = v.nan_to_num(0, 0, 0)
                ref, weighted = p @ clean, p @ clean.abs()
                dots = (k.abs() @ x.double().abs()).max() / D ** 0.5
                ref = torch.where(v.isfinite().all(0), ref, v.masked_fill(v.isfinite(), 0).sum(0))
                _same_where_not_finite(got.double(), ref, _tolerance(kind, ref.nan_to_num(0, 0, 0), weighted, dots, n))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
def test_keys_that_are_not_finite_reach_only_the_tokens_that_see_them(dtype):
    n = 260
    c = CacheCase(dtype, 2, 1, [n], seed=14)
    at, q, clean = _tokens(c, [n], 33, 2)
    step, qs = [torch.zeros((1, 2, D), device=DEV) for _ in range(2)], c.randn(1, 2, D)
    c.ctx.lfps_window_attn_decode(qs, c.kv, 33, 2, step[0])
    k = c.K[0, 0].to(torch.float32)
    k[100, 5] = float("nan")
    raw(c.K)[0, 0] = raw(k.to(c.kd))
    _, _, out = _tokens(c, [n], 33, 2, q=q)
    c.ctx.lfps_window_attn_decode(qs, c.kv, 33, 2, step[1])
    assert torch.equal(out[:100], clean[:100]) and torch.equal(out[133:], clean[133:]) and bool(out[100:133].isnan().all()) and torch.equal(*step)
    c.ctx.close()


def test_rows_that_all_score_minus_infinity():
    """Keys of -inf against positive queries weigh nothing; a token that sees only such rows gets zeros."""
    n = 150
    c = CacheCase("bf16", 1, 1, [n], seed=6)
    c.K[..., 5] = 0
    c.K[0, 0, 10:90, 5] = float("-inf")
    q = c.randn(n, 1, D).to(c.q_dtype)
    q[..., 5] = 1.0
    _, q, out = _tokens(c, [n], 20, 0, q=q)
    assert not bool(out[29:90].any()) and bool(out.isfinite().all()) and bool(out[90:].any(-1).all()) and bool(out[:29].any(-1).all())
    k, v = c.K[0, 0].double(), c.V[0, 0].double()
    for row in (15, 28, 95, 149):
        j = torch.arange(max(0, row - 19), row + 1, device=DEV)
        ref = torch.softmax(k[j] @ q[row, 0].double() / D ** 0.5, 0) @ v[j]
        assert float((out[row, 0].double() - ref).abs().max()) <= 2.0 ** -8 * 2.02 * float(v[j].abs().max())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("Hkv,news,lens", [(1, [5], [4000]), (1, [300], [300]), (8, [3] * 20, [90] * 20)])
def test_a_query_of_nan_is_nan_and_its_own_only(dtype, Hkv, news, lens):
    c = CacheCase(dtype, 4 * Hkv, Hkv, lens, 16, seed=22)
    at = packed(news)
    q = c.randn(at[-1], 4 * Hkv, D).to(c.q_dtype)
    outs = []
    for spoilt in (False, True):
        if spoilt:
            q[2, 3] = float("nan")
        outs.append(torch.zeros_like(q))
        c.ctx.lfps_window_attn(q, ints(at), c.kv, 2000, 4, outs[-1])
    assert bool(outs[1][2, 3].isnan().all())
    outs[0][2, 3] = outs[1][2, 3] = 0
    assert torch.equal(*outs)
    steps, qs = [], c.randn(c.B, 4 * Hkv, D)
    for spoilt in (False, True):
        if spoilt:
            qs[0, 3] = float("nan")
        steps.append(torch.zeros_like(qs))
        c.ctx.lfps_window_attn_decode(qs, c.kv, 2000, 4, steps[-1])
    assert bool(steps[1][0, 3].isnan().all())
    steps[0][0, 3] = steps[1][0, 3] = 0
    assert torch.equal(*steps)
    c.ctx.close()


def test_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64])
    q, out, cu = torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV), torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV), ints([0, 8])
    ok = dict(q=q, cu=cu, kv=c.kv, window=5, n_sink=0, out=out)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(out=out.float())):
        with pytest.raises(TypeError):
            c.ctx.lfps_window_attn(**{**ok, **bad})
    for bad in (dict(q=q[:, :2]), dict(out=out[:4]), dict(cu=ints([0, 4, 8]))):
        with pytest.raises(ValueError):
            c.ctx.lfps_window_attn(**{**ok, **bad})
    no_v = c.ctx.kv_view(c.K, None, c.seq)
    step = dict(q=q[:1].float(), kv=c.kv, window=5, n_sink=0, out=out[:1].float())
    for bad, word in ((dict(window=0), "window"), (dict(window=-7), "window"), (dict(n_sink=-1), "n_sink"), (dict(kv=no_v), "kv->v"), (dict(out="q"), "overlap")):
        for call, good in ((c.ctx.lfps_window_attn, ok), (c.ctx.lfps_window_attn_decode, step)):
            with pytest.raises(LfpsError) as e:
                call(**{**good, **({"out": good["q"]} if bad == {"out": "q"} else bad)})
            assert e.value.code == LFPS_EINVAL and word in str(e.value)
    before = out.clone()
    c.ctx.lfps_window_attn(q[:0], ints([0, 0]), c.kv, 5, 0, out[:0])
    assert torch.equal(out, before)
    c.ctx.close()


def test_arrays_that_make_no_sense():
    """cu that falls, or lies outside the tokens: something is computed, everything stays inside."""
    c = CacheCase("bf16", 4, 2, [64, 64, 64, 64], 16)
    q = torch.zeros((40, 4, D), dtype=torch.bfloat16, device=DEV)
    guard = torch.full((44, 4, D), 7.0, dtype=torch.bfloat16, device=DEV)
    for cu in ([0, 500, -3, 10, 40], [40, 30, 20, 10, 0], [-100, -50, 2000000000, 5, 7]):
        c.ctx.lfps_window_attn(q, ints(cu), c.kv, 9, 2, guard[2:42])
        assert bool((guard[:2] == 7).all()) and bool((guard[42:] == 7).all())
    c.ctx.close()
