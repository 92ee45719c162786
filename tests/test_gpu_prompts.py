"""New rows into the cache, and the causal attention of the new tokens over it, against plain forms in 64 bits."""
import pytest
import torch

from tests.cache_case import CacheCase, D, attend64, ints, packed, raw, to_cache
from tests.harness import DEV

pytestmark = pytest.mark.gpu

LAYOUTS = [0, 16, "rows", ("rows", 64)]


# ---------------------------------------------------------------- append

def _append_and_check(c, news, T_extra=0, lead=0):
    """Tokens of the requests from `lead` on in the token arrays, T_extra unused ones behind them; every byte of the cache is compared."""
    at = [lead + x for x in packed(news)]
    T = at[-1] + T_extra
    qkv = 3 * c.randn(T, c.Hq + 2 * c.Hkv, D)
    qkv[::3] *= 300                                      # FP8 caches saturate
    qkv = qkv.to(c.q_dtype)
    _, k_new, v_new = qkv.split([c.Hq, c.Hkv, c.Hkv], dim=1)
    want = [raw(c.K).clone(), raw(c.V).clone()]
    c.ctx.lfps_append(k_new, v_new, ints(at), c.kv)
    got = [raw(c.K).clone(), raw(c.V).clone()]
    raw(c.K).copy_(want[0])
    raw(c.V).copy_(want[1])
    for b, t in enumerate(news):
        skip = max(0, t - c.lens[b])
        for x, new in ((c.K, k_new), (c.V, v_new)):
            c.put(x, b, c.lens[b] - t + skip, to_cache(new[at[b] + skip:at[b + 1]].float(), x.dtype))
    for x, y in ((c.K, got[0]), (c.V, got[1])):
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
        assert torch.equal(raw(x).contiguous().view(bits), y.contiguous().view(bits))
    c.ctx.close()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_append_writes_its_rows_and_no_others(dtype, layout):
    _append_and_check(CacheCase(dtype, 8, 4, [40, 7, 0, 65, 33], layout), [40, 2, 0, 17, 1])


@pytest.mark.parametrize("Hkv,news,lens", [(1, [1], [1]), (8, [1] * 70, list(range(1, 71))), (3, [0, 0, 5, 0], [0, 4, 5, 9]), (2, [900, 3], [1000, 3])])
def test_append_heads_and_requests(Hkv, news, lens):
    _append_and_check(CacheCase("bf16", Hkv, Hkv, lens, 16), news)


def test_append_drops_tokens_without_a_row_and_tokens_of_no_request():
    _append_and_check(CacheCase("bf16", 4, 2, [3, 20], 16), [9, 5], T_extra=6, lead=4)


def test_append_keeps_nan_and_rounds_to_even():
    c = CacheCase("fp8kv", 1, 1, [1])
    x = torch.zeros((1, 1, D), dtype=torch.bfloat16, device=DEV)
    # 2^-9 is the smallest E4M3 value; 17 and 19 lie half-way between 16, 18 and 20; 464 and more become 448
    pattern = [float("nan"), float("inf"), -float("inf"), 464.0, -1e30, 448.0, 17.0, 19.0, -17.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, -0.0, 2.0 ** -11]
    x[0, 0, :len(pattern)] = torch.tensor(pattern)
    c.ctx.lfps_append(x, x, ints([0, 1]), c.kv)
    want = [float("nan"), 448, -448, 448, -448, 448, 16, 20, -16, 2.0 ** -9, 0, 2.0 ** -8, -0.0, 0]
    for t in (c.K, c.V):
        got = t[0, 0, 0, :len(want)].float().cpu()
        assert torch.equal(got.nan_to_num(7), torch.tensor(want).nan_to_num(7)) and bool(got[0].isnan())
    c.ctx.close()


# ---------------------------------------------------------------- prompt attention

def _tolerance(dtype, ref, weighted, dots, n):
    """Scores are sums of 128 exact products in fp32 (2^-24 of the absolute sum each), weights and their sum follow them (twice); 16-bit
    weights are off by half a step each, and so is the output; sums over n keys in fp32; the exponential 2^-21."""
    half = {"f16": 2.0 ** -11, "f32": 0.0}.get(dtype, 2.0 ** -8)
    return half * 1.01 * (ref.abs() + weighted) + (2 * 130 * 2.0 ** -24 * dots + 2.0 ** -21 + (n + 8) * 2.0 ** -24) * weighted + 1e-7


def _prompt(c, news, q=None, lead=0, extra=0):
    at = [lead + x for x in packed(news)]
    T = at[-1] + extra
    wide = c.randn(T, c.Hq + 3, D).to(c.q_dtype)          # q as a slice of something wider
    if q is not None:
        wide[:, :c.Hq] = q
    q = wide[:, :c.Hq]
    out = torch.full((T, c.Hq, D), 7.0, dtype=c.q_dtype, device=DEV)
    c.ctx.lfps_prompt_attn(q, ints(at), c.kv, out)
    return at, q, out


def _check_prompt(c, news, at, q, out):
    assert bool((out[:at[0]] == 7).all()) and bool((out[at[-1]:] == 7).all())
    for b, t in enumerate(news):
        n = c.lens[b]
        if t == 0:
            continue
        K, V = (c.values(x, b, 0, n) for x in (c.K, c.V))
        for h in range(c.Hq):
            g = h // c.G
            x = q[at[b]:at[b + 1], h].double()
            got = out[at[b]:at[b + 1], h].double()
            first = max(0, t - n)                          # tokens at no row: zeros
            assert torch.equal(got[:first], torch.zeros_like(got[:first]))
            for i0 in range(first, t, 512):
                i1 = min(t, i0 + 512)
                end = n - t + i1
                s = x[i0:i1] @ K[g, :end].T.contiguous() / D ** 0.5
                seen = torch.arange(end, device=DEV) <= (n - t + torch.arange(i0, i1, device=DEV)).view(-1, 1)
                p = torch.softmax(s.masked_fill(~seen, float("-inf")), 1)
                ref, weighted = p @ V[g, :end], p @ V[g, :end].abs()
                dots = (x[i0:i1].abs() @ K[g, :end].abs().T.contiguous()).amax(1, keepdim=True) / D ** 0.5
                err = (got[i0:i1] - ref).abs()
                assert bool((err <= _tolerance(c.dtype, ref, weighted, dots, n)).all()), (b, h, i0, float(err.max()))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_prompt_formats_and_layouts(dtype, layout):
    news = [70, 1, 0, 33, 129]
    c = CacheCase(dtype, 8, 2, [70, 91, 5, 97, 300], layout, seed=1)
    at, q, out = _prompt(c, news, lead=3, extra=5)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,news,lens", [
    (1, 1, [1], [1]), (4, 1, [8], [8]), (4, 1, [9], [9]), (2, 2, [31, 32, 33], [31, 32, 33]), (2, 1, [63, 64, 65, 16, 17], [63, 64, 65, 1000, 1000]),
    (8, 8, [127, 128, 129], [127, 128, 200]), (12, 3, [257], [700]), (4, 4, [1, 1, 1], [1, 64, 65])])
def test_prompt_edges_of_tiles_and_heads(dtype, Hq, Hkv, news, lens):
    c = CacheCase(dtype, Hq, Hkv, lens, seed=Hq + len(news))
    at, q, out = _prompt(c, news)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("news,lens", [([5], [5003]), ([1, 8, 3], [4000, 129, 2111]), ([40, 2], [3001, 1500]), ([200, 1, 0, 7], [2500, 1, 0, 3000])])
def test_prompt_few_tokens_over_long_caches(dtype, news, lens):
    """The rows are cut into parts, in either kernel, and joined."""
    c = CacheCase(dtype, 4, 1, lens, 16, seed=5)
    at, q, out = _prompt(c, news)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()


def test_prompt_of_thousands_of_tokens():
    news, lens = [2100, 777, 1500], [2100, 900, 4097]
    c = CacheCase("bf16", 4, 1, lens, 64, seed=2)
    at, q, out = _prompt(c, news)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()


def test_prompt_tokens_without_a_row_get_zeros():
    news, lens = [9, 200, 6], [3, 150, 0]
    c = CacheCase("bf16", 4, 2, lens, seed=3)
    at, q, out = _prompt(c, news)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_prompt_scores_far_apart(dtype):
    """Scores of hundreds, one key far above the others, for many maxima that grow along the row."""
    n = 700
    c = CacheCase(dtype, 2, 1, [n], seed=4)
    for i in range(0, n, 50):
        c.K[0, 0, i] *= 1 + i / 25
    at, q, out = _prompt(c, [n], q=(4 * c.randn(n, 2, D)).to(c.q_dtype))
    _check_prompt(c, [n], at, q, out)
    c.ctx.close()


def test_prompt_rows_that_all_score_minus_infinity_and_one_that_is_nan():
    """Keys of -inf against positive queries weigh nothing; a NaN among the keys makes its row's outputs NaN from there on only."""
    n = 150
    c = CacheCase("bf16", 1, 1, [n], seed=6)
    c.K[..., 5] = 0
    c.K[0, 0, 10:90, 5] = float("-inf")
    c.K[0, 0, 140, 7] = float("nan")
    q = c.randn(n, 1, D).to(c.q_dtype)
    q[..., 5] = 1.0
    at, q, out = _prompt(c, [n], q=q)
    k, v = c.K[0, 0].double(), c.V[0, 0].double()
    s = q[:, 0].double() @ k.T.contiguous() / D ** 0.5
    s = torch.where(torch.arange(n, device=DEV) >= torch.arange(1, n + 1, device=DEV).view(-1, 1), float("-inf"), s)
    ref = torch.softmax(s[:140], 1)[:, :140] @ v[:140]
    assert float((out[:140, 0].double() - ref).abs().max()) <= 2.0 ** -8 * 2.02 * float(v[:140].abs().max())
    assert bool(out[140:, 0].isnan().all())
    c.ctx.close()


def test_prompt_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64])
    q, out, cu = torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV), torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV), ints([0, 8])
    k = torch.zeros((8, 2, D), dtype=torch.bfloat16, device=DEV)
    for bad in (dict(q=q.float()), dict(q=q.cpu()), dict(out=out.float())):
        with pytest.raises(TypeError):
            c.ctx.lfps_prompt_attn(**{**dict(q=q, cu=cu, kv=c.kv, out=out), **bad})
    for bad in (dict(q=q[:, :2]), dict(out=out[:4]), dict(cu=ints([0, 4, 8])), dict(q=torch.zeros((8, 4, 2 * D), dtype=torch.bfloat16, device=DEV)[..., ::2])):
        with pytest.raises(ValueError):
            c.ctx.lfps_prompt_attn(**{**dict(q=q, cu=cu, kv=c.kv, out=out), **bad})
    with pytest.raises(ValueError):
        c.ctx.lfps_append(k, k[:4], cu, c.kv)
    odd = torch.zeros(8 * (4 * D + 4) + 4, dtype=torch.bfloat16, device=DEV).as_strided((8, 4, D), (4 * D + 4, D, 1))
    with pytest.raises(LfpsError) as e:                    # rows that are not 16-byte aligned
        c.ctx.lfps_prompt_attn(odd, cu, c.kv, out)
    assert e.value.code == LFPS_EINVAL and "aligned" in str(e.value)
    no_v = c.ctx.kv_view(c.K, None, c.seq)
    with pytest.raises(LfpsError):
        c.ctx.lfps_prompt_attn(q, cu, no_v, out)
    with pytest.raises(LfpsError):
        c.ctx.lfps_append(k, k, cu, no_v)
    before = out.clone()
    c.ctx.lfps_prompt_attn(q[:0], ints([0, 0]), c.kv, out[:0])
    c.ctx.lfps_append(k[:0], k[:0], ints([0, 0]), c.kv)
    assert torch.equal(out, before)
    c.ctx.close()


def test_prompt_with_arrays_that_make_no_sense():
    """cu that falls, or lies outside the tokens: something is computed, everything stays inside."""
    c = CacheCase("bf16", 4, 2, [64, 64, 64, 64], 16)
    q = torch.zeros((40, 4, D), dtype=torch.bfloat16, device=DEV)
    guard = torch.full((44, 4, D), 7.0, dtype=torch.bfloat16, device=DEV)
    for cu in ([0, 500, -3, 10, 40], [40, 30, 20, 10, 0], [-100, -50, 2000000000, 5, 7]):
        c.ctx.lfps_prompt_attn(q, ints(cu), c.kv, guard[2:42])
        assert bool((guard[:2] == 7).all()) and bool((guard[42:] == 7).all())
    c.ctx.close()


def _same_where_not_finite(got, ref, tol):
    assert torch.equal(got.isnan(), ref.isnan()) and torch.equal(got.isinf(), ref.isinf())
    assert torch.equal(got[ref.isinf()].sign(), ref[ref.isinf()].sign())
    fine = ref.isfinite()
    assert bool(((got - ref).abs()[fine] <= tol.expand_as(ref)[fine]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8v", "fp8kv"])
@pytest.mark.parametrize("Hq,news,lens", [(1, [200], [200]), (4, [300], [333]), (4, [5], [70]), (2, [1, 70], [64, 129])])
def test_prompt_values_that_are_not_finite_reach_only_the_tokens_that_see_them(dtype, Hq, news, lens):
    """Infinities and NaN in single channels of single rows, a row apart from tokens that do not see them."""
    c = CacheCase(dtype, Hq, 1, lens, seed=8)
    bad = float("nan") if c.vd.itemsize == 1 else float("inf")
    marks = []
    for b, n in enumerate(lens):
        for row, ch, x in ((n - 1, 3, bad), (n - 2, 77, float("nan")), (n // 2, 64, bad), (n // 2 + 1, 127, -bad)):
            v = c.V[b, 0].to(torch.float32)
            v[row, ch] = x
            raw(c.V)[b, 0] = raw(to_cache(v, c.vd) if x == x or c.vd.itemsize > 1 else v.to(c.vd))
            marks.append((b, row, ch))
    at, q, out = _prompt(c, news)
    for b, t in enumerate(news):
        n = lens[b]
        K, V = c.values(c.K, b, 0, n)[0], c.V[b, 0].to(torch.float32).double()
        for h in range(Hq):
            for i in range(max(0, t - 40), t):
                end = n - t + i + 1
                s = K[:end] @ q[at[b] + i, h].double() / D ** 0.5
                p = torch.softmax(s, 0)
                clean = V[:end].nan_to_num(0, 0, 0)
                ref, weighted = p @ clean, p @ clean.abs()
                dots = (K[:end].abs() @ q[at[b] + i, h].double().abs()).max() / D ** 0.5
                ref = torch.where(V[:end].isfinite().all(0), ref, V[:end].masked_fill(V[:end].isfinite(), 0).sum(0))
                _same_where_not_finite(out[at[b] + i, h].double(), ref, _tolerance(dtype, ref.nan_to_num(0, 0, 0), weighted, dots, n))
    c.ctx.close()


@pytest.mark.parametrize("tokens", [1, 300])
def test_prompt_every_fp8_value_is_itself(tokens):
    """Rows that all are the same: the output is that row's values, which bf16 holds (a few tokens; many, which take the other kernel)."""
    c = CacheCase("fp8kv", 2, 1, [tokens], 16, seed=21)
    for codes in (torch.arange(127), torch.arange(128, 255)):
        x = torch.cat([codes, codes[-1:]]).to(torch.uint8).to(DEV).view(torch.float8_e4m3fn)
        c.put(c.V, 0, 0, raw(x.view(1, 1, D)).expand(tokens, 1, D).contiguous().view(torch.float8_e4m3fn))
        out = torch.zeros((tokens, 2, D), dtype=torch.bfloat16, device=DEV)
        c.ctx.lfps_prompt_attn(c.randn(tokens, 2, D).to(torch.bfloat16), ints([0, tokens]), c.kv, out)
        # sums of equal values, divided by the weights' own sum: fp32 rounding, then bf16's; the values have 4 bits
        assert bool((out.float() - x.float()).abs().le(2.0 ** -8 * x.float().abs()).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("Hkv,news,lens", [(1, [5], [4000]), (1, [300], [300]), (8, [3] * 20, [90] * 20)])
def test_prompt_a_query_of_nan_is_nan_and_its_own_only(dtype, Hkv, news, lens):
    """In parts, in one, and many requests of few tokens."""
    c = CacheCase(dtype, 4 * Hkv, Hkv, lens, 16, seed=22)
    at = packed(news)
    q = c.randn(at[-1], 4 * Hkv, D).to(c.q_dtype)
    outs = []
    for spoilt in (False, True):
        if spoilt:
            q[2, 3] = float("nan")
        outs.append(torch.zeros_like(q))
        c.ctx.lfps_prompt_attn(q, ints(at), c.kv, outs[-1])
    assert bool(outs[1][2, 3].isnan().all())
    outs[0][2, 3] = outs[1][2, 3] = 0
    assert torch.equal(*outs)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv", "f32"])
def test_prompt_single_tokens_over_many_rows_beside_a_prompt(dtype):
    """Both kernels in one call, the few tokens in parts."""
    news = [900, 1, 7, 2]
    c = CacheCase(dtype, 4, 1, [900, 5000, 4001, 17], 16, seed=23)
    at, q, out = _prompt(c, news)
    _check_prompt(c, news, at, q, out)
    c.ctx.close()
