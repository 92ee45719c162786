"""Full attention of a batch whose groups share their first rows, against 64 bits."""
import pytest
import torch

from tests.cache_case import CacheCase, D, attend64, ints
from tests.harness import DEV

pytestmark = pytest.mark.gpu


def _tolerance(dtype, ref, weighted, dots, n):
    """Query and weights as sums of 16-bit terms, of which at most 2^-18 (bf16) or 2^-22 (fp16) is left (fp32 caches: nothing); products and sums as
    everywhere fp32, 2^-24 of the absolute sum a term; the scores' errors come twice (weights and their sum); the exponential 2^-21."""
    left = {"f16": 2.0 ** -22, "f32": 0.0}.get(dtype, 2.0 ** -18)
    return (2 * (left + 260 * 2.0 ** -24) * dots + 2 * left + 2.0 ** -21 + (n + 80) * 2.0 ** -24) * weighted + 1e-7


def _check(c, starts, prefixes, q=None, scale=1.0):
    """The shared rows are read from the group's first request: the others' hold NaN there."""
    for i, p in enumerate(prefixes):
        b0, b1 = starts[i], starts[i + 1]
        p = max(0, min(p, c.lens[b0]))
        for b in range(b0 + 1, b1):
            m = min(p, c.lens[b])
            nan = torch.full((m, c.Hkv, D), float("nan"), device=DEV)
            c.put(c.K, b, 0, nan.to(c.kd))
            c.put(c.V, b, 0, nan.to(c.vd))
    q = scale * c.randn(c.B, c.Hq, D) if q is None else q
    out = torch.full((c.B, c.Hq, D), 7.0, device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints(starts), ints(prefixes), out)
    inside = set()
    for i, p in enumerate(prefixes):
        b0, b1 = starts[i], starts[i + 1]
        p = max(0, min(p, c.lens[b0]))
        for b in range(b0, b1):
            inside.add(b)
            n = c.lens[b]
            if n == 0:
                assert torch.equal(out[b], torch.zeros_like(out[b]))
                continue
            m = min(p, n)
            k, v = (torch.cat([c.values(x, b0, 0, m), c.values(x, b, m, n)], 1) for x in (c.K, c.V))
            for h in range(c.Hq):
                ref, weighted, dots = attend64(q[b, h:h + 1].double(), k[h // c.G], v[h // c.G])
                err = (out[b, h].double() - ref[0]).abs()
                assert bool((err <= _tolerance(c.dtype, ref, weighted, dots, n)[0]).all()), (b, h, float(err.max()))
    for b in set(range(c.B)) - inside:
        assert bool((out[b] == 7).all())
    return q, out


@pytest.mark.parametrize("layout", [0, 16, "rows", ("rows", 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_prefix_formats_and_layouts(dtype, layout):
    c = CacheCase(dtype, 8, 2, [150, 101, 130, 70, 200, 65], layout, seed=1)
    _check(c, [0, 3, 4, 6], [100, 0, 64])
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "f16"])
@pytest.mark.parametrize("Hq,Hkv,members,prefix", [(1, 1, 1, 5), (4, 1, 8, 63), (4, 1, 9, 64), (2, 1, 33, 65), (1, 1, 70, 129), (4, 4, 40, 1), (4, 1, 33, 300), (8, 2, 16, 1025)])
def test_prefix_members_and_heads(dtype, Hq, Hkv, members, prefix):
    c = CacheCase(dtype, Hq, Hkv, [prefix + i % 5 for i in range(members)], seed=members)
    _check(c, [0, members], [prefix])
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv"])
def test_prefix_long_and_ragged(dtype):
    """Parts of the shared and of the own rows; members shorter than the prefix, empty ones, prefixes beyond the first member's rows."""
    lens = [3000, 2500, 40, 0, 2999] + [700, 1900, 1, 650] + [500]
    c = CacheCase(dtype, 8, 2, lens, 64, seed=3)
    _check(c, [0, 5, 9, 10], [2600, 100000, -4])
    c.ctx.close()


def test_prefix_requests_in_no_group_are_left_alone():
    c = CacheCase("bf16", 4, 2, [60] * 7, 16, seed=4)
    _check(c, [1, 3, 3, 6], [50, 20, 33])
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("scale", [1e-30, 30.0, 1e4])
def test_prefix_queries_of_any_size(dtype, scale):
    """(fp16 terms: any fp32 query fits.)"""
    c = CacheCase(dtype, 4, 2, [300, 280, 270], seed=5, scale=1.0 if scale < 100 else 1e-4)
    _check(c, [0, 3], [256], scale=scale)
    c.ctx.close()


def test_prefix_of_one_request_is_full_attention():
    """The same numbers as the plain call, to its precision and this one's."""
    c = CacheCase("bf16", 8, 2, [777, 123], 16, seed=6)
    q, out = _check(c, [0, 1, 2], [500, 0])
    full = torch.zeros_like(out)
    c.ctx.lfps_full_attn_decode(q, c.kv, full)
    assert float((out - full).abs().max()) <= 2e-5 * float(full.abs().max().clamp_min(1))
    c.ctx.close()


def test_prefix_refusals():
    from paper_2506_15704_amd.binding import LfpsError
    c = CacheCase("bf16", 4, 2, [64, 64])
    q, out = torch.zeros((2, 4, D), device=DEV), torch.zeros((2, 4, D), device=DEV)
    ok = dict(q=q, kv=c.kv, group_start=ints([0, 2]), prefix_len=ints([8]), out=out)
    for bad, err in ((dict(q=q.half()), TypeError), (dict(group_start=ints([0, 1, 2])), ValueError), (dict(out=out[:1]), ValueError),
                     (dict(group_start=ints([0, 1, 2, 2]), prefix_len=ints([1, 1, 1])), LfpsError), (dict(group_start=ints([0]), prefix_len=ints([])), LfpsError),
                     (dict(kv=c.ctx.kv_view(c.K, None, c.seq)), LfpsError)):
        with pytest.raises(err):
            c.ctx.lfps_prefix_attn_decode(**{**ok, **bad})
    for starts in ([0, -5, 900], [2, 0, 1], [5, 9, 9]):      # no sense, but inside
        c.ctx.lfps_prefix_attn_decode(q, c.kv, ints(starts), ints([70, 3]), out)
    torch.cuda.synchronize()
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("members", [3, 12, 40])
def test_prefix_values_that_are_not_finite_stay_out_of_requests_that_end_before_them(dtype, members):
    """Members shorter than the shared prefix: rows behind their own length are the others'."""
    Hq = 2
    lens = [300] + [300 if i % 2 else 120 + i for i in range(1, members)]
    c = CacheCase(dtype, Hq, 1, lens, seed=9)
    v = c.V[0, 0].to(torch.float32)
    v[200, 5] = float("nan")
    v[190, 9] = float("nan") if c.vd.itemsize == 1 else float("inf")
    c.V.view(torch.uint8)[0, 0] = v.to(c.vd).view(torch.uint8) if c.vd.itemsize == 1 else v.to(c.vd).view(torch.uint8)
    q = c.randn(c.B, Hq, D)
    out = torch.zeros((c.B, Hq, D), device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, members]), ints([300]), out)
    K, V = c.values(c.K, 0, 0, 300)[0], v.to(c.vd).to(torch.float32).double()
    for b, n in enumerate(lens):
        for h in range(Hq):
            clean = V[:n].nan_to_num(0, 0, 0)
            ref, weighted, dots = attend64(q[b, h:h + 1].double(), K[:n], clean)
            broken = ~V[:n].isfinite().all(0)
            assert torch.equal(~out[b, h].isfinite(), broken), (b, h)
            err = (out[b, h].double() - ref[0]).abs()[~broken]
            assert bool((err <= _tolerance(dtype, ref, weighted, dots, n)[0][~broken]).all())
    c.ctx.close()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 1)])
def test_prefix_many_requests_of_unlike_lengths_in_groups_of_unlike_sizes(Hq, Hkv):
    """More requests than a workgroup has threads; own rows from none to thousands, so that some requests are one item and one is many."""
    lens = [20 + i * 7 % 50 for i in range(600)]
    lens[300], lens[599] = 3000, 1
    starts = [0, 1, 65, 67, 299, 400, 400, 599]                # (a group without members; the last request is in none)
    c = CacheCase("bf16", Hq, Hkv, lens, 16, seed=9)
    _check(c, starts, [5, 20, 64, 21, 9, 3, 33])
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv"])
def test_prefix_one_request_with_many_rows_of_its_own(dtype):
    c = CacheCase(dtype, 2, 1, [20011], 64, seed=10)
    _check(c, [0, 1], [3])
    c.ctx.close()


@pytest.mark.parametrize("members", [2, 12, 30])
@pytest.mark.parametrize("scale", [1e-30, 30.0, 1e4])
def test_prefix_fp8_queries_of_any_size(members, scale):
    c = CacheCase("fp8kv", 4, 1, [200 + i for i in range(members)], 16, seed=11, scale=1.0 if scale < 100 else 1e-2)
    _check(c, [0, members], [190], scale=scale)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8k", "fp8v"])
def test_prefix_large_groups_hold_a_query_whole(dtype):
    """70 members x 1 head: the 256-row form, with values of unlike size in one query: 2^-18 of each element is too much here (the
    bound has 2^-20 of the absolute sum for the query, which three bf16 terms keep)."""
    c = CacheCase(dtype, 2, 2, [520] * 70, 16, seed=12)
    q = c.randn(c.B, c.Hq, D) * torch.exp2(torch.randint(-6, 3, (c.B, c.Hq, D), device=DEV, generator=c.gen).float())
    out = torch.full((c.B, c.Hq, D), 7.0, device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, c.B]), ints([520]), out)
    for b in range(0, c.B, 7):
        for h in range(c.Hq):
            k, v = c.values(c.K, 0, 0, 520)[h // c.G], c.values(c.V, 0, 0, 520)[h // c.G]
            ref, weighted, dots = attend64(q[b, h:h + 1].double(), k, v)
            # the query's terms 2^-24 of each element at most and fp32 products (260 of 2^-24), twice; two terms of a weight 2^-18; sums over 520 keys
            bound = (2 * 262 * 2.0 ** -24 * dots + 2 * 2.0 ** -18 + 2.0 ** -21 + 600 * 2.0 ** -24) * weighted + 1e-7
            assert bool(((out[b, h].double() - ref[0]).abs() <= bound[0]).all()), (b, h)
    c.ctx.close()


@pytest.mark.parametrize("members", [1, 9, 20])
def test_prefix_every_fp8_value_is_itself(members):
    """One row: its weight is 1, whatever its score, and the output its values (2 rows: all 256 codes, NaN among them)."""
    c = CacheCase("fp8kv", 4, 1, [1] * members, 16, seed=13)
    for codes in (torch.arange(128), torch.arange(128, 256)):
        x = codes.to(torch.uint8).to(DEV).view(torch.float8_e4m3fn)
        c.put(c.V, 0, 0, x.view(1, 1, D))
        out = torch.zeros((members, 4, D), device=DEV)
        c.ctx.lfps_prefix_attn_decode(c.randn(members, 4, D), c.kv, ints([0, members]), ints([1]), out)
        # The one weight is a power of two only up to the rounding of score - maximum + a constant: as two fp16 terms it is 2^-22 off at
        # most, its sum is not; product, join, sum and division round by 2^-24 each, ten times at most.
        want = x.float()
        assert torch.equal(out.isnan(), want.isnan().expand_as(out))
        assert bool((out - want).abs().nan_to_num(0).le((2.0 ** -22 + 10 * 2.0 ** -24) * want.abs().nan_to_num(0)).all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("members,prefix", [(3, 2000), (12, 40), (40, 700)])
def test_prefix_a_query_of_nan_is_nan_and_its_own_only(dtype, members, prefix):
    c = CacheCase(dtype, 4, 1, [prefix + i % 3 for i in range(members)], 16, seed=14)
    q = c.randn(members, 4, D)
    outs = []
    for spoilt in (False, True):
        if spoilt:
            q[1, 2] = float("nan")
        outs.append(torch.zeros((members, 4, D), device=DEV))
        c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, members]), ints([prefix]), outs[-1])
    assert bool(outs[1][1, 2].isnan().all())
    outs[0][1, 2] = outs[1][1, 2] = 0
    assert torch.equal(*outs)
    c.ctx.close()
