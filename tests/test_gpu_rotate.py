"""Norms and turns of the newest tokens' heads on their way into the cache, against the formulas in 64 bits."""
import math

import pytest
import torch

from tests.cache_case import CacheCase, D, ints, packed, raw
from tests.harness import DEV, stored_values

pytestmark = pytest.mark.gpu

LAYOUTS = [0, 16, "rows", ("rows", 64)]
HALF = {torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float16: (2.0 ** -11, 2.0 ** -25), torch.float32: (2.0 ** -24, 2.0 ** -150),
        torch.float8_e4m3fn: (2.0 ** -4, 2.0 ** -10)}     # half a step: of the value, and among the numbers below the normal ones


def _freq(half, base=1e4):
    return torch.tensor([base ** (-i / max(half, 1)) for i in range(half)], device=DEV)


def _turned(x, weight, eps, pos, axis, freq, interleaved):
    """x [T, H, D] -> the result in 64 bits, and the size of what it was made from."""
    x = x.double()
    half = freq.shape[0]
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    y, size = x.clone(), x.abs().clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = (pos[axis[i]].double() * freq[i].double()).view(-1, 1)
        y[..., a] = x[..., a] * angle.cos() - x[..., b] * angle.sin()
        y[..., b] = x[..., b] * angle.cos() + x[..., a] * angle.sin()
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def _close(got, ref, size, dtype):
    """A norm: 128 squares and their sum, a root, a quotient, two products: (128 / 2 + 6) 2^-24.  Sine and cosine: the reduced angle, at most pi / 4,
    is off by 2^-25, the sums' last roundings and what they leave out by 2^-23; two products and a sum 2 * 2^-24: together less than 80 * 2^-24 of the
    sizes.  Positions of 2^24 and angles of a position each: 64 bits leave 2^-27.  Then half a step of the type."""
    step, least = HALF[dtype]
    if dtype == torch.float8_e4m3fn:
        ref = ref.clamp(-448, 448)
    before = 80 * 2.0 ** -24 * size
    assert bool(((got - ref).abs() <= before + step * (ref.abs() + before) + least).all()), float(((got - ref).abs() - before - step * ref.abs()).max())


def _run(c, news, rot, interleaved=False, norm=True, q_f32=False, axes=1, positions="given", lead=0, extra=0, q_scale=1.0):
    at = [lead + x for x in packed(news)]
    T, half = at[-1] + extra, rot // 2
    qkv = (c.randn(T, c.Hq + 2 * c.Hkv + 1, D) * q_scale * (0.01 + 8 * torch.rand((T, c.Hq + 2 * c.Hkv + 1, 1), device=DEV, generator=c.gen))).to(c.q_dtype)
    q, k, v = qkv[:, :c.Hq], qkv[:, c.Hq:c.Hq + c.Hkv], qkv[:, c.Hq + c.Hkv:c.Hq + 2 * c.Hkv]
    wq, wk = (1 + 0.3 * c.randn(D) if norm else None for _ in range(2))
    freq, eps = _freq(half), 1e-5
    row = torch.zeros(T, dtype=torch.long, device=DEV)
    for b, t in enumerate(news):
        row[at[b]:at[b + 1]] = torch.arange(c.lens[b] - t, c.lens[b], device=DEV)
    if positions is None:
        pos, given = row.view(1, -1), None
    else:
        pos = torch.randint(-50, 2 ** 24, (axes, T), device=DEV, generator=c.gen)
        given = pos.to(torch.int32)
    axis = torch.randint(0, axes, (max(half, 1),), device=DEV, generator=c.gen)
    r = c.ctx.rotary(inv_freq=freq if half else None, q_weight=wq, k_weight=wk, eps=eps, pair_axis=axis[:half].to(torch.int32) if axes > 1 else None,
                     n_axes=axes, interleaved=interleaved)
    out_dtype = torch.float32 if q_f32 else c.q_dtype
    out = torch.full((T, c.Hq, D), 7.0, dtype=out_dtype, device=DEV)
    before = [raw(c.K).clone(), raw(c.V).clone()]
    c.ctx.lfps_rotate_append(r, q, k, v, given, ints(at), c.kv, out)
    axis = axis.tolist()
    refq, sizeq = _turned(q, wq, eps, pos, axis, freq, interleaved)
    refk, sizek = _turned(k, wk, eps, pos, axis, freq, interleaved)
    assert bool((out[:at[0]] == 7).all()) and bool((out[at[-1]:] == 7).all())
    _close(torch.where((row >= 0).view(-1, 1, 1), out.double(), refq)[at[0]:at[-1]], refq[at[0]:at[-1]], sizeq[at[0]:at[-1]], out_dtype)
    assert bool((out[at[0]:at[-1]][row[at[0]:at[-1]] < 0] == 0).all())
    # the cache: new rows, and not a byte elsewhere
    for b, t in enumerate(news):
        n = c.lens[b]
        skip = max(0, t - n)
        lo, hi = at[b] + skip, at[b + 1]
        if lo < hi:
            _close(stored_values(c.get(c.K, b, n - t + skip, n)).double(), refk[lo:hi], sizek[lo:hi], c.kd)
            want = v[lo:hi].float()
            want = (want.clamp(-448, 448) if c.vd.itemsize == 1 else want).to(c.vd)
            assert torch.equal(raw(c.get(c.V, b, n - t + skip, n)), raw(want))
            for x, old in ((c.K, before[0]), (c.V, before[1])):
                c.put(x, b, n - t + skip, c.get(old.view(x.dtype) if old.dtype == torch.uint8 else old, b, n - t + skip, n))
    bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}
    for x, old in ((c.K, before[0]), (c.V, before[1])):
        assert torch.equal(raw(x).contiguous().view(bits[x.element_size()]), old.contiguous().view(bits[x.element_size()]))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8k", "fp8v", "fp8kv"])
def test_formats_and_layouts(dtype, layout):
    c = CacheCase(dtype, 8, 4, [40, 7, 0, 65, 33], layout, seed=1)
    _run(c, [40, 2, 0, 17, 1], 128, lead=2, extra=3)
    c.ctx.close()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", list(range(0, 129, 16)))
def test_channels_that_are_turned(rot, interleaved):
    for norm in (False, True):
        c = CacheCase("f32", 2, 1, [33], seed=rot)
        _run(c, [20], rot, interleaved, norm)
        c.ctx.close()


@pytest.mark.parametrize("Hq,Hkv,news,lens", [(1, 1, [1], [1]), (4, 1, [1] * 70, list(range(1, 71))), (3, 3, [0, 0, 5, 0], [0, 4, 5, 9]),
                                              (32, 8, [900, 3], [1000, 3]), (64, 16, [17], [17]), (40, 20, [2, 2], [2, 9])])
@pytest.mark.parametrize("q_f32", [False, True])
def test_heads_and_requests(Hq, Hkv, news, lens, q_f32):
    c = CacheCase("bf16", Hq, Hkv, lens, 16, seed=3)
    _run(c, news, 128, q_f32=q_f32)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("Hq,Hkv,news,lens", [(32, 8, [1400, 2], [1405, 2]), (4, 2, [8192], [8192]), (9, 9, [2100], [2100])])
def test_thousands_of_tokens(dtype, Hq, Hkv, news, lens):
    c = CacheCase(dtype, Hq, Hkv, lens, 16, seed=Hq)
    _run(c, news, 96, interleaved=Hq == 4, lead=1, extra=2)
    c.ctx.close()


@pytest.mark.parametrize("axes,interleaved", [(2, False), (3, False), (3, True), (8, False)])
def test_positions_of_several_axes(axes, interleaved):
    c = CacheCase("bf16", 4, 2, [100, 9], 16, seed=axes)
    _run(c, [77, 9], 96, interleaved, axes=axes)
    c.ctx.close()


def test_positions_are_the_rows_if_none_are_given():
    c = CacheCase("f16", 4, 2, [100, 9], 16, seed=4)
    _run(c, [77, 9], 128, positions=None)
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "fp8kv"])
def test_tokens_without_a_row_and_large_and_small_heads(dtype):
    c = CacheCase(dtype, 4, 2, [3, 20, 0], 16, seed=5)
    _run(c, [9, 5, 4], 128, lead=4, extra=6)
    _run(c, [9, 5, 4], 64, norm=False, q_scale=300.0)             # FP8 saturates
    _run(c, [9, 5, 4], 128, q_scale=1e-6)                         # eps counts
    c.ctx.close()


def test_a_position_far_out_is_turned_as_exactly_as_a_near_one():
    """Up to 2^31: 64 bits hold the product of position and frequency to 2^-53 * 2^31 = 2^-22 of a turn's radian."""
    c = CacheCase("f32", 1, 1, [64], seed=6)
    pos = torch.randint(2 ** 30, 2 ** 31 - 1, (1, 64), device=DEV, generator=c.gen)
    x, v = c.randn(64, 1, D), c.randn(64, 1, D)
    out, freq = torch.zeros_like(x), _freq(64)
    c.ctx.lfps_rotate_append(c.ctx.rotary(inv_freq=freq), x, v, v, pos.to(torch.int32), ints([0, 64]), c.kv, out)
    ref, size = _turned(x, None, 0, pos, [0] * 64, freq, False)
    assert bool(((out.double() - ref).abs() <= (2.0 ** -21 + 80 * 2.0 ** -24) * size).all())
    c.ctx.close()


@pytest.mark.parametrize("interleaved", [False, True])
def test_sines_of_far_positions_near_whole_half_turns(interleaved):
    """Pairs (0, 1) become (-sin, cos) with no rounding of their own.  Position and frequency have 55 bits together, so the angle is taken here as a sum
    of two that 64 bits hold.  The reduced angle is rounded once (2^-24 of it), its sine's and cosine's sums twice more: less than 4 * 2^-24 of either,
    which is next to nothing where the sine is small.  The reduction in two terms leaves 2^-45."""
    c = CacheCase("f32", 1, 1, [128], seed=8)
    far = 2 ** 31 - torch.randint(1, 2 ** 29, (128,), device=DEV, generator=c.gen)
    pos = torch.where(torch.arange(128, device=DEV) % 2 == 0, far, -far)
    freq = 0.5 + 0.5 * torch.rand(64, device=DEV, generator=c.gen)
    x, out = torch.zeros((128, 1, D), device=DEV), torch.zeros((128, 1, D), device=DEV)
    first, second = (slice(0, None, 2), slice(1, None, 2)) if interleaved else (slice(0, 64), slice(64, None))
    x[..., second] = 1
    c.ctx.lfps_rotate_append(c.ctx.rotary(inv_freq=freq, interleaved=interleaved), x, x, x, pos.to(torch.int32), ints([0, 128]), c.kv, out)
    got_sin, got_cos = -out[:, 0, first].double().cpu(), out[:, 0, second].double().cpu()
    small = 0
    for t, p in enumerate(pos.tolist()):
        high, low = p >> 16 << 16, p & 0xFFFF
        for i, f in enumerate(freq.double().tolist()):
            a, b = high * f, low * f                                # (31 - 16 and 16 bits times 24: exact)
            sin = math.sin(a) * math.cos(b) + math.cos(a) * math.sin(b)
            cos = math.cos(a) * math.cos(b) - math.sin(a) * math.sin(b)
            small += min(abs(sin), abs(cos)) < 2.0 ** -5
            assert abs(float(got_sin[t, i]) - sin) <= 4 * 2.0 ** -24 * abs(sin) + 2.0 ** -45, (p, f)
            assert abs(float(got_cos[t, i]) - cos) <= 4 * 2.0 ** -24 * abs(cos) + 2.0 ** -45, (p, f)
    assert small > 100
    c.ctx.close()


def test_values_that_are_not_finite_stay_in_their_head():
    """Without a norm in their pair, with one in their head; channels that are not turned keep their infinities."""
    c = CacheCase("bf16", 2, 1, [8], seed=7)
    x, k = c.randn(8, 3, D).to(torch.bfloat16).split([2, 1], 1)
    clean, out = (torch.zeros((8, 2, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for weight in (None, torch.ones(D, device=DEV)):
        for rot, bad, touched in ((64, 5, [5, 37]), (64, 100, [100]), (0, 5, [5])):
            r = c.ctx.rotary(inv_freq=_freq(rot // 2) if rot else None, q_weight=weight)
            c.ctx.lfps_rotate_append(r, x, k, k, None, ints([0, 8]), c.kv, clean)
            was = x[3, 1, bad].clone()
            x[3, 1, bad] = float("inf")
            c.ctx.lfps_rotate_append(r, x, k, k, None, ints([0, 8]), c.kv, out)
            x[3, 1, bad] = was
            same = out == clean
            assert bool(same[:, 0].all()) and bool(same[:3, 1].all()) and bool(same[4:, 1].all())
            if weight is None:
                rest = [i for i in range(D) if i not in touched]
                assert bool(same[3, 1, rest].all()) and not bool(out[3, 1, touched].isfinite().any())
                assert rot and bad < rot or bool(out[3, 1, bad] == float("inf"))
            else:
                assert bool(out[3, 1, bad].isnan())
    c.ctx.close()


def test_rows_whose_table_entry_is_no_block_are_dropped():
    c = CacheCase("bf16", 2, 1, [40], 16, seed=8)
    c.table[0, 1], c.table[0, 2] = -1, c.n_blocks
    x, k = c.randn(40, 3, D).to(torch.bfloat16).split([2, 1], 1)
    before, out = c.K.clone(), torch.zeros((40, 2, D), dtype=torch.bfloat16, device=DEV)
    c.ctx.lfps_rotate_append(c.ctx.rotary(inv_freq=_freq(64)), x, k, k, None, ints([0, 40]), c.kv, out)
    mine = int(c.table[0, 0])
    others = [i for i in range(c.n_blocks) if i != mine]
    assert torch.equal(c.K[others].view(torch.int16), before[others].view(torch.int16)) and torch.equal(c.V[mine, 0], k[:16, 0])
    c.ctx.close()


def test_arrays_that_make_no_sense():
    c = CacheCase("bf16", 4, 2, [64, 64, 64, 64], 16)
    x = torch.ones((40, 4, D), dtype=torch.bfloat16, device=DEV)
    r = c.ctx.rotary(inv_freq=_freq(64), pair_axis=torch.randint(-2 ** 31, 2 ** 31 - 1, (64,), device=DEV).to(torch.int32), n_axes=2)
    pos = torch.zeros((2, 40), dtype=torch.int32, device=DEV)
    guard = torch.full((44, 4, D), 7.0, dtype=torch.bfloat16, device=DEV)
    for cu in ([0, 500, -3, 10, 40], [40, 30, 20, 10, 0], [-100, -50, 2000000000, 5, 7]):
        c.ctx.lfps_rotate_append(r, x[:, :4], x[:, :2], x[:, 2:], pos, ints(cu), c.kv, guard[2:42])
        assert bool((guard[:2] == 7).all()) and bool((guard[42:] == 7).all())
    c.ctx.close()


def test_refusals():
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    c = CacheCase("bf16", 4, 2, [64])
    qkv = torch.zeros((8, 8, D), dtype=torch.bfloat16, device=DEV)
    q, k, v = qkv.split([4, 2, 2], 1)
    ok = dict(rot=c.ctx.rotary(inv_freq=_freq(64)), q=q, k_new=k, v_new=v, positions=None, cu=ints([0, 8]), kv=c.kv,
              q_out=torch.zeros((8, 4, D), dtype=torch.bfloat16, device=DEV))
    call = lambda **bad: c.ctx.lfps_rotate_append(**{**ok, **bad})  # noqa: E731
    call()
    for bad in (dict(q=q.float()), dict(v_new=v.cpu()), dict(q_out=ok["q_out"].half()), dict(positions=torch.zeros((1, 8), device=DEV))):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in (dict(k_new=k[:4]), dict(k_new=k.contiguous()), dict(q_out=ok["q_out"][:4]), dict(positions=ints([0] * 7)), dict(cu=ints([0, 8, 8]))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        c.ctx.rotary(inv_freq=_freq(64), pair_axis=ints([0] * 63))
    w = torch.ones(D + 1, device=DEV)
    for rot, word in ((dict(inv_freq=_freq(60)), "rotary_dim"), (dict(inv_freq=_freq(72)), "rotary_dim"), (dict(n_axes=0), "n_axes"), (dict(n_axes=9), "n_axes"),
                      (dict(inv_freq=_freq(64), n_axes=2, pair_axis=ints([0] * 64)), "axes"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                      (dict(eps=float("inf")), "eps"), (dict(q_weight=w[1:]), "aligned")):
        with pytest.raises(LfpsError) as e:
            call(rot=c.ctx.rotary(**rot))
        assert e.value.code == LFPS_EINVAL and word in str(e.value), rot
    for out in (qkv.view(-1)[:8 * 4 * D].view(8, 4, D), qkv.view(-1)[4 * D + 8 * 4 * D - 8 * D:][:8 * 4 * D - 8 * D].view(-1, 4, D)):
        n = out.shape[0]
        with pytest.raises(LfpsError) as e:
            c.ctx.lfps_rotate_append(ok["rot"], q[:n], k[:n], v[:n], None, ints([0, n]), c.kv, out)
        assert "overlap" in str(e.value)
    with pytest.raises(LfpsError):
        call(kv=c.ctx.kv_view(c.K, None, c.seq))
    before = c.K.clone()
    c.ctx.lfps_rotate_append(ok["rot"], q[:0], k[:0], v[:0], None, ints([0, 0]), c.kv, ok["q_out"][:0])
    assert torch.equal(c.K.view(torch.int16), before.view(torch.int16))
    c.ctx.close()
