"""A NaN among the scores of one part of a row's keys, or a value there that is not finite, beside a key elsewhere that scores so much more
that the part weighs nothing: it shows in the row, as it does where the row's keys are one part."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints
from tests.harness import DEV

pytestmark = pytest.mark.gpu


def _spoil(c, b, g, n, bad):
    """Key 5 of all keys is `bad` in channel 0, where queries have 0: a NaN score.  Key n - 3 scores 16 * 400 / sqrt(128) = 566 (816 powers
    of two) where the queries have 16 in channel 1; the others next to nothing."""
    k = 0.01 * c.randn(n, c.Hkv, D)
    k[:, :, :2] = 0
    k[n - 3, :, 1] = 400.0
    k[5, g, 0] = bad
    c.put(c.K, b, 0, k.to(c.kd))


def _query(c, *shape):
    q = c.randn(*shape, D)
    q[..., 0], q[..., 1] = 0, 16.0
    return q


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("tokens", [1, 4])
def test_prompt_in_parts(dtype, tokens):
    n = 4000
    c = CacheCase(dtype, 4, 2, [n], 16, seed=1)
    _spoil(c, 0, 1, n, float("nan"))
    q = _query(c, tokens, 4).to(c.q_dtype)
    out = torch.zeros_like(q)
    c.ctx.lfps_prompt_attn(q, ints([0, tokens]), c.kv, out)
    assert bool(out[:, 2:].isnan().all()) and bool(out[:, :2].isfinite().all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_prompt_of_few_tokens_in_many_requests(dtype):
    """(The kernel for few tokens, and its joining.)"""
    lens = [4000] + [3] * 40
    c = CacheCase(dtype, 16, 4, lens, 16, seed=2)
    _spoil(c, 0, 3, 4000, float("inf"))                          # 0 times infinity
    q = _query(c, 41, 16).to(c.q_dtype)
    out = torch.zeros_like(q)
    c.ctx.lfps_prompt_attn(q, ints(list(range(42))), c.kv, out)
    assert bool(out[0, 12:].isnan().all()) and bool(out[0, :12].isfinite().all()) and bool(out[1:].isfinite().all())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("prefix", [0, 3, 2000, 4000])
@pytest.mark.parametrize("members", [1, 3, 40])
def test_prefix_like_full_attention(dtype, prefix, members):
    """The NaN in the shared rows, or in the first request's own; all of its members have a key that scores far above it."""
    n = 4000
    c = CacheCase(dtype, 4, 2, [n] * members, 16, seed=3)
    for b in range(members):
        _spoil(c, b, 1, n, float("nan") if b == 0 else 0.0)
    q, out = _query(c, members, 4), torch.zeros((members, 4, D), device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, members]), ints([prefix]), out)
    see = members if prefix > 5 else 1                           # requests that have key 5 of the first
    assert bool(out[:see, 2:].isnan().all()) and bool(out[:, :2].isfinite().all()) and bool(out[see:].isfinite().all())
    if prefix == 0:
        full = torch.zeros_like(out)
        c.ctx.lfps_full_attn_decode(q, c.kv, full)
        assert torch.equal(full.isnan(), out.isnan())
    c.ctx.close()


def _spoil_value(c, b, g):
    v = c.randn(1, c.Hkv, D)
    v[0, g, 9] = float("nan") if c.vd.itemsize == 1 else float("inf")
    c.put(c.V, b, 5, v.to(c.vd))


def _only_channel_9(out, spoilt):
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[spoilt] = torch.arange(D, device=DEV) == 9
    assert torch.equal(~out.isfinite(), bad)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("lens", [[4000], [4000] + [3] * 40, [120]])
def test_prompt_values_that_are_not_finite(dtype, lens):
    """In parts by either kernel, and in one."""
    B, Hkv = len(lens), 4 if len(lens) > 1 else 2
    c = CacheCase(dtype, 4 * Hkv, Hkv, lens, 16, seed=4)
    _spoil(c, 0, 1, lens[0], 0.0)
    _spoil_value(c, 0, 1)
    q = _query(c, B, 4 * Hkv).to(c.q_dtype)
    out = torch.zeros_like(q)
    c.ctx.lfps_prompt_attn(q, ints(list(range(B + 1))), c.kv, out)
    _only_channel_9(out, (0, slice(4, 8)))
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32", "fp8kv"])
@pytest.mark.parametrize("prefix", [0, 3, 2000, 4000])
@pytest.mark.parametrize("members", [1, 3, 40])
def test_prefix_values_that_are_not_finite(dtype, prefix, members):
    n = 4000
    c = CacheCase(dtype, 4, 2, [n] * members, 16, seed=5)
    for b in range(members):
        _spoil(c, b, 1, n, 0.0)
    _spoil_value(c, 0, 1)
    q, out = _query(c, members, 4), torch.zeros((members, 4, D), device=DEV)
    c.ctx.lfps_prefix_attn_decode(q, c.kv, ints([0, members]), ints([prefix]), out)
    _only_channel_9(out, (slice(0, members if prefix > 5 else 1), slice(2, 4)))
    if prefix == 0:
        full = torch.zeros_like(out)
        c.ctx.lfps_full_attn_decode(q, c.kv, full)
        assert torch.equal(full.isfinite(), out.isfinite())
    c.ctx.close()
