"""Appends whose token bounds leave the arrays: the rows are those that lfps_prompt_attn takes the tokens for."""
import pytest
import torch

from tests.cache_case import CacheCase, D, ints, raw, to_cache

pytestmark = pytest.mark.gpu


def clamped(cu, T):
    """[first token, end) of every request, of a rising cu."""
    at = [min(max(x, 0), T) for x in cu]
    return list(zip(at, at[1:]))


@pytest.mark.parametrize("dtype,layout", [("bf16", 0), ("f32", 16), ("fp8kv", 64), ("fp8v", "rows")])
@pytest.mark.parametrize("T,lens,cu", [(16, [20], [0, 20]), (16, [20, 9, 30], [-3, 7, 7, 26]), (5, [3, 6, 40], [0, 4, 9, 2 ** 31 - 1]),
                                       (70, [100, 3, 8], [-2 ** 31, 60, 75, 90]), (3, [8, 8], [3, 5, 9])])
def test_append_takes_bounds_beyond_the_tokens_as_their_number(dtype, layout, T, lens, cu):
    c = CacheCase(dtype, 2, 2, lens, layout, seed=3)
    k, v = (c.randn(T, c.Hkv, D).to(c.q_dtype) for _ in range(2))
    start = [raw(x).clone() for x in (c.K, c.V)]
    c.ctx.lfps_append(k, v, ints(cu), c.kv)
    got = [raw(x).clone() for x in (c.K, c.V)]
    raw(c.K).copy_(start[0])
    raw(c.V).copy_(start[1])
    for b, (t0, t1) in enumerate(clamped(cu, T)):
        t0 = max(t0, t1 - lens[b])                             # tokens at no row
        for x, new in ((c.K, k), (c.V, v)):
            c.put(x, b, lens[b] - (t1 - t0), to_cache(new[t0:t1].float(), x.dtype))
    for x, y in ((c.K, got[0]), (c.V, got[1])):
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
        assert torch.equal(raw(x).contiguous().view(bits), y.contiguous().view(bits))
    c.ctx.close()


def test_what_is_appended_is_what_the_prompt_attends():
    """One token seen by each row's query only with a large score: the output is that token's own value."""
    T, n = 16, 40
    c = CacheCase("f32", 1, 1, [n], 16, seed=4, scale=0.0)
    k = torch.zeros((T, 1, D), device=c.K.device)
    k[torch.arange(T), 0, torch.arange(T)] = 4000.0            # token t's key and query meet in channel t: its score is 1414 above the others'
    v = c.randn(T, 1, D)
    q, out, cu = torch.where(k > 0, 4.0, 0.0), torch.zeros((T, 1, D), device=c.K.device), ints([0, T + 10])
    c.ctx.lfps_append(k, v, cu, c.kv)
    c.ctx.lfps_prompt_attn(q, cu, c.kv, out)
    assert torch.equal(out, v)                                 # (one weight of 1, the others 0: every product and sum is exact)
    c.ctx.close()


def test_append_with_arrays_that_make_no_sense():
    """Bounds that fall: something is written, all of it below the requests' lengths."""
    c = CacheCase("bf16", 2, 2, [30, 30, 30, 30], 16, cap=48, seed=5)
    k = c.randn(40, 2, D).to(torch.bfloat16)
    for cu in ([0, 500, -3, 10, 40], [40, 30, 20, 10, 0], [-100, -50, 2000000000, 5, 7]):
        c.ctx.lfps_append(k, k, ints(cu), c.kv)
    for x in (c.K, c.V):
        used = torch.zeros(x.shape[0], x.shape[2], dtype=torch.bool, device=x.device)
        for b in range(4):
            block, at = c._where(b, 0, 30)
            used[block, at] = True
        assert bool(raw(x).transpose(1, 2)[~used].isnan().all()) and not bool(raw(x).transpose(1, 2)[used].isnan().any())
    c.ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "fp8kv"])
@pytest.mark.parametrize("page", [1, 16])
def test_append_drops_rows_whose_table_entry_is_no_block(dtype, page):
    """(lfps_pages_update leaves -1 for rows that a request did not get.)"""
    c = CacheCase(dtype, 2, 2, [70, 40, 33], page, seed=6)
    k, v = (c.randn(90, 2, D).to(c.q_dtype) for _ in range(2))
    first = [70 - 50, 40 - 20, 33 - 20]
    want = [raw(x).clone() for x in (c.K, c.V)]
    for w, x, new in zip(want, (c.K, c.V), (k, v)):
        for b, t0, t in ((0, 0, 50), (1, 50, 20), (2, 70, 20)):
            for i in range(t):
                j = (first[b] + i) // page
                if not (b == 0 and j >= 48 // page or b == 2 and j == 32 // page):
                    w[c.table[b, j], :, (first[b] + i) % page] = raw(to_cache(new[t0 + i].float(), x.dtype))
    c.table[0, 48 // page:] = -1
    c.table[2, 32 // page] = c.n_blocks
    c.table[0, -1] = 2 ** 31 - 1
    c.ctx.lfps_append(k, v, ints([0, 50, 70, 90]), c.view())
    for x, w in zip((c.K, c.V), want):
        bits = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
        assert torch.equal(raw(x).contiguous().view(bits), w.contiguous().view(bits))
    c.ctx.close()
