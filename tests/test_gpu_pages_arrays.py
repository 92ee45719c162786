"""Arrays of lfps_pages_update and lfps_pages_compact that overlap: what is written must not be what is read, nor another result."""
import pytest
import torch

from tests.cache_case import CacheCase, ints
from tests.harness import DEV

pytestmark = pytest.mark.gpu


def _refused(call, ok, bad):
    from paper_2506_15704_amd.binding import LFPS_EINVAL, LfpsError
    for change in bad:
        with pytest.raises(LfpsError) as e:
            call(**{**ok, **change})
        assert e.value.code == LFPS_EINVAL and "overlap" in str(e.value), change.keys()


def test_update_refuses_overlapping_arrays():
    B = 4
    c = CacheCase("bf16", 2, 2, [30, 30, 17, 0], 16, cap=64)
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
    new_lens, parent, held, work = ints([31, 31, 17, 5]), ints([0, 1, 2, 3]), z(c.n_blocks), c.ctx.pages_workspace(c.n_blocks)
    per = c.table.shape[1]
    ok = dict(kv=c.kv, parent=parent, new_lens=new_lens, table_out=z(B, per), lens_out=z(B), copies=z(B, 3), work=work, held=held)
    big = z(64 + B * per)
    c.seq = big[2:2 + B].copy_(c.seq)
    shifted = c.view()                                           # the view's lengths are the third to sixth of `big`
    inside = work[:B * 4].view(torch.int32)
    _refused(c.ctx.lfps_pages_update, ok, [
        dict(lens_out=new_lens), dict(lens_out=parent), dict(lens_out=held[:B]), dict(lens_out=ok["table_out"].view(-1)[:B]),
        dict(lens_out=ok["copies"].view(-1)[3 * B - B:]), dict(lens_out=inside), dict(new_lens=inside), dict(parent=inside), dict(copies=c.table.view(-1)[:3 * B].view(B, 3)),
        dict(table_out=big[:B * per].view(B, per), kv=shifted), dict(kv=shifted, lens_out=big[:B]), dict(kv=shifted, lens_out=big[5:5 + B]),
        dict(kv=shifted, copies=big[:3 * B].view(B, 3)), dict(held=work[:c.n_blocks * 4].view(torch.int32))])
    c.ctx.lfps_pages_update(**{**ok, "new_lens": c.seq, "parent": None, "held": None, "kv": shifted})      # lengths that stay: read twice
    c.ctx.lfps_pages_update(**{**ok, "kv": shifted, "lens_out": big[2 + B:2 + 2 * B]})                     # side by side
    assert big[2 + B:2 + 2 * B].tolist() == [31, 31, 17, 5]
    one = CacheCase("bf16", 2, 2, [30], 16, cap=48)                # a table's row and its lengths in one buffer
    row = z(8)
    row[:3], row[3] = one.table[0], 30
    one.table, one.seq = row.view(1, 8)[:, :3], row[3:4]
    one.ctx.lfps_pages_update(one.view(), None, ints([33]), z(1, 8), row[4:5], row[5:].view(1, 3), one.ctx.pages_workspace(one.n_blocks))
    assert row.tolist()[3:] == [30, 33, -1, -1, 0]
    one.ctx.close()
    c.ctx.close()


def test_compact_refuses_overlapping_arrays():
    B = 4
    c = CacheCase("bf16", 2, 2, [30, 30, 17, 0], 16, cap=64)
    n, per = c.n_blocks, c.table.shape[1]
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device=DEV)  # noqa: E731
    held, work = z(n), c.ctx.pages_workspace(n)
    ok = dict(kv=c.kv, table_out=z(B, per), moves=z(n // 2, 3), block_map=z(n), n_live=z(1), work=work, held=held)
    _refused(c.ctx.lfps_pages_compact, ok, [
        dict(block_map=held), dict(n_live=held[3:4]), dict(n_live=c.seq[:1]), dict(n_live=c.table.view(-1)[:1]), dict(n_live=ok["block_map"][n - 1:]),
        dict(n_live=work[:4].view(torch.int32)), dict(held=work[:4 * n].view(torch.int32)), dict(table_out=ok["block_map"][:B * per].view(B, per)),
        dict(n_live=ok["moves"].view(-1)[-1:]), dict(n_live=ok["table_out"].view(-1)[:1])])
    c.ctx.lfps_pages_compact(**ok)
    c.ctx.close()
