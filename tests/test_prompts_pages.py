"""What appends, prompts, prefixes and pages refuse, as far as it shows without a GPU."""
import ctypes

import pytest
import torch

from paper_2506_15704_amd import binding as b


def test_page_workspace_sizes():
    assert b.pages_workspace_bytes(1) >= 4096 and b.pages_workspace_bytes(1 << 24) > 17 * (1 << 24)
    for n, code in ((0, b.LFPS_EINVAL), (-3, b.LFPS_EINVAL), ((1 << 24) + 1, b.LFPS_ECAP)):
        with pytest.raises(b.LfpsError) as ei:
            b.pages_workspace_bytes(n)
        assert ei.value.code == code and "n_blocks" in str(ei.value)


def test_calls_without_a_context():
    kv = ctypes.byref(b.lfps_kv())
    assert b._lib.lfps_append(None, None, None, 0, None, 0, kv, None) == b.LFPS_EINVAL
    assert b._lib.lfps_prompt_attn(None, None, 0, None, 0, kv, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_prefix_attn_decode(None, None, kv, None, None, 1, None, None) == b.LFPS_EINVAL
    assert b._lib.lfps_pages_update(None, kv, None, None, None, None, None, None, None, 0, None) == b.LFPS_EINVAL
    assert b._lib.lfps_pages_compact(None, kv, None, None, None, None, None, None, 0, None) == b.LFPS_EINVAL
    assert b._lib.lfps_pages_copy(None, kv, None, 0, None) == b.LFPS_EINVAL


def test_token_rows_have_to_be_on_the_gpu():
    with pytest.raises(TypeError):
        b._token_rows(torch.zeros(4, 2, 128), torch.float32, 2, "q", torch.device("cuda", 0))


def test_the_rooms_for_partial_results_count_in_the_workspace():
    """65536 rows of 132 floats at least, two for every (request, head) of a large batch."""
    cfg = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, kv_dtype=1, max_seq_len=64, max_k=1, radius=1, n_recent=1, n_sink=0, cand_cap=0, device=0)
    assert b.workspace_bytes(batch=1, **cfg) >= 65536 * 132 * 4
    assert b.workspace_bytes(batch=2047, **cfg) >= 2 * 2047 * 32 * 132 * 4
