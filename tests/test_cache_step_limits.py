"""The largest and the smallest calls of rl_rope_append and rl_prefix_attn: what no launch
can hold is answered UNSUPPORTED on the host, before anything reaches a device, and what
holds nothing does nothing (CPU)."""
import pytest
import torch

from paper_2512_22492_amd import binding as B
from test_cache_step_checks import cache, prefix, rope

UNSUPPORTED = B.RL_DA_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw", [
    dict(batch=1 << 20, max_q_per_seq=100),        # 8 pages each, four work-groups a page
    dict(batch=1 << 12, max_q_per_seq=1 << 16),
    dict(batch=1 << 24, max_q_per_seq=1, q_start=None),
    dict(batch=1 << 22, max_q_per_seq=8),
    dict(batch=1 << 22, max_q_per_seq=8, kv_dtype=1, k_scale=1 << 20, v_scale=1 << 20),
    dict(batch=(1 << 31) - 1, max_q_per_seq=(1 << 31) - 1),
    # three work-groups a token: the first call past 2^24 of them
    dict(batch=5592406, max_q_per_seq=1, q_start=None),
])
def test_appends_of_more_work_groups_than_a_launch_holds(kw):
    assert rope(**kw) == UNSUPPORTED, kw


def test_attention_of_more_rows_than_a_merge_launch_holds():
    def size(batch, hq, hkv, max_pages=4, groups=0):
        return B.rl_prefix_attn_workspace_size(max_pages, batch, groups, hq, hkv)[0]

    assert size((1 << 22) - 1, 32, 8) == B.RL_DA_OK
    assert size(1 << 22, 32, 8) == UNSUPPORTED
    assert size(1 << 27, 1, 1) == UNSUPPORTED
    assert prefix(batch=1 << 22, out=1 << 40) == UNSUPPORTED
    # units for all kv heads, whose number leaves 64 bits if multiplied out
    assert size(1, 1 << 26, 1 << 26, (1 << 27) - 2, (1 << 31) - 1) == UNSUPPORTED
    assert size(1, 1 << 20, 1 << 20, 1 << 26, (1 << 31) - 1) == UNSUPPORTED


def test_one_token_per_sequence_is_a_bound_of_one():
    """Without q_start every sequence brings a token: a bound of none would drop them."""
    assert rope(batch=3, q_start=None, max_q_per_seq=0) == B.RL_DA_ERR_INVALID_ARG
    assert rope(batch=0, q_start=None, max_q_per_seq=0) == B.RL_DA_ERR_INVALID_ARG
    assert rope(batch=3, max_q_per_seq=0) == B.RL_DA_OK


def test_empty_batches_are_no_calls(monkeypatch):
    """Tensors without elements have no address, which the C entry refuses; a step of no
    sequences is not an error."""
    monkeypatch.setattr(B, "_device_index", lambda d: 0)
    monkeypatch.setattr(B, "_on_device", lambda i, fn, *args: fn(*args))
    p = cache(batch=0)
    for groups in (0, 2):
        attend = B.PrefixAttention(p, torch.zeros(groups + 1, dtype=torch.int32),
                                   torch.ones(groups, dtype=torch.int32),
                                   torch.zeros(1 << 16, dtype=torch.uint8))
        attend(p.q, torch.empty_like(p.q))
    append = B.RopeAppender(p, torch.zeros((32, 128)))
    rows = [torch.zeros((5, h, 128), dtype=torch.bfloat16) for h in (4, 2, 2)]
    append(*(r[:0] for r in rows), rows[0][:0])
    # rows behind the last sequence's, here all of them, are left as they are
    append(*rows, torch.ones_like(rows[0]), torch.zeros(1, dtype=torch.int32), 3)
