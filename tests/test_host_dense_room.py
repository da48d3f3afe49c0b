"""CPU tests of the workspace that serves every smaller call of dense attention."""
import random

import pytest

import paper_2505_16864_amd as J

HEADS = [(1, 1), (2, 2), (5, 1), (6, 3), (12, 12), (32, 8), (40, 8), (40, 40), (64, 1), (96, 96), (4096, 4096)]


def _spread(rng, most):
    return max(1, min(most, round(most ** rng.random())))


@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("d", [64, 128])
def test_room_for_all_smaller_calls(heads, kv_heads, d):
    rng = random.Random(heads * d + kv_heads)
    for rows, sequences in [(1, 1), (64, 16), (278, 4), (8192, 4), (31712, 2), (33000, 8), (20000, 300), (500, 500), (3000, 1), (60000, 65)]:
        if rows * heads > 1 << 24:
            continue
        most = J.jenga_dense_attn_workspace_up_to(rows, rows, sequences, heads, kv_heads, d)
        some = {1, 2, 15, 16, 17, 64, 65, 127, 128, 129, rows // 2, rows - 1, rows} | {_spread(rng, rows) for _ in range(60)}
        for n in (n for n in some if 1 <= n <= rows):
            for s in {1, 2, sequences // 2, sequences, min(64, sequences), min(65, sequences), _spread(rng, sequences), -(-n // 4)}:
                if 1 <= s <= sequences:
                    assert J.jenga_dense_attn_workspace(n, n, s, heads, kv_heads, d) <= most, (rows, sequences, n, s)
        # larger calls, larger room
        assert most <= J.jenga_dense_attn_workspace_up_to(rows + 1, rows, sequences, heads, kv_heads, d)
        assert most <= J.jenga_dense_attn_workspace_up_to(rows, rows, sequences + 1, heads, kv_heads, d)


# Fewer rows, or fewer sequences, that need more than the whole.
def test_fewer_may_need_more():
    assert J.jenga_dense_attn_workspace(33000, 33000, 8, 40, 8, 128) < J.jenga_dense_attn_workspace(1000, 1000, 8, 40, 8, 128)
    assert J.jenga_dense_attn_workspace(64, 64, 16, 8, 8, 128) < J.jenga_dense_attn_workspace(64, 64, 1, 8, 8, 128)


def test_refusals():
    for bad in ((16, 16, 1, 4, 4, 80), (1 << 31, 1, 1, 1, 1, 64), (1 << 24, 1, 1, 4096, 4096, 64), (300000, 1, 60000, 120, 120, 64)):   # the last: smaller calls have too many workgroups
        with pytest.raises(J.JengaError) as e:
            J.jenga_dense_attn_workspace_up_to(*bad)
        assert e.value.status == -2
    with pytest.raises(J.JengaError) as e:
        J.jenga_dense_attn_workspace_up_to(16, 16, 1, 4, 3, 64)
    assert e.value.status == -1


# The limits that the header names: rows with the heads that share keys, and workgroups.
@pytest.mark.parametrize("rows,sequences,heads,kv_heads,taken", [
    ((1 << 30) // 64, 1, 64, 64, False), ((1 << 30) // 64 - 128, 1, 64, 64, True), ((1 << 31) // 8 - 1, 1, 8, 1, False), ((1 << 30) // 8 - 128 * 8, 1, 8, 1, True),
    (1 << 20, 1 << 16, 128, 128, False), (1 << 20, (1 << 16) - (1 << 13), 128, 128, True), (1 << 16, 1 << 16, 40, 40, True), (1 << 16, 1 << 16, 121, 121, False),
    (1 << 16, 1 << 16, 120, 120, True)])
def test_limits(rows, sequences, heads, kv_heads, taken):
    if taken:
        assert J.jenga_dense_attn_workspace(rows, rows, sequences, heads, kv_heads, 64) > 0
        return
    with pytest.raises(J.JengaError) as e:
        J.jenga_dense_attn_workspace(rows, rows, sequences, heads, kv_heads, 64)
    assert e.value.status == -2
