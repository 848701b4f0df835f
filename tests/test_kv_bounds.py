"""Bounds of the paged cache's calls that hold without a GPU."""
from oracle import kv


def test_tokens_without_a_row_by_hand():
    # 6 rows for 5 + 7 + 1 new tokens: the second request gets one, the third none; 6 + 1 are left
    r = kv.resize(old=[0, 3, 2], want=[5, 10, 3], page=32, ring=[2, 3, 4], pool=[0, 3, 0, 0], table=[[-1, -1], [0, -1], [1, -1]], max_tokens=6)
    assert r["kv_len"] == [5, 4, 2] and r["cu"] == [0, 5, 6, 6] and r["pool"] == [1, 2, 7, 0]
    assert r["slots"] == [64, 65, 66, 67, 68, 3] and r["positions"] == [0, 1, 2, 3, 4, 3]
