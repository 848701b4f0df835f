"""Bounds of the paged cache's calls that hold without a GPU."""
import pytest

from oracle import kv
from paper_2512_23367_amd import binding as ql


def test_tokens_without_a_row_by_hand():
    # 6 rows for 5 + 7 + 1 new tokens: the second request gets one, the third none; 6 + 1 are left
    r = kv.resize(old=[0, 3, 2], want=[5, 10, 3], page=32, ring=[2, 3, 4], pool=[0, 3, 0, 0], table=[[-1, -1], [0, -1], [1, -1]], max_tokens=6)
    assert r["kv_len"] == [5, 4, 2] and r["cu"] == [0, 5, 6, 6] and r["pool"] == [1, 2, 7, 0]
    assert r["slots"] == [64, 65, 66, 67, 68, 3] and r["positions"] == [0, 1, 2, 3, 4, 3]


HEADS = (1, 2, 3, 7, 8, 60, 100, 255, 256, 300, 510, 511, 512, 513, 600, 1000, 2047, 2048, 4000, 4095, 4096, 5000, 65535)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("bits", [16, 8])
def test_the_workspace_is_at_most_137_mb(D, bits):
    """ql_paged_attention_bytes over head counts, those above any tile limit among them, and over calls from one row to the largest."""
    most = 0
    for heads in HEADS:
        fmt = ql.QlKvFormat(heads=heads, head_dim=D, page_size=32, pages=4, bits=bits)
        for group in (1, 4, 32):
            if heads * group >= 1 << 31:
                continue
            for T, requests in ((1, 1), (1, 64), (33, 4), (1000, 4), (60000, 1), (4000, 4000), (1 << 20, 65536)):
                for max_new in (0, 1, 40):
                    most = max(most, ql.ql_paged_attention_bytes(fmt, T, requests, heads * group, max_new))
    assert most <= 137 * 10 ** 6


def test_fewer_tokens_need_no_more_with_many_heads():
    for heads, D, group in ((1, 64, 1), (8, 128, 4), (300, 256, 1), (511, 128, 1), (512, 128, 1), (600, 256, 2), (4095, 64, 1), (4096, 64, 1)):
        fmt = ql.QlKvFormat(heads=heads, head_dim=D, page_size=32, pages=4, bits=8)
        for T, requests in ((1, 1), (5, 2), (300, 3)):
            for max_new in (0, 1, 20):
                of = [ql.ql_paged_attention_bytes(fmt, t, requests, heads * group, max_new) for t in (1, max(1, T // 2), T)]
                assert of == sorted(of)
