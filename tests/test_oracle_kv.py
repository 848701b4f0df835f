"""Pins of the oracle of the paged cache: hand-derived examples, none computed by the library."""
import numpy as np
import pytest

from oracle import kv


def test_resize_by_hand():
    # pages of 32; 6 of them, 3 free: 4, 0, 2 (from place 5 on); request 0 ends, 1 grows over a page border, 2 starts, 3 finds no page left
    r = kv.resize(old=[40, 31, 0, 32], want=[0, 34, 33, 35], page=32, ring=[0, 2, 9, 9, 9, 4], pool=[5, 3, 0, 0],
                  table=[[1, 3, -1], [5, -1, -1], [-1, -1, -1], [7, -1, -1]], max_tokens=100)
    assert r["table"] == [[1, 3, -1], [5, 4, -1], [0, 2, -1], [7, -1, -1]]
    assert r["kv_len"] == [0, 34, 33, 32] and r["cu"] == [0, 0, 3, 36, 39]
    assert r["slots"][:3] == [5 * 32 + 31, 4 * 32, 4 * 32 + 1] and r["slots"][3:36] == list(range(32)) + [64] and r["slots"][36:] == [-1] * 3
    assert r["positions"][:3] == [31, 32, 33] and r["positions"][36:] == [32, 33, 34]
    assert r["pool"] == [2, 2, 3, 0] and r["ring"] == [0, 2, 1, 3, 9, 4]


def test_layout_is_a_bijection_and_matches_the_documented_strides():
    for D in (64, 128, 256):
        for bits in (8, 16):
            e = bits // 8
            t, c = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
            ko, vo = kv.key_offset(t, c, D, bits), kv.value_offset(t, c, D, bits)
            both = np.concatenate([ko.ravel(), vo.ravel()])
            assert sorted(both) == list(range(0, 64 * D * e, e))
    # written out from the description: K [D/16][2][32][8], V [D/32][2][2][32][8] with token 16 s + 8 (j / 4) + 4 h + j % 4
    k = np.arange(128 // 16 * 2 * 32 * 8).reshape(8, 2, 32, 8) * 2
    v = np.arange(4 * 2 * 2 * 32 * 8).reshape(4, 2, 2, 32, 8) * 2 + 64 * 128
    assert kv.key_offset(5, 16 * 3 + 8 + 2, 128, 16) == k[3, 1, 5, 2]
    assert kv.value_offset(16 * 1 + 8 * 1 + 4 * 0 + 3, 32 * 2 + 7, 128, 16) == v[2, 1, 0, 7, 4 * 1 + 3]
    k8 = np.arange(4 * 2 * 32 * 16).reshape(4, 2, 32, 16)
    v8 = np.arange(4 * 2 * 32 * 16).reshape(4, 2, 32, 16) + 32 * 128
    assert kv.key_offset(9, 32 * 1 + 16 + 4, 128, 8) == k8[1, 1, 9, 4]
    assert kv.value_offset(16 * 1 + 8 * 0 + 4 * 1 + 2, 32 * 3 + 30, 128, 8) == v8[3, 1, 30, 8 * 1 + 4 * 0 + 2]


def test_rotation_keeps_lengths_and_turns_by_the_angle():
    x = np.zeros((1, 1, 64), np.float16)
    x[0, 0, 3], x[0, 0, 40] = 2, 5
    cs = np.zeros((4, 32), np.float32)
    cs[2, 3], cs[2, 16 + 3] = 0.6, 0.8
    y = kv.rotate(x, cs, np.array([2]), 32)
    assert y[0, 0, 3] == np.float32(0.6) * 2 and y[0, 0, 19] == np.float32(0.8) * 2 and y[0, 0, 40] == 5


def test_attention_by_hand():
    # two tokens, scores 0 and ln 3: weights 1/4 and 3/4
    q = np.zeros((1, 1, 64), np.float16)
    q[0, 0, 0] = 1
    k, v = np.zeros((3, 1, 64)), np.zeros((3, 1, 64))
    k[1, 0, 0], k[2] = np.log(3.0), np.nan
    v[0, 0, 5], v[1, 0, 5], v[2] = 4, 8, np.inf
    y = kv.attention(q, k, v, [1], 1.0, True, 0)[0]
    assert y[0, 0, 5] == pytest.approx(7, rel=1e-14) and np.count_nonzero(y) == 1
    assert kv.attention(q, k, v, [1], 1.0, True, 1)[0][0, 0, 5] == 8           # window of one: itself
    assert not kv.attention(q, k, v, [-1], 1.0, True, 0)[0].any()              # sees nothing
    assert not kv.attention(q, k[:0], v[:0], [0], 1.0, False, 0)[0].any()


def test_quantizer_by_hand():
    x = np.array([[0, 0, 0, 0], [127, -63.5, 0.5, 1.5], [1e-35, 0, 0, 0]], np.float32)
    codes, scale = kv.quantize(x)
    assert codes.tolist() == [[0] * 4, [127, -64, 0, 2], [0] * 4] and scale.tolist() == [2.0 ** -31, 1, 2.0 ** -31]
    k, v = kv.stored(np.full((1, 1, 64), np.inf, np.float32), np.ones((1, 1, 64), np.float32), 16)
    assert np.isnan(k).all() and not v.any()
