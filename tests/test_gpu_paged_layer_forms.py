"""A decoder layer over the paged cache in forms that a serving loop may have."""
import numpy as np
import pytest
import torch

from oracle import kv
from paper_2512_23367_amd import binding as ql, synth
from paper_2512_23367_amd.layer import PagedDecoderLayer, PagedRequests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def U():
    import kv_util
    return kv_util


@pytest.mark.parametrize("kv_bits", [16, 8])
def test_a_layer_without_rotary_embedding(U, kv_bits):
    D, q_heads, heads, d, F, n = 64, 4, 2, 256, 384, 2
    fmt = ql.QlKvFormat(heads=heads, head_dim=D, page_size=32, pages=12, bits=kv_bits)
    ws = [synth.weights((q_heads + 2 * heads) * D, d, 1, "qkv"), synth.weights(d, q_heads * D, 1, "o"), synth.weights(2 * F, d, 1, "gate_up"), synth.weights(d, F, 1, "down")]
    layer = PagedDecoderLayer(*(U.dev(w) for w in ws), 8, 64, fmt, None, n)
    requests, cache = PagedRequests(fmt, n, 4, 64, U.DEV), torch.full((ql.ql_kv_cache_bytes(fmt),), 0xFF, dtype=torch.uint8, device=U.DEV)
    x = U.dev(synth.activations(50, d, 0, "single"))
    requests.step(U.ints([33, 17]))
    y = layer.forward(x, requests, cache)
    assert torch.isfinite(y).all()
    rows = layer.y_qkv[:50].cpu().numpy()
    k, v = (rows[:, (q_heads + i * heads) * D:(q_heads + (i + 1) * heads) * D].reshape(50, heads, D).astype(np.float32) for i in range(2))
    ks, vs = kv.stored(k, v, kv_bits)
    r = object.__new__(U.Requests)
    r.ctx, r.D, r.heads, r.q, r.cu, r.k, r.v = [0, 0], D, q_heads, rows[:, :q_heads * D], np.array([0, 33, 50]), [ks[:33], ks[33:]], [vs[:33], vs[33:]]
    r.check(layer.y_attention[:50])
