"""Attention over the paged cache where its kernels' loops, searches and number formats end: contexts beyond what a wavefront looks up of
the block table at once, batches without parts, every token seen by every token in every kernel.  Long contexts are few pages that
occur many times in a block table."""
import numpy as np
import pytest
import torch

from paper_2512_23367_amd import binding as ql

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def U():
    import kv_util
    return kv_util


def aliased(U, seed, ctx, new, heads, kv_heads, D, bits, page, pool=9, missing=()):
    """Requests whose pages are drawn from a pool of `pool`, each as often as it comes.  `missing`: (request, column) without a page,
    all below the request's new tokens; for the oracle those tokens are not there."""
    r = U.Requests(seed, [pool * page - 1], [1], heads, kv_heads, D, bits, page)
    rng = np.random.default_rng(seed + 1000)
    k, v = r.k[0].reshape(pool, page, kv_heads, D), r.v[0].reshape(pool, page, kv_heads, D)
    r.ctx, r.new, r.len = list(ctx), list(new), [c + n for c, n in zip(ctx, new)]
    which = rng.integers(0, pool, (len(ctx), -(-max(r.len) // page) + 1))
    r.table = r.table[0][which]
    r.k = [k[which[b, :-(-n // page)]].reshape(-1, kv_heads, D)[:n] for b, n in enumerate(r.len)]
    r.v = [v[which[b, :-(-n // page)]].reshape(-1, kv_heads, D)[:n] for b, n in enumerate(r.len)]
    r.T, r.cu = sum(new), np.concatenate([[0], np.cumsum(new)])
    r.q = rng.standard_normal((r.T, heads * D)).astype(np.float16)
    for i, (b, column) in enumerate(missing):
        r.table[b, column] = (-1, r.fmt.pages)[i % 2]
    r.gone = {b: np.concatenate([c * page + np.arange(page) for bb, c in missing if bb == b]) for b in {b for b, _ in missing}}
    return r


def without_the_missing(r):
    """The oracle's view: tokens on missing pages taken out, positions moved up."""
    r.ctx = list(r.ctx)
    for b, gone in r.gone.items():
        left = np.setdiff1d(np.arange(r.len[b]), gone)
        assert gone.max() < r.ctx[b]
        r.k[b], r.v[b], r.ctx[b] = r.k[b][left], r.v[b][left], r.ctx[b] - len(gone)
    return r


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,heads", [(64, 16), (128, 8)])
def test_few_rows_over_more_than_64_turns_of_a_wavefront(U, D, heads, bits):
    """So many requests that none is cut into parts (tiles * heads > 4095), one of about 20000 tokens: a wavefront's 64 turns are 8192 tokens
    (fp16) or 16384 (int8)."""
    rng = np.random.default_rng(D)
    ctx = rng.integers(0, 90, 600)
    ctx[411] = 20011
    gone = [(411, c) for c in (3, 127, 128, 129, 255, 256, 300)]
    r = aliased(U, D + bits, ctx.tolist(), [1] * 600, heads, 8, D, bits, 64, missing=gone)
    y = r.call(max_new=1)
    without_the_missing(r).check(y, rows=[0, 1, 63, 64, 255, 256, 410, 411, 412, 512, 599])
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("missing", [(), (1, 2, 61, 63, 64, 65, 67)])
def test_tiles_of_256_rows_over_more_than_64_tiles_of_tokens(U, missing, causal, bits):
    """4500 tokens and more before the new ones; pages (= tiles) missing at even and odd places and around the 64th."""
    r = aliased(U, 5, [4531, 4600], [400, 401], 64, 4, 128, bits, 64, missing=[(b, c) for b in range(2) for c in missing])
    y = r.call(causal=causal)
    rows = np.unique(np.r_[0, 15, 16, 399, 400, 415, 416, 800, np.random.default_rng(2).integers(0, r.T, 3)])
    without_the_missing(r).check(y, causal=causal, rows=rows)
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("requests,new_most,max_new", [(65, 1, 1), (130, 1, 1), (300, 3, 3), (70, 60, 0), (300, 9, 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_many_requests_without_parts(U, D, requests, new_most, max_new, bits):
    """More than 64 requests whose tables are too short for parts: the workgroups search all requests for their tile, the last first."""
    rng = np.random.default_rng(requests)
    ctx, new = rng.integers(0, 400, requests), rng.integers(0, new_most + 1, requests)
    new[-1], new[3] = new_most, 0
    r = aliased(U, requests, ctx.tolist(), new.tolist(), 4, 2, D, bits, 32)
    assert r.table.shape[1] * 32 <= 512
    y = r.call(max_new=max_new)
    r.check(y, rows=np.unique(np.r_[0, r.T - 1, rng.integers(0, r.T, 40)]))
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [128, 256])
@pytest.mark.parametrize("ctx,new,heads,kv_heads", [([300, 0, 41], [1, 1, 1], 8, 2), ([90, 700], [5, 3], 6, 1), ([33, 0], [70, 129], 4, 2)])
def test_every_token_sees_every_token_of_wider_heads(U, ctx, new, heads, kv_heads, D, bits):
    r = U.Requests(D, ctx, new, heads, kv_heads, D, bits, 32)
    r.check(r.call(causal=False), causal=False)
