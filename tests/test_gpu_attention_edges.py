"""Attention over the paged cache where its kernels' loops, searches and number formats end: contexts beyond what a wavefront looks up of
the block table at once, batches without parts, every token seen by every token in every kernel.  Long contexts are few pages that
occur many times in a block table."""
import numpy as np
import pytest
import torch

from oracle import kv
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


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 1], [60, 140]])
def test_queries_that_are_not_finite(U, new, D, bits):
    """One of them makes every score of its row infinite or NaN, so its row is NaN, with whatever number of tokens it sees (exp(-inf) / 0 where all of its
    scores are -inf); a row that sees nothing is 0 still.  Nobody else is touched."""
    r = U.Requests(D, [0, 77], new, 4, 2, D, bits, 32)
    clean = r.call()
    r.check(clean)
    empty = U.Requests(D, [0, 0], new, 4, 2, D, bits, 32, kv_len=[0, 0])
    for what in (float("inf"), float("-inf"), float("nan")):
        for t in {0, r.T - 1, new[0]}:
            for head in (0, 3):
                for channel in (0, D // 2 + 9, D - 1):
                    q = U.dev(r.q)
                    q[t, head * D + channel] = what
                    y = r.call(q=q).view(r.T, 4, D)
                    assert torch.isnan(y[t, head]).all(), (what, t, head, channel)
                    y[t, head] = clean.view(r.T, 4, D)[t, head]
                    r.check(y, rows=[t, max(0, t - 1), min(r.T - 1, t + 1)])
                    assert (empty.call(q=q) == 0).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("new", [[1, 1], [60, 140]])
def test_queries_below_the_normal_range_of_fp16(U, new, D, bits):
    r = U.Requests(D + 1, [9, 77], new, 4, 2, D, bits, 32)
    r.q = (r.q.astype(np.float32) * 2.0 ** -18).astype(np.float16)
    scale = 2.0 ** 18 * D ** -0.5
    r.check(r.call(scale=scale), scale=scale)


def _tail(U, bits, D, kv_heads, t, v_tail, n):
    """A cache of two pages of 1024 tokens, key (score in powers of two, 0, 0, ...): a first token of score 0 and value 1, all others of score -t
    and value v_tail; block table entries for n tokens."""
    fmt = ql.QlKvFormat(heads=kv_heads, head_dim=D, page_size=1024, pages=2, bits=bits)
    cache = torch.full((ql.ql_kv_cache_bytes(fmt),), 0xFF, dtype=torch.uint8, device=U.DEV)
    k = torch.zeros((2048, kv_heads, D), dtype=torch.float16, device=U.DEV)
    v = torch.full_like(k, v_tail)
    k[1:, :, 0], v[0] = -t, 1.0
    ql.ql_kv_append(None, k.view(2048, -1), v.view(2048, -1), None, None, U.ints(np.arange(2048)), None, cache, fmt)
    return fmt, cache, [0] + [1] * (n // 1024 - 1)


def _check_tail(y, t, v_tail, n, adds):
    """y = (1 + tail v_tail) / (1 + tail), tail = (n - 1) 2^-t; sum p |v| / sum p = 1.  Off by: y rounded to fp16, 2^-11 |y|; the weights rounded to fp16, 2^-11 in
    all (the first one is a power of two); weights below fp16's normal range, which the largest one is 2^7 of at least: 2^-32 each in the sum of the
    values and in that of the weights; `adds` additions to a sum, each within a step of 2^-23; scores: 2^-22 (|score| + 4), 32 2^-23 for the logarithm of the scale, twice."""
    tail = (n - 1) * 2.0 ** -t
    ref = (1 + tail * v_tail) / (1 + tail)
    tol = 2.0 ** -11 * abs(ref) + 2.0 ** -11 + 2 * n * 2.0 ** -32 + adds * 2.0 ** -23 + 2 * (2.0 ** -22 * (t + 4) + 32 * 2.0 ** -23) + 2.0 ** -24
    err = (y.double() - ref).abs().max().item()
    assert err <= tol, f"{err:.3g}, tolerance {tol:.3g}"


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("t", [16, 20.5, 23.25, 24.9375, 25.0625, 27, 30])
@pytest.mark.parametrize("v_tail", [1.0, -1.0])
def test_a_long_tail_of_small_weights_few_rows(U, v_tail, t, D, bits):
    """One token ahead of 2^19 others, none cut into parts: the wavefront that holds the first one adds up a quarter of the others beside it, 32 at a time."""
    n, requests = 1 << 19, 4200
    fmt, cache, entries = _tail(U, bits, D, 1, t, v_tail, n)
    table = torch.zeros((requests, len(entries)), dtype=torch.int32, device=U.DEV)
    table[7] = U.ints(entries)
    length = torch.ones(requests, dtype=torch.int32, device=U.DEV)
    length[7] = n
    q = torch.zeros((requests, D), dtype=torch.float16, device=U.DEV)
    q[:, 0] = 1
    y = torch.zeros_like(q)
    ws = torch.empty(max(1, ql.ql_paged_attention_bytes(fmt, requests, requests, 1, 1)), dtype=torch.uint8, device=U.DEV)
    ql.ql_paged_attention(q, cache, fmt, table, U.ints(np.arange(requests + 1)), None, length, float(np.log(2)), y, ws, causal=False, max_new=1)
    _check_tail(y[7], t, v_tail, n, n / 4 / 32)
    assert (y[:7] == 1).all() and (y[8:] == 1).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("t", [16, 20.5, 23.25, 24.9375, 25.0625, 27, 30])
@pytest.mark.parametrize("v_tail", [1.0, -1.0])
def test_a_long_tail_of_small_weights_many_rows(U, v_tail, t, D, bits):
    """The same in tiles of 128 (D = 128: 256) rows, too many of them for parts: 120832 tokens, 16 at a time."""
    n, T, heads, kv_heads = 118 * 1024, 1100, 64, 4
    fmt, cache, entries = _tail(U, bits, D, kv_heads, t, v_tail, n)
    q = torch.zeros((T, heads, D), dtype=torch.float16, device=U.DEV)
    q[..., 0] = 1
    y = torch.zeros((T, heads * D), dtype=torch.float16, device=U.DEV)
    ql.ql_paged_attention(q.view(T, -1), cache, fmt, U.ints([entries]), U.ints([0, T]), None, U.ints([n]), float(np.log(2)), y,
                          torch.empty(max(1, ql.ql_paged_attention_bytes(fmt, T, 1, heads)), dtype=torch.uint8, device=U.DEV), causal=False)
    _check_tail(y, t, v_tail, n, n / 16)


def _cache_of(U, k, v, bits, page=64):
    """A cache that holds fp32 keys and values [tokens, kv_heads, D] in its first slots, and a block table of one request."""
    n, kv_heads, D = k.shape
    pages = -(-n // page)
    fmt = ql.QlKvFormat(heads=kv_heads, head_dim=D, page_size=page, pages=pages, bits=bits)
    cache = torch.full((ql.ql_kv_cache_bytes(fmt),), 0xFF, dtype=torch.uint8, device=U.DEV)
    ql.ql_kv_append(None, U.dev(k.reshape(n, -1).astype(np.float16)), U.dev(v.reshape(n, -1).astype(np.float16)), None, None, U.ints(np.arange(n)), None, cache, fmt)
    return fmt, cache, U.ints([list(range(pages))])


def _attend(U, fmt, cache, table, q, n, scale, heads):
    """All rows see all n tokens: y [T, heads, D]."""
    T = q.shape[0]
    y = torch.full((T, heads * fmt.head_dim), float("nan"), dtype=torch.float16, device=U.DEV)
    ws = torch.empty(max(1, ql.ql_paged_attention_bytes(fmt, T, 1, heads)), dtype=torch.uint8, device=U.DEV)
    ql.ql_paged_attention(q.reshape(T, -1), cache, fmt, table, U.ints([0, T]), None, U.ints([n]), scale, y, ws, causal=False)
    return y.view(T, heads, fmt.head_dim).double().cpu().numpy()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("rows", [1, 30])
@pytest.mark.parametrize("n", [50, 3000])
def test_scores_of_any_size(U, n, rows, D, bits):
    """Scores from 2^8 to 2^39: the keys are multiples 0 .. 47 of a vector, the largest one's token has 47 / 46 of the next score and takes the whole
    row; where two tokens have it, each half.  Off by: y rounded, 2^-11 |y|; the weight rounded, 2^-11; the halves by ds of the larger value, the
    scores' error: fp16, equal keys have equal scores, and what is rounded once the maximum (up to 2^10) is subtracted is 2^-14 each; int8, 2^-22 (score + 4) and
    32 2^-23 for the logarithm of the scale of v."""
    rng = np.random.default_rng(n + rows)
    kv_heads, heads = 2, 8
    for a in (2.0, 31.0, 500.0, 3000.0, 20000.0, 60000.0):
        for top in ((0,), (n - 1,), (n // 2,), (3, n - 2)):
            g = rng.integers(0, 47, (n, kv_heads))
            g[list(top)] = 47
            sign = rng.choice([-1.0, 1.0], D)
            k = (g[..., None] * sign * (a / 64)).astype(np.float16).astype(np.float32)
            v = rng.standard_normal((n, kv_heads, D)).astype(np.float16).astype(np.float32)
            held = kv.stored(k, v, bits)[1][list(top)].repeat(heads // kv_heads, 1)
            fmt, cache, table = _cache_of(U, k, v, bits)
            q = U.dev(np.broadcast_to(sign * a, (rows, heads, D)).astype(np.float16))
            for scale in (D ** -0.5, 1.0):
                score = a * a / 64 * 47 * D * scale
                if score / 47 < 30:                   # (the second one would still count)
                    continue
                y = _attend(U, fmt, cache, table, q, n, scale, heads)
                ds = 2.0 ** -13 if bits == 16 else 2.0 ** -22 * (score + 4) + 32 * 2.0 ** -23
                tol = 2.0 ** -10 * np.abs(held).max(0) + 2.0 ** -24 + (min(1.0, 2 * ds) * np.abs(held[0] - held[1]) if len(top) == 2 else 0)
                err = np.abs(y - held.mean(0))
                assert (err <= tol).all(), (a, top, scale, err.max())


@pytest.mark.parametrize("rows", [1, 30])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("power", [8, 20, 23, 24])
@pytest.mark.parametrize("ahead", [2.0, 6.0, 8.0, 10.0, 16.0])
def test_a_maximum_that_follows_late_at_large_scores(U, ahead, power, D, rows):
    """Two scores 2^power and 2^power + ahead (exact in fp32) in different turns of a wavefront, all others 0: weights 2^-ahead and 1, whichever comes first."""
    n = 300
    for first, second in ((0, 128), (128, 0), (5, 261), (1, 70)):
        k = np.zeros((n, 1, D))
        k[first, 0, 0] = k[second, 0, 0] = 2.0 ** (power - power // 2)
        k[second, 0, 1] = ahead
        v = np.zeros((n, 1, D))
        v[first], v[second] = 1.0, -1.0
        fmt, cache, table = _cache_of(U, k, v, 16)
        q = np.zeros((rows, 4, D), np.float16)
        q[..., 0], q[..., 1] = 2.0 ** (power // 2), 1.0
        y = _attend(U, fmt, cache, table, U.dev(q), n, float(np.log(2)), 4)
        w = 2.0 ** -ahead
        # the score times scale and log2 e: off by 2^-22 of itself for both alike, their difference by 2^-22 of the difference; y rounded
        assert np.abs(y - (w - 1) / (w + 1)).max() <= 2.0 ** -11 + 2.0 ** -16, (first, second, y[0, 0, 0])
