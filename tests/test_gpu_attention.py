"""Attention over the paged cache against the oracle's 64 bits (tolerance: kv_util.Requests.check), at the sizes and masks where it can
go wrong: the caches hold 0xFF (NaN) wherever no token was written."""
import numpy as np
import pytest
import torch

from paper_2512_23367_amd import binding as ql

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def U():
    import kv_util
    return kv_util


#       ctx, new of the requests                                heads, kv_heads
SHAPES = [
    ([0], [1], 1, 1), ([0], [1], 12, 12), ([31], [1], 4, 4), ([300], [1], 12, 12), ([63, 64, 65], [1, 1, 1], 8, 2),
    ([1, 0, 700, 95, 0, 31], [1, 0, 1, 1, 2, 1], 8, 2), ([2000, 5, 130], [1, 1, 1], 32, 4), ([500, 77], [5, 3], 24, 4), ([40], [17], 3, 1),
    ([0], [100], 4, 2), ([0, 0, 0], [33, 1, 64], 2, 2), ([129], [200], 6, 1), ([1000, 0], [65, 300], 4, 1), ([0, 0], [0, 5], 10, 2),
    ([3], [9], 71, 1), ([5000], [1], 2, 1), ([4000], [70], 2, 2)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("D,page", [(64, 32), (128, 64), (256, 128)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_causal(U, shape, D, page, bits):
    ctx, new, heads, kv_heads = SHAPES[shape]
    r = U.Requests(shape, ctx, new, heads, kv_heads, D, bits, page)
    r.check(r.call())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("window", [1, 31, 64, 200])
@pytest.mark.parametrize("shape", [3, 5, 7, 11, 12, 16])
def test_window(U, shape, window, bits):
    ctx, new, heads, kv_heads = SHAPES[shape]
    r = U.Requests(shape, ctx, new, heads, kv_heads, 128, bits, 32)
    r.check(r.call(window=window), window=window)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("shape", [0, 5, 7, 9, 11])
def test_every_token_sees_every_token(U, shape, bits):
    ctx, new, heads, kv_heads = SHAPES[shape]
    r = U.Requests(shape, ctx, new, heads, kv_heads, 64, bits, 64)
    r.check(r.call(causal=False), causal=False)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("max_new", [1, 7, 1000])
def test_a_wrong_number_of_new_tokens_costs_time_only(U, max_new, bits):
    r = U.Requests(5, [100, 0, 2000, 9], [1, 40, 3, 150], 8, 2, 128, bits, 64)
    r.check(r.call(max_new=max_new))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("max_new", [0, 1])
def test_lengths_and_rows_that_leave_nothing(U, max_new, bits):
    """No token in the cache, fewer than the rows' positions (pages ran out), cu_new that starts late and ends early."""
    r = U.Requests(1, [0, 10, 50], [3, 40, 2], 4, 2, 64, bits, 32, kv_len=[0, 20, 52])
    r.check(r.call(max_new=max_new))
    late = U.Requests(2, [5, 5], [4, 6], 4, 2, 64, bits, 32)
    y = torch.full((14, 4 * 64), 7.0, dtype=torch.float16, device=U.DEV)
    q = torch.zeros((14, 4 * 64), dtype=torch.float16, device=U.DEV)
    q[2:12] = U.dev(late.q)
    late.cu = late.cu + 2
    late.call(q=q, y=y, max_new=max_new)
    assert (y[:2] == 7).all() and (y[12:] == 7).all()
    late.cu = late.cu - 2
    late.check(y[2:12])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [[1, 1], [40, 70]])
def test_strides_and_y_over_q(U, new, bits):
    r = U.Requests(4, [90, 333], new, 6, 2, 128, bits, 64)
    wide = torch.full((r.T, 6 * 128 + 2 * 2 * 128), float("nan"), dtype=torch.float16, device=U.DEV)
    q = wide[:, :6 * 128]
    q.copy_(U.dev(r.q))
    y = r.call(q=q)
    r.check(y)
    r.call(q=q, y=q)
    assert torch.equal(q, y) and torch.isnan(wide[:, 6 * 128:]).all()
    table = U.ints(np.concatenate([r.table, np.full((2, 3), 1 << 30)], 1))
    assert torch.equal(r.call(table=table[:, :r.table.shape[1]]), y)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [[1], [50]])
def test_large_scores_and_uneven_values(U, new, bits):
    """Scores of hundreds (weights that vanish), and value vectors whose sizes differ by factors up to 2^20."""
    r = U.Requests(6, [400], new, 4, 2, 128, bits, 64, k_gain=20.0)
    r.check(r.call(scale=0.5), scale=0.5)
    r.check(r.call(scale=-0.25), scale=-0.25)
    r.check(r.call(scale=0.0), scale=0.0)
    r = U.Requests(7, [400], new, 4, 2, 128, bits, 64, v_gain=lambda rng, n: 2.0 ** rng.integers(-14, 7, n))
    r.check(r.call())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [[3, 2], [70, 40]])
def test_tokens_that_are_not_finite_touch_only_who_sees_them(U, new, bits):
    ctx = [40, 100]
    r = U.Requests(8, ctx, new, 4, 2, 64, bits, 32)
    clean = r.call(window=60)
    # request 0, its second new token: NaN in head 1, as ql_kv_append stores it
    slot = int(U.slots_of(r.table, 0, [ctx[0] + 1], 32)[0])
    k, v = U.dev(r.k[0][ctx[0] + 1:ctx[0] + 2].reshape(1, -1).astype(np.float16)), U.dev(r.v[0][ctx[0] + 1:ctx[0] + 2].reshape(1, -1).astype(np.float16))
    v[0, 64 + 9] = float("inf")
    ql.ql_kv_append(None, k, v, None, None, U.ints([slot]), None, r.cache, r.fmt)
    y = r.call(window=60).view(r.T, 4, 64)
    clean = clean.view(r.T, 4, 64)
    for t in range(r.T):
        sees = 1 <= t < min(new[0], 1 + 60)
        assert torch.isnan(y[t, 2:]).all() if sees else torch.equal(y[t, 2:], clean[t, 2:]), t
    if bits == 16:                                    # (int8: requantizing the first head's rounded values may change its codes)
        assert torch.equal(y[:, :2], clean[:, :2])


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [[2, 1], [60, 90]])
def test_pages_outside_the_pool_are_not_seen(U, new, bits):
    r = U.Requests(9, [300, 64], new, 4, 2, 128, bits, 32)
    table = r.table.copy()
    table[0, 2], table[0, 5], table[1, 0] = -1, r.fmt.pages, 1 << 30
    y = r.call(table=U.ints(table))
    gone = [np.r_[64:96, 160:192], np.r_[0:32]]
    for b in range(2):
        r.k[b][gone[b]] = np.nan
    # the oracle on the tokens that are left, positions kept
    from oracle import kv
    got = y.cpu().numpy().astype(np.float64).reshape(-1, 4, 128)
    for b in range(2):
        left = np.setdiff1d(np.arange(r.len[b]), gone[b])
        for i in range(0, new[b], 7):
            seen = left[left <= r.ctx[b] + i]
            t = r.cu[b] + i
            ref, a, _, _ = kv.attention(r.q[t].reshape(1, 4, 128), r.k[b][seen], r.v[b][seen], [0], 128 ** -0.5, False, 0)
            assert (np.abs(got[t] - ref[0]) <= 2.0 ** -11 * np.abs(ref[0]) + 2.0 ** -10 * a[0] + 2.0 ** -16).all()


def test_long_caches_and_offsets_beyond_32_bits(U):
    """A pool of 5 GB whose pages lie at both ends; 40000 tokens for one new one."""
    D, page, bits, kv_heads, heads = 128, 64, 16, 4, 8
    n = 40000
    held = -(-n // page)
    pages = 40960
    fmt = ql.QlKvFormat(heads=kv_heads, head_dim=D, page_size=page, pages=pages, bits=bits)
    assert ql.ql_kv_cache_bytes(fmt) > 1 << 32
    cache = torch.full((ql.ql_kv_cache_bytes(fmt),), 0xFF, dtype=torch.uint8, device=U.DEV)
    g = torch.Generator(device=U.DEV)
    g.manual_seed(1)
    k, v = (torch.randn((n, kv_heads * D), generator=g, device=U.DEV).half() for _ in range(2))
    table = torch.cat([torch.arange(held // 2, device=U.DEV), pages - 1 - torch.arange(held - held // 2, device=U.DEV)]).int()[None].contiguous()
    at = torch.arange(n, device=U.DEV)
    slots = (table[0, at // page] * page + at % page).int()
    ql.ql_kv_append(None, k, v, None, None, slots, None, cache, fmt)
    q = torch.randn((1, heads * D), generator=g, device=U.DEV).half()
    y = torch.empty_like(q)
    ws = torch.empty(max(1, ql.ql_paged_attention_bytes(fmt, 1, 1, heads, 1)), dtype=torch.uint8, device=U.DEV)
    ql.ql_paged_attention(q, cache, fmt, table, U.ints([0, 1]), U.ints([n - 1]), U.ints([n]), D ** -0.5, y, ws, max_new=1)
    kk, vv, qq = k.double().view(n, kv_heads, D).permute(1, 2, 0).contiguous(), v.double().view(n, kv_heads, D).transpose(0, 1).contiguous(), q.double().view(kv_heads, 2, D)
    p = torch.softmax(torch.matmul(qq, kk) * D ** -0.5, -1)
    ref, a = torch.matmul(p, vv), torch.matmul(p, vv.abs())
    err = (y.double().view(kv_heads, 2, D) - ref).abs()
    assert (err <= 2.0 ** -11 * ref.abs() + a * (2.0 ** -11 + n * 2.0 ** -23) + 2.0 ** -24).all()
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    ql.ql_kv_read(cache, fmt, slots, kb, vb)
    assert torch.equal(kb, k) and torch.equal(vb, v)


def test_refusals_of_the_binding(U):
    r = U.Requests(1, [5], [2], 4, 2, 64, 16, 32)
    q, y = U.dev(r.q), U.dev(r.q)
    with pytest.raises(TypeError):
        r.call(q=q.float(), y=y)
    with pytest.raises(ValueError):
        r.call(q=q, y=y[:1])
    with pytest.raises(ValueError):
        r.call(q=q[:, :100], y=y[:, :100])
    with pytest.raises(ValueError):
        ql.ql_paged_attention(q, r.cache[:-1], r.fmt, U.ints(r.table), U.ints(r.cu), U.ints(r.ctx), U.ints(r.len), 1.0, y)
    with pytest.raises(ValueError):
        ql.ql_paged_attention(q, r.cache, r.fmt, U.ints(r.table), U.ints(r.cu)[:1], U.ints(r.ctx), U.ints(r.len), 1.0, y)
    with pytest.raises(ql.QlError) as e:
        ql.ql_paged_attention(q, r.cache, r.fmt, U.ints(r.table), U.ints(r.cu), None, U.ints(r.len), 1.0, y)
    assert e.value.status == 1


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("requests,new_most,max_new", [(63, 1, 1), (64, 3, 3), (65, 1, 1), (130, 60, 0), (300, 2, 2), (700, 1, 1)])
def test_many_requests(U, requests, new_most, max_new, bits):
    """Around and beyond a wavefront's and a workgroup's number of requests, one of them long, some with nothing to do."""
    rng = np.random.default_rng(requests)
    ctx, new = rng.integers(0, 90, requests), rng.integers(0, new_most + 1, requests)
    ctx[requests // 2], new[requests // 2], ctx[-1], new[-1] = 3000, 1, 700, new_most
    r = U.Requests(requests, ctx.tolist(), new.tolist(), 4, 2, 64, bits, 32)
    r.check(r.call(max_new=max_new), rows=np.unique(np.r_[rng.integers(0, r.T, 60), r.T - 1, r.cu[requests // 2]]))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("ctx,new,heads,kv_heads,window", [([0, 100], [900, 760], 32, 32, 0), ([0, 64, 5], [1200, 31, 900], 24, 8, 0), ([0, 700], [1000, 700], 32, 32, 300)])
def test_long_prompts(U, ctx, new, heads, kv_heads, window, bits):
    """Enough rows for the largest tiles; some of the rows against the oracle: the first and last ones, those around the tiles' borders."""
    r = U.Requests(30, ctx, new, heads, kv_heads, 128, bits, 64)
    y = r.call(window=window)
    g = heads // kv_heads
    edges = np.concatenate([c + np.arange(0, n, 256 // g) for c, n in zip(r.cu[:-1], new)])
    rows = np.unique(np.clip(np.concatenate([edges, edges + 1, edges - 1, r.cu[1:] - 1, np.random.default_rng(1).integers(0, r.T, 20)]), 0, r.T - 1))
    r.check(y, window=window, rows=rows)
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("max_new", [1, 0])
def test_first_rows_that_decrease_stay_inside_the_workspace(U, max_new):
    """cu_new [0, T, 0, T, ...] makes more of the workspace's items than the sizes allow for: the rest is left out, nothing behind it written."""
    r = U.Requests(6, [1500] * 60, [16] * 60, 8, 2, 128, 8, 64)
    need = ql.ql_paged_attention_bytes(r.fmt, r.T, 60, r.heads, max_new)
    room = torch.full((need + (4 << 20),), 0xA5, dtype=torch.uint8, device=U.DEV)
    q = U.dev(r.q)
    y = torch.full((r.T + 64, q.shape[1]), 5.0, dtype=torch.float16, device=U.DEV)
    cu = U.ints([0, r.T] * 30 + [0])
    ql.ql_paged_attention(q, r.cache, r.fmt, U.ints(r.table), cu, U.ints(r.ctx), U.ints(r.len), r.D ** -0.5, y[:r.T], room[:need], max_new=max_new)
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xA5).all()) and bool((y[r.T:] == 5).all())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 150), (False, 0)])
@pytest.mark.parametrize("ctx,new,kv_heads", [([0, 500, 3, 100, 0, 40], [400, 1, 0, 700, 129, 270], 32), ([7 * i % 90 for i in range(50)], [11 * i % 61 for i in range(50)], 64)])
def test_whole_tiles_of_ragged_requests(U, ctx, new, kv_heads, causal, window, bits):
    """More tiles than are cut into parts, in either order in which workgroups take them."""
    r = U.Requests(7, ctx, new, kv_heads, kv_heads, 64, bits, 32)
    r.check(r.call(causal=causal, window=window), causal=causal, window=window)


@pytest.mark.parametrize("bits", [16, 8])
def test_whole_tiles_over_long_contexts(U, bits):
    """More than 64 tiles of tokens for one workgroup, whose table entries are looked up 64 tiles at a time."""
    r = U.Requests(8, [4500, 90], [520, 600], 64, 64, 64, bits, 32)
    rows = np.unique(np.r_[0, 127, 128, 519, 520, 647, 1119, np.random.default_rng(8).integers(0, r.T, 12)])
    r.check(r.call(), rows=rows)
