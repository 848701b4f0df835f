"""Bookkeeping, filling and reading of the paged cache on the GPU, against the oracle: whole numbers, codes and fp16 values are equal,
stored bytes too (they are functions of the stated fp32 steps; the logarithm of a value scale within 2^-20 of |log2| + 1)."""
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


def _pool(rng, old, page, columns, extra, pages=None):
    from kv_util import tables
    table, n = tables(rng, old, page, spare=extra, columns=columns)
    used = set(table[table >= 0].tolist())
    free = [p for p in rng.permutation(n).tolist() if p not in used]
    head = int(rng.integers(n))
    ring = np.full(n, -7, np.int32)
    ring[(head + np.arange(len(free))) % n] = free
    return table, ring, [head, len(free), 99, 0]


def _resize(U, page, old, want, ring, pool, table, room, in_place):
    n = len(old)
    d = dict(ring=U.ints(ring), pool=U.ints(pool), table=U.ints(table), kv_len=U.ints([-3] * n), cu=U.ints([-3] * (n + 1)),
             slots=U.ints([-3] * max(room, 1))[:room], positions=U.ints([-3] * max(room, 1))[:room])
    out = d["pool"] if in_place else U.ints([5, 5, 5, 0])
    ql.ql_kv_resize(page, U.ints(old), U.ints(want), d["ring"], d["pool"], out, d["table"], d["kv_len"], d["cu"], d["slots"], d["positions"])
    torch.cuda.synchronize()
    return {k: v.cpu().numpy() for k, v in {**d, "pool": out}.items()}


CASES = [
    # requests, page, columns, most old, most new, share that shrinks, spare pages
    (1, 64, 4, 0, 1, 0.0, 2), (1, 32, 3, 96, 0, 1.0, 1), (5, 32, 8, 200, 40, 0.4, 9), (64, 64, 20, 1000, 3, 0.1, 40), (64, 64, 20, 1000, 90, 0.1, 5),
    (300, 128, 10, 900, 400, 0.3, 500), (1025, 32, 6, 150, 60, 0.5, 100), (4096, 32, 3, 60, 40, 0.2, 3000), (7, 1024, 2, 2048, 1500, 0.3, 4), (3, 32, 500, 100, 12000, 0.0, 1100)]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n,page,columns,old_most,new_most,shrink,spare", CASES)
def test_resize(U, n, page, columns, old_most, new_most, shrink, spare, in_place):
    rng = np.random.default_rng(n + page)
    old = rng.integers(0, min(old_most, columns * page) + 1, n)
    want = np.where(rng.random(n) < shrink, (old * rng.random(n)).astype(int) * (rng.random(n) < 0.7), old + rng.integers(0, new_most + 1, n))
    old, want = old.tolist(), want.tolist()
    table, ring, pool = _pool(rng, old, page, columns, spare)
    total = sum(max(0, w - o) for o, w in zip(old, want))
    for room in (total + 6, max(0, total // 2)):              # rows to spare, and too few
        ref = kv.resize(old, want, page, ring.tolist(), pool, table.tolist(), room)
        got = _resize(U, page, old, want, ring, pool, table, room, in_place)
        for name in ("ring", "pool", "table", "kv_len", "cu"):
            assert (got[name] == np.array(ref[name])).all(), name
        m = len(ref["slots"])
        for name in ("slots", "positions"):
            assert (got[name][:m] == np.array(ref[name], dtype=int)).all() and (got[name][m:] == -3).all(), name


def test_resize_of_no_requests_and_of_odd_lengths(U):
    got = _resize(U, 32, [], [], [4, 5, 6], [1, 2, 9, 0], np.zeros((0, 4), np.int32), 4, False)
    assert got["cu"].tolist() == [0] and got["pool"].tolist() == [1, 2, 0, 0] and (got["slots"] == -3).all()
    # negative lengths count as 0, an old length beyond the table as the table's
    table = np.array([[0, 1], [-1, -1]], np.int32)
    got = _resize(U, 32, [1000, -5], [0, -9], [9, 9, 9, 9], [0, 0, 0, 0], table, 4, True)
    assert got["kv_len"].tolist() == [0, 0] and got["pool"].tolist() == [0, 2, 0, 0] and got["ring"][:2].tolist() == [0, 1]


def test_resize_steps_keep_every_page_once(U):
    """Forty steps in place: what the table holds and what the ring holds are together always the pool, each page once."""
    rng = np.random.default_rng(3)
    n, page, columns, pages = 33, 32, 9, 150
    ring, pool, table = U.ints(np.arange(pages)), U.ints([0, pages, 0, 0]), U.ints(np.full((n, columns), -1))
    length, cu, room = U.ints([0] * n), U.ints([0] * (n + 1)), 4000
    slots, positions = U.ints([0] * room), U.ints([0] * room)
    host = np.zeros(n, int)
    for _ in range(40):
        want = np.where(rng.random(n) < 0.15, 0, np.minimum(host + rng.integers(0, 60, n), columns * page))
        new = U.ints([0] * n)
        ql.ql_kv_resize(page, length, U.ints(want), ring, pool, pool, table, new, cu, slots, positions)
        length, host = new, new.cpu().numpy()
        head, free, lost, zero = pool.cpu().tolist()
        held = [p for b in range(n) for p in table.cpu().numpy()[b, :-(-int(host[b]) // page)]]
        left = ring.cpu().numpy()[(head + np.arange(free)) % pages].tolist()
        assert sorted(held + left) == list(range(pages)) and zero == 0
        assert (host <= want).all() and lost == (want - host).sum()


def _bytes_match(got, ref, D, bits, heads, page):
    if bits == 16:
        assert (got == ref).all()
        return
    g, r = got.reshape(-1, kv.block_bytes(D, 8)), ref.reshape(-1, kv.block_bytes(D, 8))
    assert (g[:, :64 * D + 256] == r[:, :64 * D + 256]).all()                          # codes, scales
    gs, rs = (np.ascontiguousarray(x[:, 64 * D:]).view(np.float32).reshape(-1, 4, 32) for x in (g, r))
    wrote = (r[:, 64 * D:].reshape(-1, 4, 32, 4) != 0xEE).any(-1)
    assert (np.abs(gs - rs)[:, 2][wrote[:, 2]] <= 2.0 ** -20 * (np.abs(rs[:, 2][wrote[:, 2]]) + 1)).all()
    assert (gs[:, 3].view(np.uint32) == rs[:, 3].view(np.uint32)).all()


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("T,heads,kv_heads,D,rotary,page,order", [
    (1, 4, 4, 64, 64, 32, "near"), (3, 6, 2, 128, 128, 64, "near"), (33, 8, 8, 128, 64, 32, "near"), (70, 5, 1, 256, 256, 128, "near"), (257, 12, 12, 128, 128, 64, "near"),
    (100, 4, 2, 64, 32, 32, "any"), (500, 2, 2, 128, 16, 256, "any"), (41, 0, 3, 128, 0, 64, "near"), (41, 0, 3, 64, 48, 64, "any"), (1025, 4, 2, 256, 128, 1024, "near"),
    (700, 8, 2, 64, 64, 64, "gaps"), (700, 3, 3, 128, 128, 64, "gaps")])
def test_append_and_read(U, bits, T, heads, kv_heads, D, rotary, page, order):
    rng = np.random.default_rng(T + D)
    pages = -(-2 * T // page) + 2
    fmt = ql.QlKvFormat(heads=kv_heads, head_dim=D, page_size=page, pages=pages, bits=bits)
    if order == "any":
        slots = rng.permutation(pages * page)[:T]
    else:
        first = int(rng.integers(page))
        slots = first + np.arange(T) + (np.cumsum(rng.random(T) < 0.1) if order == "gaps" else 0)
    slots = slots.astype(np.int64)
    off = rng.random(T) < 0.15 if T > 3 else np.zeros(T, bool)
    given = np.where(off, rng.choice([-1, pages * page, -2 ** 31, 2 ** 31 - 1], T), slots)
    width = (heads + 2 * kv_heads) * D + 8
    qkv = rng.standard_normal((T, width)).astype(np.float16)
    k, v = qkv[:, heads * D:(heads + kv_heads) * D], qkv[:, (heads + kv_heads) * D:(heads + 2 * kv_heads) * D]
    k[:, ::17] *= 12
    if T > 3:
        k[1], v[2] = 0, 0
        v[0, :] = 2.0 ** -24
        k[3, 5] = np.inf                                                              # head 0 of token 3
        v[T - 1, -1] = np.nan                                                         # the last head of the last token
    most = 50
    cos_sin = rng.standard_normal((most, max(rotary, 1))).astype(np.float32)
    positions = rng.integers(-3, most + 3, T)
    kr = kv.rotate(k.reshape(T, kv_heads, D), cos_sin, positions, rotary)
    vr = v.reshape(T, kv_heads, D).astype(np.float32)
    ks, vs = kv.stored(kr, vr, bits)
    bad = np.isnan(ks).any(-1)

    d = U.dev(qkv)
    cache = torch.full((ql.ql_kv_cache_bytes(fmt),), 0xEE, dtype=torch.uint8, device=U.DEV)
    q = d[:, :heads * D] if heads else None
    q_out = torch.full((T, heads * D + 8), float("nan"), dtype=torch.float16, device=U.DEV)[:, :heads * D] if heads else None
    args = (U.dev(cos_sin) if rotary else None, U.ints(positions) if rotary else None, U.ints(given))
    ql.ql_kv_append(q, d[:, heads * D:(heads + kv_heads) * D], d[:, (heads + kv_heads) * D:(heads + 2 * kv_heads) * D], *args, q_out, cache, fmt)
    if heads:
        with np.errstate(over="ignore"):
            ref = kv.rotate(qkv[:, :heads * D].reshape(T, heads, D), cos_sin, positions, rotary).astype(np.float16).reshape(T, -1)
        assert (q_out.cpu().numpy() == ref).all()
        assert (d.cpu().numpy()[:, :heads * D] == qkv[:, :heads * D]).all()
        ql.ql_kv_append(q, d[:, heads * D:(heads + kv_heads) * D], d[:, (heads + kv_heads) * D:(heads + 2 * kv_heads) * D], *args, q, cache, fmt)   # over q itself, same slots again
        assert (d.cpu().numpy()[:, :heads * D] == ref).all()

    ref = np.full(cache.numel(), 0xEE, np.uint8)
    kp, vp = np.where(bad[..., None], np.nan, kr), np.where(bad[..., None], 0, vr)
    keep = ~off
    with np.errstate(all="ignore"):
        kv.pack(ref, kv_heads, D, page, bits, slots[keep], np.where(bad[..., None] & (bits == 8), 0, kp)[keep].astype(np.float32), vp[keep].astype(np.float32))
    got = cache.cpu().numpy()
    if bits == 8:                                     # the key scale of a token that is not finite: NaN, whatever its bits
        at_s = (((slots // page)[:, None] * kv_heads + np.arange(kv_heads)) * (page // 32) + (slots % page // 32)[:, None]) * kv.block_bytes(D, 8) + 64 * D + (slots % 32)[:, None] * 4
        for at in at_s[bad & keep[:, None]]:
            assert np.isnan(got[at:at + 4].view(np.float32)).all()
            ref[at:at + 4] = got[at:at + 4]
        _bytes_match(got, ref, D, bits, kv_heads, page)
    else:
        g, r = got.view(np.float16), ref.view(np.float16)
        assert (np.isnan(g) == np.isnan(r)).all() and ((g.view(np.uint16) == r.view(np.uint16)) | np.isnan(r)).all()

    kb, vb = (torch.full((T, kv_heads * D + 8), float("nan"), dtype=torch.float16, device=U.DEV)[:, :kv_heads * D] for _ in range(2))
    ql.ql_kv_read(cache, fmt, U.ints(given), kb, vb)
    want_k, want_v = (np.where(off[:, None], 0, x.reshape(T, -1)).astype(np.float16) for x in (ks, vs))
    # code * scale: one fp32 rounding before the one to fp16, so a value next to a border may come out one step away from the oracle's
    for g, w in ((kb.cpu().numpy(), want_k), (vb.cpu().numpy(), want_v)):
        g, w = g.astype(np.float64), w.astype(np.float64)
        assert (np.isnan(g) == np.isnan(w)).all()
        fine = ~np.isnan(w)
        assert (np.abs(g - w)[fine] <= (0 if bits == 16 else 2.0 ** -10) * np.abs(w[fine]) + (0 if bits == 16 else 2.0 ** -24)).all()
    only = torch.zeros((T, kv_heads * D), dtype=torch.float16, device=U.DEV)
    ql.ql_kv_read(cache, fmt, U.ints(given), None, only)
    assert torch.equal(only.view(torch.int16), vb.contiguous().view(torch.int16))
