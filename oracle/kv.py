"""Oracle of the paged key/value cache and the attention over it: plain numpy, 64 bits where values are computed, one IEEE
fp32 operation per line where the operator states its fp32 steps.  Keys and values are arrays [slots, heads, D] here;
pack() and unpack() go by the documented byte layout, element by element."""
from __future__ import annotations

import numpy as np

NOTHING = np.float32(2.0 ** -100)


def resize(old, want, page, ring, pool, table, max_tokens):
    """One step of the bookkeeping, request by request.  ring, table: lists (changed copies are returned)."""
    ring, table, n_pages = list(ring), [list(r) for r in table], len(ring)
    columns = len(table[0]) if table else 0
    head, free, cap = pool[0], pool[1], columns * page
    out_ring = list(ring)
    taken = given = lost = 0
    wanted = 0                                        # pages asked for so far, met or not
    cu, kv_len, slots, positions = [0], [], [], []
    for b, (o, w) in enumerate(zip(old, want)):
        o, w = min(max(o, 0), cap), max(w, 0)
        has = -(-o // page)
        if w < o:
            keeps = -(-w // page)
            for j in range(keeps, has):
                out_ring[(head + free + given) % n_pages] = table[b][j]
                given += 1
            kv_len.append(w)
            cu.append(cu[-1])
            continue
        n = min(w - o, max_tokens - cu[-1])
        target = min(o + n, cap)
        have = has
        for j in range(has, -(-target // page)):
            if wanted < free:
                table[b][j] = ring[(head + wanted) % n_pages]
                taken += 1
                have = j + 1
            wanted += 1
        length = min(target, have * page)
        for i in range(n):
            p = o + i
            positions.append(p)
            slots.append(table[b][p // page] * page + p % page if p < length else -1)
        lost += w - length                            # for want of a page, a column or a row
        kv_len.append(length)
        cu.append(cu[-1] + n)
    pool_out = [(head + taken) % n_pages, free - taken + given, lost, 0]
    return dict(ring=out_ring, pool=pool_out, table=table, kv_len=kv_len, cu=cu, slots=slots, positions=positions)


def rotate(x, cos_sin, positions, rotary):
    """x fp16 [T, heads, D] -> fp32, in the stated fp32 steps (each product rounded, then each sum)."""
    y = x.astype(np.float32)
    half = rotary // 2
    at = np.clip(positions, 0, len(cos_sin) - 1)
    co, si = cos_sin[at][:, None, :half], cos_sin[at][:, None, half:]
    a, b = y[..., :half].copy(), y[..., half:rotary].copy()
    y[..., :half] = np.multiply(a, co) - np.multiply(b, si)
    y[..., half:rotary] = np.multiply(b, co) + np.multiply(a, si)
    return y


def quantize(x):
    """x fp32 [..., D] -> codes (int), scale fp32 [...]."""
    amax = np.abs(x).max(-1).astype(np.float32)
    some = amax >= NOTHING
    inv = np.divide(np.float32(127), np.where(some, amax, np.float32(1)))
    codes = np.clip(np.rint(np.multiply(x, inv[..., None])), -127, 127).astype(np.int32)
    scale = np.where(some, np.divide(amax, np.float32(127)), np.float32(2.0 ** -31)).astype(np.float32)
    return np.where(some[..., None], codes, 0), scale


def stored(k, v, bits):
    """What the cache holds of fp32 keys (after the rotation) and values [T, heads, D], in 64 bits."""
    if bits == 16:
        with np.errstate(over="ignore"):
            k, v = k.astype(np.float16).astype(np.float64), v.astype(np.float64)
        fine = (np.isfinite(k) & np.isfinite(v)).all(-1)
    else:
        fine = (np.isfinite(k) & np.isfinite(v)).all(-1)
        kc, ks = quantize(np.where(fine[..., None], k, 0).astype(np.float32))
        vc, vs = quantize(np.where(fine[..., None], v, 0).astype(np.float32))
        k, v = kc * ks.astype(np.float64)[..., None], vc * vs.astype(np.float64)[..., None]
    return np.where(fine[..., None], k, np.nan), np.where(fine[..., None], v, 0.0)


def block_bytes(D, bits):
    return 32 * D * 2 * bits // 8 + (512 if bits == 8 else 0)


def key_offset(token, c, D, bits):
    if bits == 16:
        return (c // 16) * 1024 + (c // 8 % 2) * 512 + token * 16 + c % 8 * 2
    return (c // 32) * 1024 + (c // 16 % 2) * 512 + token * 16 + c % 16


def value_offset(token, c, D, bits):
    # token = 16 s + 8 jh + 4 h + jl
    s, jh, h, jl = token // 16, token // 8 % 2, token // 4 % 2, token % 4
    if bits == 16:
        return 64 * D + (c // 32) * 2048 + s * 1024 + h * 512 + c % 32 * 16 + (4 * jh + jl) * 2
    return 32 * D + (c // 32) * 1024 + h * 512 + c % 32 * 16 + 8 * s + 4 * jh + jl


def pack(cache, heads, D, page, bits, slots, k, v):
    """Writes fp32 keys and values [T, heads, D] to their slots of a cache (uint8, changed in place)."""
    slots = np.asarray(slots, dtype=np.int64)
    channel = np.arange(D)
    rest, h = slots % page, np.arange(heads)
    at = (((slots // page)[:, None] * heads + h) * (page // 32) + (rest // 32)[:, None]) * block_bytes(D, bits)    # [T, heads]
    token = (rest % 32)[:, None, None]
    at_k = at[..., None] + key_offset(token, channel, D, bits)
    at_v = at[..., None] + value_offset(token, channel, D, bits)
    if bits == 16:
        cache.view(np.float16)[at_k // 2] = k.astype(np.float16)
        cache.view(np.float16)[at_v // 2] = v.astype(np.float16)
        return
    (kc, ks), (vc, vs) = quantize(k), quantize(v)
    cache[at_k] = (kc + 128).astype(np.uint8)
    cache[at_v] = (vc + 128).astype(np.uint8)
    at_s = (at + 64 * D) // 4 + token[..., 0]
    for i, s in enumerate((ks, vs, np.log2(vs), np.float32(1) / vs)):
        cache.view(np.float32)[at_s + 32 * i] = s


def attention(q, k, v, positions, scale, causal, window):
    """q [n, heads, D] fp16, k, v [len, kv_heads, D] in 64 bits -> (y, per row: sum p |v| / sum p, largest sum |q k|, number of tokens).
    Tokens that a row does not see take no part, whatever they hold."""
    n, heads, D = q.shape
    group = heads // k.shape[1] if len(k) else 1
    y, a = np.zeros((n, heads, D)), np.zeros((n, heads, D))
    spread, seen = np.zeros((n, heads)), np.zeros(n)
    for i in range(n):
        low, high = 0, len(k)
        if causal:
            high = min(high, int(positions[i]) + 1)
            low = max(0, int(positions[i]) - window + 1) if window else 0
        if high <= low:
            continue
        seen[i] = high - low
        kk, vv = k[low:high].astype(np.float64), v[low:high].astype(np.float64)
        for h in range(heads):
            qh = q[i, h].astype(np.float64)
            s = scale * (kk[:, h // group] @ qh)
            spread[i, h] = abs(scale) * (np.abs(kk[:, h // group]) @ np.abs(qh)).max()
            p = np.exp(s - s.max())
            y[i, h] = p @ vv[:, h // group] / p.sum()
            a[i, h] = p @ np.abs(vv[:, h // group]) / p.sum()
    return y, a, spread, seen
