"""Helpers of the paged cache's GPU tests: requests laid out on the host, the oracle's cache as a device buffer."""
from __future__ import annotations

import numpy as np
import torch

from oracle import kv
from paper_2512_23367_amd import binding as ql

DEV = "cuda:0"


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def ints(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def tables(rng, lengths, page, spare=3, columns=None):
    """Block table [requests, columns] with pages in no order, and the number of pages."""
    held = [-(-n // page) for n in lengths]
    columns = columns or max(held + [1]) + 1
    pages = sum(held) + spare
    ids = rng.permutation(pages)
    t = np.full((len(lengths), columns), -1, np.int32)
    at = 0
    for b, n in enumerate(held):
        t[b, :n] = ids[at:at + n]
        at += n
    return t, pages


def slots_of(table, b, positions, page):
    positions = np.asarray(positions)
    return table[b, positions // page].astype(np.int64) * page + positions % page


class Requests:
    """Requests with `ctx` tokens before and `new` ones, keys and values of all in a packed cache whose other bytes are `rubbish`."""

    def __init__(self, seed, ctx, new, heads, kv_heads, D, bits, page, kv_len=None, k_gain=1.0, v_gain=None, rubbish=0xFF):
        rng = np.random.default_rng(seed)
        self.ctx, self.new, self.D, self.bits, self.page, self.heads, self.kv_heads = ctx, new, D, bits, page, heads, kv_heads
        self.len = [c + n for c, n in zip(ctx, new)] if kv_len is None else kv_len
        self.table, pages = tables(rng, self.len, page)
        self.fmt = ql.QlKvFormat(heads=kv_heads, head_dim=D, page_size=page, pages=pages, bits=bits)
        cache = np.full(ql.ql_kv_cache_bytes(self.fmt), rubbish, np.uint8)
        self.k, self.v = [], []
        for b, n in enumerate(self.len):
            k = (k_gain * rng.standard_normal((n, kv_heads, D))).astype(np.float16).astype(np.float32)
            v = rng.standard_normal((n, kv_heads, D)).astype(np.float16).astype(np.float32)
            if v_gain is not None:
                v = (v * v_gain(rng, n)[:, None, None]).astype(np.float16).astype(np.float32)
            if n:
                kv.pack(cache, kv_heads, D, page, bits, slots_of(self.table, b, np.arange(n), page), k, v)
            ks, vs = kv.stored(k, v, bits) if n else (k, v)
            self.k.append(ks)
            self.v.append(vs)
        self.cache = torch.from_numpy(cache).to(DEV)
        self.T = sum(new)
        self.q = rng.standard_normal((self.T, heads * D)).astype(np.float16)
        self.cu = np.concatenate([[0], np.cumsum(new)])

    def call(self, scale=None, causal=True, window=0, max_new=0, q=None, y=None, ws=None, table=None):
        q = dev(self.q) if q is None else q
        y = torch.full_like(q, float("nan")) if y is None else y
        n = len(self.ctx)
        if ws is None:
            ws = torch.full((max(1, ql.ql_paged_attention_bytes(self.fmt, q.shape[0], n, self.heads, max_new)),), 0xFF, dtype=torch.uint8, device=DEV)
        ql.ql_paged_attention(q, self.cache, self.fmt, ints(self.table) if table is None else table, ints(self.cu), ints(self.ctx), ints(self.len),
                              self.D ** -0.5 if scale is None else scale, y, ws, causal=causal, window=window, max_new=max_new)
        return y

    def check(self, y, scale=None, causal=True, window=0, rows=None):
        """y against the oracle, element by element.  With A = sum p |v| / sum p and n tokens seen:
        2^-11 |y|       y rounded to fp16 (2^-25 absolute below its normal range)
        2^-11 A         every p rounded to fp16 (p is relative to a bound at most 2^8 above ... the row's largest, so the absolute error of
                        one below the normal range, 2^-25, stays below n 2^-25 max|v| / sum p, and sum p >= 1)
        2 ds A          a score that is off by ds moves every p by that factor: D products added in fp32, each addition of the matrix
                        instruction within a whole step (2^-23) of sum |q k|; the multiplications by the scales and log2 e, the
                        subtraction of the maximum and the exponential, 2^-22 relative to |score| + 4 together, 32 2^-23 for the
                        logarithm of a value scale
        n 2^-23 A       n products added in fp32"""
        scale = self.D ** -0.5 if scale is None else scale
        y = y.cpu().numpy().astype(np.float64).reshape(-1, self.heads, self.D)
        for b in range(len(self.ctx)):
            lo, hi = self.cu[b], self.cu[b + 1]
            pick = np.arange(lo, hi) if rows is None else np.array([r for r in rows if lo <= r < hi], dtype=int)
            if not len(pick):
                continue
            pos = self.ctx[b] + pick - lo
            ref, a, spread, n = kv.attention(self.q.reshape(-1, self.heads, self.D)[pick], self.k[b], self.v[b], pos, scale, causal, window)
            ds = self.D * 2.0 ** -23 * spread + 2.0 ** -22 * (spread + 4) + 32 * 2.0 ** -23
            vmax = np.abs(self.v[b]).max() if len(self.v[b]) else 0
            n = n[:, None, None]
            tol = 2.0 ** -11 * np.abs(ref) + a * (2.0 ** -11 + 2 * ds[..., None] + n * 2.0 ** -23) + n * 2.0 ** -25 * vmax + 2.0 ** -24
            err = np.abs(y[pick] - ref)
            assert np.isfinite(y[pick]).all(), f"request {b}: not finite"
            assert (err <= tol).all(), f"request {b}: {(err / tol).max():.3g} times the tolerance at {np.unravel_index((err / tol).argmax(), err.shape)}"
