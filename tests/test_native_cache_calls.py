"""Native argument marshalling of the paged cache's calls (csrc/pycall.cpp) against the Python of binding.py: the same calls, the same results, and
whatever is wrong is handed back to binding.py, which says so as without it."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2512_23367_amd import binding as ql

D, HEADS, Q_HEADS, T, REQUESTS, COLUMNS, PAGES = 64, 2, 4, 3, 3, 4, 9
PYTHON = {"kv_resize": "ql_kv_resize", "kv_append": "ql_kv_append", "kv_read": "ql_kv_read", "paged_attention": "ql_paged_attention"}
BOUND = ("ql_kv_cache_bytes",) + tuple(PYTHON.values())


def _outcome(f):
    try:
        return ("returned", f())
    except Exception as e:                                            # noqa: BLE001  (any exception is an outcome)
        return (type(e).__name__, str(e))


def _format(**kw):
    return ql.QlKvFormat(**{**dict(heads=HEADS, head_dim=D, page_size=32, pages=PAGES, bits=8), **kw})


def good_arguments(device="cuda:0"):
    def half(*shape):
        return torch.zeros(shape, dtype=torch.float16, device=device)

    def ints(*values):
        return torch.tensor(values, dtype=torch.int32, device=device)
    fmt = _format()
    cache = torch.zeros(ql.ql_kv_cache_bytes(fmt), dtype=torch.uint8, device=device)
    table = torch.arange(REQUESTS * COLUMNS, dtype=torch.int32, device=device).view(REQUESTS, COLUMNS) % PAGES
    qkv = half(T, (Q_HEADS + 2 * HEADS) * D)
    q, k, v = qkv[:, :Q_HEADS * D], qkv[:, Q_HEADS * D:(Q_HEADS + HEADS) * D], qkv[:, (Q_HEADS + HEADS) * D:]
    cos_sin = torch.zeros((50, D), dtype=torch.float32, device=device)
    ws = torch.zeros(ql.ql_paged_attention_bytes(fmt, T, REQUESTS, Q_HEADS, 0), dtype=torch.uint8, device=device)
    return {
        "kv_resize": [32, ints(0, 0, 0), ints(1, 1, 1), torch.arange(PAGES, dtype=torch.int32, device=device), ints(0, PAGES, 0, 0), ints(0, 0, 0, 0), table,
                      ints(0, 0, 0), ints(0, 0, 0, 0), ints(0, 0, 0, 0, 0), ints(0, 0, 0, 0, 0)],
        "kv_append": [q, k, v, cos_sin, ints(0, 1, 2), ints(0, 40, 70), half(T, Q_HEADS * D), cache, fmt],
        "kv_read": [cache, fmt, ints(0, 40, 70), half(T, HEADS * D), half(T, HEADS * D)],
        "paged_attention": [half(T, Q_HEADS * D), cache, fmt, table, ints(0, 1, 2, 3), ints(0, 5, 9), ints(1, 6, 10), 0.125, half(T, Q_HEADS * D), ws, True, 0, 1],
    }


def _strided(t):
    return torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device=t.device)[..., ::2]


HOST = {"host": lambda t: t.cpu()}
INTS = {"int64": lambda t: t.long(), "strided": _strided, **HOST}
KINDS = {
    "rows": {"fp32": lambda t: t.float(), "flat": lambda t: t.reshape(-1), "strided": _strided, "half a head": lambda t: t[:, :-D // 2], **HOST},
    "given": {"a head short": lambda t: t[:, :-D], "a row short": lambda t: t[:-1]},     # (what another argument fixes the size of)
    "None": {"None": lambda t: None},
    "ints": INTS,
    "short": {"one short": lambda t: t[:-1]},
    "table": {"int64": lambda t: t.long(), "flat": lambda t: t.reshape(-1), "strided": _strided, "a request short": lambda t: t[:-1], **HOST},
    "cache": {"a byte short": lambda t: t[:-1], "strided": _strided, **HOST},
    "cos_sin": {"fp64": lambda t: t.double(), "flat": lambda t: t.reshape(-1), "strided": _strided, **HOST},
    "format": {"another type": lambda f: (f.heads, f.head_dim, f.page_size, f.pages, f.bits), "None": lambda f: None, "other heads": lambda f: _format(heads=HEADS + 1),
               "no channels": lambda f: _format(head_dim=0), "unknown bits": lambda f: _format(bits=5), "more pages": lambda f: _format(pages=PAGES + 1)},
    "number": {"float": float, "text": str},
    "scale": {"text": lambda s: "scale", "None": lambda s: None},
    "host": HOST,
}
WRONG = [(f, i, what, make) for f, i, kinds in [
    ("kv_resize", 0, "number"), ("kv_resize", 1, "ints"), ("kv_resize", 2, "ints short"), ("kv_resize", 3, "ints"), ("kv_resize", 4, "ints short"), ("kv_resize", 5, "ints short"),
    ("kv_resize", 6, "table"), ("kv_resize", 7, "ints short"), ("kv_resize", 8, "ints short"), ("kv_resize", 9, "ints"), ("kv_resize", 10, "ints"),
    ("kv_append", 0, "rows"), ("kv_append", 1, "rows given"), ("kv_append", 2, "rows given"), ("kv_append", 3, "cos_sin None"), ("kv_append", 4, "ints short"),
    ("kv_append", 5, "ints short"), ("kv_append", 6, "rows given None"), ("kv_append", 7, "cache"), ("kv_append", 8, "format"),
    ("kv_read", 0, "cache"), ("kv_read", 1, "format"), ("kv_read", 2, "ints short"), ("kv_read", 3, "rows given"), ("kv_read", 4, "rows given"),
    ("paged_attention", 0, "rows given"), ("paged_attention", 1, "cache"), ("paged_attention", 2, "format"), ("paged_attention", 3, "table"), ("paged_attention", 4, "ints short"),
    ("paged_attention", 5, "ints short None"), ("paged_attention", 6, "ints"), ("paged_attention", 7, "scale"), ("paged_attention", 8, "rows given"), ("paged_attention", 9, "host"),
    ("paged_attention", 11, "number"), ("paged_attention", 12, "number")]
    for kind in kinds.split() for what, make in KINDS[kind].items()]
# what the library itself refuses, not the native checks
LIBRARY = {("kv_append", 3, "None"), ("paged_attention", 5, "None")}


def bind_stand_ins(module):
    """Binds the cache's native calls to functions that note their name and return QL_OK (cache sizes: the library's).  Returns the notes, and what
    has to be kept alive while it is bound."""
    lib, called, kept, addresses = ql.lib(), [], [], []
    for name in BOUND:
        f = getattr(lib, name)
        if not name.endswith("_bytes"):
            f = ctypes.CFUNCTYPE(ctypes.c_int, *f.argtypes)(lambda *a, name=name: called.append(name) or 0)
            kept.append(f)
        addresses.append(ctypes.cast(f, ctypes.c_void_p).value)
    module.bind_cache(tuple(addresses))
    return called, kept


def test_wrong_calls_are_reported_as_before_on_the_host(monkeypatch):
    ql.lib()
    assert ql._native is not None
    for f, args in good_arguments("cpu").items():
        call = getattr(ql, PYTHON[f])
        with_native = _outcome(lambda: call(*args))
        with monkeypatch.context() as m:
            m.setattr(ql, "_native", None)
            assert with_native == _outcome(lambda: call(*args)) and with_native[0] != "returned", f


@pytest.mark.gpu
def test_no_wrong_argument_passes_the_native_checks(monkeypatch):
    ql.lib()
    stream = lambda: 0  # noqa: E731
    try:
        called, kept = bind_stand_ins(ql._native)
        good = good_arguments()
        for f, args in good.items():
            assert getattr(ql._native, f)(*args, stream) == 0 and called == [PYTHON[f]], f
            called.clear()
        let_through = []
        for f, i, what, make in WRONG:
            args = list(good[f])
            args[i] = make(args[i])
            if (f, i, what) not in LIBRARY and (getattr(ql._native, f)(*args, stream) is not None or called):
                let_through.append((f, i, what))
            called.clear()
        assert let_through == []
        for f, args in good.items():                      # one argument more or less
            assert getattr(ql._native, f)(*args) is None and getattr(ql._native, f)(*args, stream, stream) is None and called == []
    finally:
        ql._bind_native(ql.lib())
    for f, i, what, make in WRONG:                        # and binding.py or the library says what is wrong with it, as without the native code
        args = list(good_arguments()[f])
        args[i] = make(args[i])
        call = getattr(ql, PYTHON[f])
        with_native = _outcome(lambda: call(*args))
        with monkeypatch.context() as m:
            m.setattr(ql, "_native", None)
            assert with_native == _outcome(lambda: call(*args)) and with_native[0] != "returned", (f, i, what)


@pytest.mark.gpu
def test_functions_that_are_not_bound_are_not_called():
    """A module whose cache functions have no addresses hands every cache call back."""
    ql.lib()
    try:
        ql._native.bind_cache((0,) * len(BOUND))
        for f, args in good_arguments().items():
            assert getattr(ql._native, f)(*args, lambda: 0) is None
    finally:
        ql._bind_native(ql.lib())


@pytest.mark.gpu
@pytest.mark.parametrize("bits,head_dim,new", [(8, 64, [1, 0, 1]), (16, 128, [3, 40, 1]), (8, 256, [1, 0, 0])])
def test_the_same_results_with_and_without_the_native_code(bits, head_dim, new, monkeypatch):
    """A step through all four calls: column ranges of one buffer as inputs, a single row, outputs over q, optional arguments left out."""
    import kv_util as U
    ql.lib()
    assert ql._native is not None
    heads, q_heads, page, ctx = 2, 6, 32, [70, 31, 0]
    n, t = len(new), sum(new)

    def step():
        rng = np.random.default_rng(head_dim)
        fmt = ql.QlKvFormat(heads=heads, head_dim=head_dim, page_size=page, pages=20, bits=bits)
        ring, pool, table = U.ints(rng.permutation(20)), U.ints([0, 20, 0, 0]), U.ints(np.full((n, 5), -1))
        before, cache = U.ints([0] * n), torch.zeros(ql.ql_kv_cache_bytes(fmt), dtype=torch.uint8, device=U.DEV)
        cos_sin = U.dev(rng.standard_normal((200, head_dim)).astype(np.float32))
        out = []
        for want in (ctx, [a + b for a, b in zip(ctx, new)]):
            room = sum(w - o for w, o in zip(want, before.tolist()))
            kv_len, cu, slots, positions = U.ints([0] * n), U.ints([0] * (n + 1)), U.ints([-1] * room), U.ints([0] * room)
            ql.ql_kv_resize(page, before, U.ints(want), ring, pool, pool, table, kv_len, cu, slots, positions)
            qkv = U.dev(rng.standard_normal((room, (q_heads + 2 * heads) * head_dim)).astype(np.float16))
            q, k, v = (qkv[:, a * head_dim:b * head_dim] for a, b in ((0, q_heads), (q_heads, q_heads + heads), (q_heads + heads, q_heads + 2 * heads)))
            turned = torch.empty((room, q_heads * head_dim), dtype=torch.float16, device=U.DEV)
            ql.ql_kv_append(q, k, v, cos_sin, positions, slots, turned, cache, fmt)
            ql.ql_kv_append(None, k, v, cos_sin, positions, slots, None, cache, fmt)
            ql.ql_kv_append(q, k, v, cos_sin, positions, slots, q, cache, fmt)
            kb, vb, only = (torch.empty((room, heads * head_dim), dtype=torch.float16, device=U.DEV) for _ in range(3))
            ql.ql_kv_read(cache, fmt, slots, kb, vb)
            ql.ql_kv_read(cache, fmt, slots, None, only)
            ws = torch.empty(max(1, ql.ql_paged_attention_bytes(fmt, room, n, q_heads)), dtype=torch.uint8, device=U.DEV)
            for kw in (dict(), dict(causal=False), dict(window=9), dict(max_new=max(new)), dict(ws=ws, window=40)):
                y = torch.empty_like(turned)
                ql.ql_paged_attention(q, cache, fmt, table, cu, before if kw.get("causal", True) else None, kv_len, head_dim ** -0.5, y, **{"ws": ws, **kw})
                out.append(y)
            y = torch.empty_like(turned)
            ql.ql_paged_attention(q, cache, fmt, table, cu, before, kv_len, 1, y, ws)                   # (a whole number as scale)
            out += [y, ring.clone(), pool.clone(), table.clone(), kv_len, cu, slots, positions, turned, q.contiguous(), kb, vb, only, cache.clone()]
            before = kv_len
        torch.cuda.synchronize()
        return out

    made = []
    real = ql._done
    monkeypatch.setattr(ql, "_done", lambda status: made.append(status) or real(status))
    native = step()
    assert made.count(0) >= 2 * 11 and t > 0               # (made by the native code, all but those with a whole number as scale)
    monkeypatch.setattr(ql, "_native", None)
    python = step()
    assert len(native) == len(python) and all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(native, python))
