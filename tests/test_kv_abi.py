"""Refusals of the paged cache's calls: host-side checks, nothing is launched (no GPU)."""
import ctypes

import pytest
import torch

from paper_2512_23367_amd import binding as ql

NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
vp = ctypes.c_void_p


def fmt(**kw):
    return ql.QlKvFormat(**{**dict(heads=2, head_dim=128, page_size=64, pages=10, bits=8), **kw})


@pytest.mark.parametrize("bits,D,block", [(8, 64, 4096 + 512), (8, 128, 8192 + 512), (16, 64, 8192), (16, 256, 32768)])
def test_cache_bytes(bits, D, block):
    assert ql.ql_kv_cache_bytes(fmt(bits=bits, head_dim=D, page_size=128, pages=7)) == 7 * 2 * 4 * block


@pytest.mark.parametrize("bad,status", [(dict(bits=4), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(heads=0), SHAPE), (dict(page_size=48), SHAPE),
                                        (dict(page_size=16), SHAPE), (dict(page_size=2048), SHAPE), (dict(pages=0), SHAPE), (dict(pages=1 << 25), SHAPE)])
def test_formats_that_are_refused(bad, status):
    with pytest.raises(ql.QlError) as e:
        ql.ql_kv_cache_bytes(fmt(**bad))
    assert e.value.status == status
    f = fmt(**bad)
    lib = ql.lib()
    assert lib.ql_paged_attention(vp(4096), 256, 1, 2, vp(4096), ctypes.byref(f), vp(4096), 4, 4, vp(4096), vp(4096), vp(4096), 1, 1.0, 1, 0, 0, vp(1 << 20), 256,
                                  vp(4096), 1 << 20, None) == status
    assert lib.ql_kv_read(vp(4096), ctypes.byref(f), vp(4096), 1, vp(4096), 256, None, 0, None) == status


RESIZE = dict(old=vp(0x1000), want=vp(0x2000), requests=4, page=64, ring=vp(0x3000), pages=10, pool=vp(0x4000), pool_out=vp(0x4000), table=vp(0x5000), ld=8, columns=8,
              kv_len=vp(0x6000), cu=vp(0x7000), slots=vp(0x8000), positions=vp(0x9000), tokens=16)


@pytest.mark.parametrize("bad,status", [
    (dict(old=None), NULL), (dict(want=None), NULL), (dict(ring=None), NULL), (dict(pool=None), NULL), (dict(pool_out=None), NULL), (dict(table=None), NULL),
    (dict(kv_len=None), NULL), (dict(cu=None), NULL), (dict(slots=None), NULL), (dict(positions=None), NULL), (dict(requests=-1), SHAPE), (dict(tokens=-1), SHAPE),
    (dict(columns=0), SHAPE), (dict(ld=7), SHAPE), (dict(page=65), SHAPE), (dict(pages=0), SHAPE), (dict(requests=4097), UNSUPPORTED),
    (dict(requests=4096, columns=1 << 20, ld=1 << 20, page=1024), UNSUPPORTED), (dict(columns=1 << 26, ld=1 << 26), UNSUPPORTED), (dict(slots=vp(0x8002)), ALIGN),
    (dict(kv_len=vp(0x1008)), UNSUPPORTED), (dict(kv_len=vp(0x2000)), UNSUPPORTED), (dict(pool_out=vp(0x4008)), UNSUPPORTED)])
def test_resize_refusals(bad, status):
    assert ql.lib().ql_kv_resize(*{**RESIZE, **bad}.values(), None) == status


APPEND = dict(q=vp(0x100000), ldq=512, k=vp(0x200000), ldk=256, v=vp(0x300000), ldv=256, T=4, q_heads=4, cs=vp(0x400000), rot=128, most=100, pos=vp(0x500000),
              slots=vp(0x600000), q_out=vp(0x700000), ldo=512, cache=vp(0x800000))


@pytest.mark.parametrize("bad,status", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL), (dict(pos=None), NULL), (dict(q_out=None), NULL), (dict(cache=None), NULL),
    (dict(cache=vp(0x800010)), ALIGN), (dict(k=vp(0x200008)), ALIGN), (dict(ldk=255), ALIGN), (dict(ldk=128), ALIGN), (dict(ldv=(1 << 27) + 8), SHAPE),
    (dict(T=-1), SHAPE), (dict(q_heads=3), SHAPE), (dict(q_heads=0), SHAPE), (dict(rot=24), SHAPE), (dict(rot=0), SHAPE), (dict(rot=144), SHAPE), (dict(most=0), SHAPE),
    (dict(cs=None), UNSUPPORTED), (dict(cs=None, rot=0), UNSUPPORTED), (dict(cs=vp(0x400004)), ALIGN), (dict(q=None), SHAPE), (dict(q=None, q_heads=0), SHAPE),
    (dict(q_out=vp(0x100010)), UNSUPPORTED), (dict(q_out=vp(0x100000), ldo=520), UNSUPPORTED), (dict(q_out=vp(0x200000)), UNSUPPORTED), (dict(q_out=vp(0x300100)), UNSUPPORTED)])
def test_append_refusals(bad, status):
    assert ql.lib().ql_kv_append(*{**APPEND, **bad}.values(), ctypes.byref(fmt()), None) == status


def test_append_and_read_of_nothing_are_no_ops():
    f = ctypes.byref(fmt())
    assert ql.lib().ql_kv_append(None, 0, None, 0, None, 0, 0, 0, None, 0, 0, None, None, None, 0, None, f, None) == 0
    assert ql.lib().ql_kv_read(None, f, None, 0, None, 0, None, 0, None) == 0
    assert ql.lib().ql_kv_read(vp(0x1000), f, vp(0x1000), 3, None, 0, None, 0, None) == NULL


ATTEND = dict(q=vp(0x100000), ldq=512, T=4, q_heads=4, cache=vp(0x200000), fmt=None, table=vp(0x300000), ld=8, columns=8, cu=vp(0x400000), ctx=vp(0x500000),
              len=vp(0x600000), requests=2, scale=1.0, causal=1, window=0, max_new=0, y=vp(0x700000), ldy=512, ws=vp(0x800000), wsb=1 << 40)


@pytest.mark.parametrize("bad,status", [
    (dict(q=None), NULL), (dict(cache=None), NULL), (dict(table=None), NULL), (dict(cu=None), NULL), (dict(ctx=None), NULL), (dict(len=None), NULL), (dict(y=None), NULL),
    (dict(T=-1), SHAPE), (dict(requests=-1), SHAPE), (dict(max_new=-1), SHAPE), (dict(q_heads=0), SHAPE), (dict(q_heads=5), SHAPE), (dict(columns=0), SHAPE), (dict(ld=7), SHAPE),
    (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(causal=2), SHAPE), (dict(window=-1), SHAPE), (dict(causal=0, window=5), SHAPE),
    (dict(columns=1 << 26, ld=1 << 26), SHAPE), (dict(requests=65537), UNSUPPORTED), (dict(T=1 << 30), UNSUPPORTED), (dict(q=vp(0x100008)), ALIGN), (dict(ldy=500), ALIGN),
    (dict(cache=vp(0x200010)), ALIGN), (dict(ws=vp(0x800010)), ALIGN), (dict(table=vp(0x300002)), ALIGN), (dict(y=vp(0x100010)), UNSUPPORTED),
    (dict(y=vp(0x100000), ldy=520), UNSUPPORTED)])
def test_attention_refusals(bad, status):
    f = fmt()
    args = {**ATTEND, "fmt": ctypes.byref(f), **bad}
    assert ql.lib().ql_paged_attention(*args.values(), None) == status


def test_attention_of_nothing_is_a_no_op():
    f = fmt()
    for none in (dict(T=0), dict(requests=0)):
        args = {**ATTEND, "fmt": ctypes.byref(f), **none, "q": None, "cache": None, "y": None, "ws": None, "wsb": 0}
        assert ql.lib().ql_paged_attention(*args.values(), None) == 0


def test_a_short_workspace_is_refused():
    f = fmt(heads=1)
    need = ql.ql_paged_attention_bytes(f, 1, 1, 4, 1)
    if not need:
        pytest.skip("no workspace at this size")
    args = {**ATTEND, "fmt": ctypes.byref(f), "T": 1, "requests": 1, "max_new": 1, "wsb": need - 1}
    assert ql.lib().ql_paged_attention(*args.values(), None) == WORKSPACE
    assert ql.lib().ql_paged_attention(*{**args, "ws": None, "wsb": 0}.values(), None) == NULL


def test_binding_checks_tensors_on_the_host():
    f = fmt()
    half, i32 = torch.zeros((4, 256), dtype=torch.float16), torch.zeros(8, dtype=torch.int32)
    cache = torch.zeros(ql.ql_kv_cache_bytes(f), dtype=torch.uint8)
    for call in (lambda: ql.ql_kv_resize(64, i32, i32, i32, i32, i32, i32.view(2, 4), i32, i32, i32, i32),
                 lambda: ql.ql_kv_append(None, half, half, None, None, i32, None, cache, f),
                 lambda: ql.ql_kv_read(cache, f, i32, half, half),
                 lambda: ql.ql_paged_attention(half, cache, f, i32.view(2, 4), i32, i32, i32, 1.0, half)):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


@pytest.mark.parametrize("bad", [dict(cu=vp(0x100C)), dict(cu=vp(0x2000 - 16)), dict(slots=vp(0x2008)), dict(positions=vp(0x1000 - 60))])
def test_resize_refuses_outputs_over_the_lengths(bad):
    assert ql.lib().ql_kv_resize(*{**RESIZE, **bad}.values(), None) == UNSUPPORTED
