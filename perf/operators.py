"""The paged KV cache and the attention that reads it, as cases that can be timed.

A case is a dict of plain values.  `op` names the operator, the other entries its sizes:
  resize  the bookkeeping of one serving step: request lengths old -> wanted, pages from and to the ring of free pages,
          block table, slot and position of every new token (ql_kv_resize)
  append  rotary embedding of the new tokens' queries and keys, keys and values into the cache (ql_kv_append), and the
          rows of their slots read back (ql_kv_read)
  attend  attention of the new tokens over the cache (ql_paged_attention)
Requests have lengths of their own, drawn from the ranges in the case by its entry `lengths`.

The cache is made of blocks: 32 tokens of one key/value head, ordered [page][head][block of the page].  In a block
  16 bits  K  [D/16][2][32 tokens][8]          channel 16 a + 8 b + j at [a][b][token][j]
           V  [D/32][2][2][32 channels][8]     token 16 s + 8 (j / 4) + 4 h + j % 4 at [channel / 32][s][h][channel % 32][j]
  8 bits   K  [D/32][2][32 tokens][16]         channel 32 a + 16 b + j; codes stored plus 128
           V  [D/32][2][32 channels][16]       token 16 (j / 8) + 8 (j % 8 / 4) + 4 h + j % 4 at [channel / 32][h][channel % 32][j]
           then fp32 [4][32 tokens]: scale of K, scale of V, log2 and reciprocal of the scale of V
"""
import math
import random

import torch

own = False
DEV = "cuda"


def listed():
    return [
        # A decode step of 64 requests: one token each, a page now and then.
        dict(name="resize_step_b64", op="resize", requests=64, old_low=100, old_high=8000, new_low=1, new_high=1, ended=0.0, page=64, columns=128, lengths=1),
        # A step of a busy server: prompts come in, requests end, 1024 of them in the table.
        dict(name="resize_mixed_b1024", op="resize", requests=1024, old_low=0, old_high=4000, new_low=0, new_high=70, ended=0.25, page=32, columns=130, lengths=2),
        # A decode step's tokens, shared key/value heads, int8 cache.
        dict(name="append_step_w8_t32", op="append", tokens=32, requests=32, heads=32, kv_heads=8, head_dim=128, rotary=128, bits=8, page=64, lengths=3),
        # The prompt of the 7B-class layer (4096 tokens, 32 heads) into an fp16 cache.
        dict(name="append_prompt_f16_t4096", op="append", tokens=4096, requests=1, heads=32, kv_heads=32, head_dim=128, rotary=128, bits=16, page=64, lengths=4),
        # Several long prompts of odd lengths in one batch, int8.
        dict(name="append_prompts_w8_t16001", op="append", tokens=16001, requests=7, heads=32, kv_heads=8, head_dim=128, rotary=128, bits=8, page=128, lengths=5),
        # The smallest call: one token of one short conversation, 12 heads of the 1B-class layer (d = 1536).
        dict(name="attend_token_f16_b1", op="attend", requests=1, ctx_low=300, ctx_high=300, new_low=1, new_high=1, heads=12, kv_heads=12, head_dim=128, bits=16, page=64, causal=True, window=0, lengths=6),
        # A decode step of 32 requests of different lengths, int8 cache.
        dict(name="attend_step_w8_b32", op="attend", requests=32, ctx_low=200, ctx_high=4096, new_low=1, new_high=1, heads=32, kv_heads=8, head_dim=128, bits=8, page=64, causal=True, window=0, lengths=7),
        # A decode step of a few very long conversations.
        dict(name="attend_long_w8_b4", op="attend", requests=4, ctx_low=60000, ctx_high=131071, new_low=1, new_high=1, heads=32, kv_heads=8, head_dim=128, bits=8, page=128, causal=True, window=0, lengths=8),
        # Drafted tokens to be verified: five new tokens per request.
        dict(name="attend_drafts_f16_b16", op="attend", requests=16, ctx_low=1000, ctx_high=9000, new_low=5, new_high=5, heads=64, kv_heads=8, head_dim=128, bits=16, page=32, causal=True, window=0, lengths=9),
        # Chunks of two long prompts over what is in the cache already.
        dict(name="attend_chunk_w8_b2", op="attend", requests=2, ctx_low=9000, ctx_high=17000, new_low=1000, new_high=1024, heads=32, kv_heads=8, head_dim=128, bits=8, page=64, causal=True, window=0, lengths=10),
        # A ragged batch of short prompts, small heads, sliding window.
        dict(name="attend_prompts_d64_b6", op="attend", requests=6, ctx_low=0, ctx_high=0, new_low=700, new_high=1900, heads=24, kv_heads=4, head_dim=64, bits=16, page=32, causal=True, window=1024, lengths=11),
        # A long prompt at once: the largest.
        dict(name="attend_prompt_f16_m16384", op="attend", requests=1, ctx_low=0, ctx_high=0, new_low=16384, new_high=16384, heads=32, kv_heads=8, head_dim=128, bits=16, page=64, causal=True, window=0, lengths=12),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    lengths = rng.randrange(1 << 20)
    page = rng.choice((32, 64, 128, 256))
    what = rng.random()
    if what < 0.2:
        return dict(op="resize", requests=_log_uniform(rng, 1, 2048), old_low=0, old_high=_log_uniform(rng, 50, 4000), new_low=0,
                    new_high=_log_uniform(rng, 1, 60), ended=rng.choice((0.0, 0.1, 0.5)), page=page, columns=4200 // page, lengths=lengths)
    kv_heads = rng.choice((1, 2, 4, 8, 12))
    heads = kv_heads * rng.choice((1, 2, 3, 4, 6, 8))
    bits, head_dim = rng.choice((8, 16)), rng.choice((64, 128, 128, 256))
    if what < 0.4:
        tokens = _log_uniform(rng, 1, 12000)
        return dict(op="append", tokens=tokens, requests=min(tokens, _log_uniform(rng, 1, 64)), heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                    rotary=rng.choice((head_dim, head_dim // 2)), bits=bits, page=page, lengths=lengths)
    if what < 0.7:                                    # decode steps and drafts
        requests, new = _log_uniform(rng, 1, 128), rng.choice((1, 1, 1, 4, 7))
        most = int(min(65536, 4.0e8 / (requests * kv_heads * head_dim)))
        ctx = _log_uniform(rng, 16, max(17, most))
    else:                                             # prompts and chunks of prompts
        requests, new = _log_uniform(rng, 1, 8), _log_uniform(rng, 16, 6000)
        scores = min(6.0e9, 2.0e12 / (4 * head_dim))
        new = min(new, int(math.sqrt(scores / (requests * heads))))
        most = int(scores / (requests * heads * new)) - new
        ctx = rng.choice((0, _log_uniform(rng, 16, min(30000, most)))) if most > 16 else 0
    causal = rng.random() < 0.85
    return dict(op="attend", requests=requests, ctx_low=ctx // 4, ctx_high=ctx, new_low=max(1, new // 2) if new > 8 else new, new_high=new, heads=heads,
                kv_heads=kv_heads, head_dim=head_dim, bits=bits, page=page, causal=causal, window=rng.choice((0, 0, 0, 100, 1500)) if causal else 0, lengths=lengths)


# ---- sizes -------------------------------------------------------------------------------------------------------

def _lengths(case):
    """Host lists of a case: what every request has and gets."""
    r = random.Random(case["lengths"])
    n = case["requests"]
    if case["op"] == "resize":
        old = [r.randint(case["old_low"], case["old_high"]) for _ in range(n)]
        new = [r.randint(case["new_low"], case["new_high"]) for _ in range(n)]
        want = [r.randint(0, o) if r.random() < case["ended"] else o + k for o, k in zip(old, new)]
        return old, want
    if case["op"] == "append":
        cuts = sorted(r.randint(0, case["tokens"]) for _ in range(n - 1))
        return [r.randint(0, 2000) for _ in range(n)], [b - a for a, b in zip([0] + cuts, cuts + [case["tokens"]])]
    ctx = [r.randint(case["ctx_low"], case["ctx_high"]) for _ in range(n)]
    ctx[r.randrange(n)] = case["ctx_high"]
    return ctx, [r.randint(case["new_low"], case["new_high"]) for _ in range(n)]


def _block_bytes(case):
    return 64 * case["head_dim"] * case["bits"] // 8 + (512 if case["bits"] == 8 else 0)


def _pages(length, page):
    return (length + page - 1) // page


def work(case):
    first, second = _lengths(case)
    if case["op"] == "resize":
        cap = case["columns"] * case["page"]
        tokens = sum(max(0, w - o) for o, w in zip(first, second))
        moved = sum(abs(_pages(min(w, cap), case["page"]) - _pages(o, case["page"])) for o, w in zip(first, second))
        return {"bytes": 16 * case["requests"] + 8 * tokens + 8 * moved, "flops": 0}
    per_kv_head = 2 * case["head_dim"] * case["bits"] // 8 + (8 if case["bits"] == 8 else 0)
    if case["op"] == "append":
        row = 2 * case["head_dim"] * (case["heads"] + 2 * case["kv_heads"])
        out = 2 * case["head_dim"] * case["heads"] + case["kv_heads"] * per_kv_head
        back = case["kv_heads"] * (per_kv_head + 4 * case["head_dim"])
        return {"bytes": case["tokens"] * (row + 4 * case["rotary"] + 8 + out + back), "flops": case["tokens"] * case["head_dim"] * (3 * case["heads"] + 6 * case["kv_heads"])}
    seen = reads = 0
    for c, n in zip(first, second):
        kv, w = c + n, case["window"]
        low = max(0, c - w + 1) if w and case["causal"] else 0
        reads += kv - low
        if not case["causal"]:
            seen += n * kv
        else:                                         # query i sees min(c + i + 1, window) tokens
            full = n * c + n * (n + 1) // 2
            over = max(0, kv - w) if w else 0         # the last ones see fewer
            start = max(c + 1, w + 1) - w if w else 0
            seen += full - ((start + over) * (over - start + 1) // 2 if w and over >= start else 0)
    tokens = sum(second)
    return {"bytes": 4 * tokens * case["heads"] * case["head_dim"] + reads * case["kv_heads"] * per_kv_head,
            "flops": 4 * case["head_dim"] * case["heads"] * seen}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _keys(g, rows, kv_heads, head_dim):
    """Keys: a few channels of every head are large, as they are in the layers of language models."""
    gain = 0.7 + 3.0 * (torch.rand((kv_heads, head_dim), generator=g, device=DEV) < 0.03)
    return _normal(g, rows, kv_heads, head_dim) * gain


def _new_cache(case, pages):
    return torch.zeros((pages, case["kv_heads"], case["page"] // 32, _block_bytes(case)), dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    first, second = _lengths(case)
    page, n = case["page"], case["requests"]
    state = dict(case=case)
    if case["op"] == "resize":
        held = [_pages(o, page) for o in first]
        most = max(0, sum(max(0, w - o) for o, w in zip(first, second)))
        grown = sum(_pages(w, page) for w in second)
        total = sum(held) + grown + 8
        ids = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        table = torch.full((n, case["columns"]), -1, dtype=torch.int32, device=DEV)
        at = torch.arange(case["columns"], device=DEV)
        count = torch.tensor(held, device=DEV)
        begin = torch.cumsum(count, 0) - count
        mine = at[None] < count[:, None]
        table[mine] = ids[(begin[:, None] + at[None])[mine]]
        free = total - sum(held)
        head = int(torch.randint(0, total, (1,), generator=g, device=DEV))
        ring = torch.full((total,), -1, dtype=torch.int32, device=DEV)
        ring[(head + torch.arange(free, device=DEV)) % total] = ids[sum(held):]
        none = lambda k: torch.full((k,), -1, dtype=torch.int32, device=DEV)  # noqa: E731
        state.update(old=_ints(first), want=_ints(second), ring=ring, pool=_ints([head, free, 0, 0]), pool_out=torch.zeros(4, dtype=torch.int32, device=DEV),
                     table=table, kv_len=none(n), cu=none(n + 1), slots=none(most + 5), positions=none(most + 5), pages=total)
        return state
    heads, kv_heads, head_dim = case["heads"], case["kv_heads"], case["head_dim"]
    lengths = [a + b for a, b in zip(first, second)]
    held = [_pages(k, page) for k in lengths]
    pages, columns, tokens = sum(held) + 3, max(held) + 1, sum(second)
    ids = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    at = torch.arange(columns, device=DEV)
    count = torch.tensor(held, device=DEV)
    mine = at[None] < count[:, None]
    table = torch.full((n, columns), -1, dtype=torch.int32, device=DEV)
    table[mine] = ids[((torch.cumsum(count, 0) - count)[:, None] + at[None])[mine]]
    cu = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
    cu[1:] = torch.cumsum(torch.tensor(second, device=DEV), 0)
    if case["op"] == "append":
        whose = torch.repeat_interleave(torch.arange(n, device=DEV), torch.tensor(second, device=DEV))
        position = torch.arange(tokens, device=DEV) - cu[whose] + torch.tensor(first, device=DEV)[whose]
        slots = table[whose, position // page].long() * page + position % page
        most = max(lengths)
        half = case["rotary"] // 2
        angle = torch.arange(most, device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
        qkv = torch.empty((tokens, (heads + 2 * kv_heads) * head_dim), dtype=torch.float16, device=DEV)   # the fused projection's output
        qkv[:, :heads * head_dim] = _normal(g, tokens, heads * head_dim)
        qkv[:, heads * head_dim:(heads + kv_heads) * head_dim] = _keys(g, tokens, kv_heads, head_dim).view(tokens, -1)
        qkv[:, (heads + kv_heads) * head_dim:] = 0.5 * _normal(g, tokens, kv_heads * head_dim)
        rows = lambda h: torch.empty((tokens, h * head_dim), dtype=torch.float16, device=DEV)  # noqa: E731
        state.update(q=qkv[:, :heads * head_dim], k=qkv[:, heads * head_dim:(heads + kv_heads) * head_dim], v=qkv[:, (heads + kv_heads) * head_dim:],
                     cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(), positions=position.int(), slots=slots.int(), cache=_new_cache(case, pages),
                     q_out=rows(heads), k_back=rows(kv_heads), v_back=rows(kv_heads), pages=pages)
        return state
    cache = _new_cache(case, pages)
    step = max(1, (1 << 28) // (kv_heads * page * head_dim))
    for begin in range(0, pages, step):               # keys and values of some pages at a time: the fp32 draws are large
        some = min(step, pages - begin)
        k = _keys(g, some * page, kv_heads, head_dim)
        v = 0.5 * _normal(g, some * page, kv_heads, head_dim)
        _store(case, cache[begin:begin + some], torch.arange(some * page, device=DEV), k, v)
    q = (1.5 * _normal(g, tokens, heads * head_dim)).half()
    state.update(q=q, cache=cache, table=table, cu=cu.int(), ctx=_ints(first), kv_len=_ints(lengths), y=torch.empty_like(q), pages=pages, longest=max(lengths), most=max(second))
    return state


# ---- the framework's calls ---------------------------------------------------------------------------------------

def _ql():
    from paper_2512_23367_amd import binding
    return binding


def _format(s):
    c = s["case"]
    return _ql().QlKvFormat(heads=c["kv_heads"], head_dim=c["head_dim"], page_size=c["page"], pages=s["pages"], bits=c["bits"])


def _own(s):
    c, ql = s["case"], _ql()
    if c["op"] == "resize":
        ql.ql_kv_resize(c["page"], s["old"], s["want"], s["ring"], s["pool"], s["pool_out"], s["table"], s["kv_len"], s["cu"], s["slots"], s["positions"])
        return _resized(s)
    fmt = _format(s)
    if c["op"] == "append":
        ql.ql_kv_append(s["q"], s["k"], s["v"], s["cos_sin"], s["positions"], s["slots"], s["q_out"], s["cache"], fmt)
        ql.ql_kv_read(s["cache"], fmt, s["slots"], s["k_back"], s["v_back"])
        return s["q_out"], s["k_back"], s["v_back"]
    if "ws" not in s:                                 # once: a program keeps its workspace
        s["ws"] = torch.empty(ql.ql_paged_attention_bytes(fmt, s["q"].shape[0], c["requests"], c["heads"], s["most"]), dtype=torch.uint8, device=DEV)
    ql.ql_paged_attention(s["q"], s["cache"], fmt, s["table"], s["cu"], s["ctx"], s["kv_len"], c["head_dim"] ** -0.5, s["y"], s["ws"],
                          causal=c["causal"], window=c["window"], max_new=s["most"])
    return s["y"]


def _resized(s):
    return {k: s[k] for k in ("ring", "pool_out", "table", "kv_len", "cu", "slots", "positions")}


def run(state):
    if own:
        return _own(state)
    return {"resize": _plain_resize, "append": _plain_append, "attend": _plain_attend}[state["case"]["op"]](state)


# ---- plain forms -------------------------------------------------------------------------------------------------

def _plain_resize(s):
    page, ring, table = s["case"]["page"], s["ring"], s["table"]
    n, columns = table.shape
    cap, total, rows = columns * page, ring.numel(), s["slots"].numel()
    old, want = s["old"].long().clamp(0, cap), s["want"].long().clamp(min=0)
    head, free = s["pool"][0].long(), s["pool"][1].long()
    s["cu"].zero_()
    s["cu"][1:] = torch.cumsum((want - old).clamp(min=0), 0).clamp(max=rows)
    cu = s["cu"].long()
    new = cu[1:] - cu[:-1]
    target = torch.where(want < old, want, torch.minimum(old + new, torch.full_like(old, cap)))
    has, needs = (old + page - 1) // page, (target + page - 1) // page
    take, give = (needs - has).clamp(min=0), (has - needs).clamp(min=0)
    taken_before, given_before = torch.cumsum(take, 0) - take, torch.cumsum(give, 0) - give
    got = torch.minimum((free - taken_before).clamp(min=0), take)
    kv = torch.minimum(target, torch.where(want < old, target, (has + got) * page))
    at = torch.arange(columns, device=DEV)[None]
    to = torch.where((at >= needs[:, None]) & (at < has[:, None]), (head + free + given_before[:, None] + at - needs[:, None]) % total, total)
    longer = torch.cat([ring, ring[:1]])
    longer.scatter_(0, to.reshape(-1), table.reshape(-1))
    fresh = ring.long()[(head + taken_before[:, None] + at - has[:, None]) % total].int()
    table.copy_(torch.where((at >= has[:, None]) & (at < (has + got)[:, None]), fresh, table))
    ring.copy_(longer[:total])
    s["kv_len"].copy_(kv)
    t = torch.arange(rows, device=DEV)
    whose = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=n - 1)
    position = old[whose] + t - cu[whose]
    own_page = table[whose, (position // page).clamp(max=columns - 1)].long()
    slot = torch.where((position < kv[whose]) & (own_page >= 0) & (own_page < total), own_page * page + position % page, -1)
    s["slots"].copy_(torch.where(t < cu[-1], slot, s["slots"]))
    s["positions"].copy_(torch.where(t < cu[-1], position, s["positions"]))
    used = got.sum()
    s["pool_out"].copy_(torch.stack([(head + used) % total, free - used + give.sum(), torch.where(want < old, 0, old + new - kv).sum(), torch.zeros_like(head)]))
    return _resized(s)


def _places(case, slots):
    """Page, block of the page and token of the block of every slot, and the three parts that a token of V is stored by."""
    slots = slots.long()
    page, rest = slots // case["page"], slots % case["page"]
    r = rest % 32
    return page, rest // 32, r, r // 16, r % 16 // 8, r % 8 // 4, r % 4


def _views(case, cache):
    """K, V and the scales of a cache, as the strided arrays of the layout above."""
    d, e = case["head_dim"], 32 * case["head_dim"] * case["bits"] // 8
    k, v, scales = cache[..., :e], cache[..., e:2 * e], cache[..., 2 * e:]
    if case["bits"] == 16:
        return k.view(torch.float16).unflatten(-1, (d // 16, 2, 32, 8)), v.view(torch.float16).unflatten(-1, (d // 32, 2, 2, 32, 2, 4)), None
    return k.unflatten(-1, (d // 32, 2, 32, 16)), v.unflatten(-1, (d // 32, 2, 32, 2, 2, 4)), scales.view(torch.float32).unflatten(-1, (4, 32))


def _quantize(x):
    most = x.abs().amax(-1, keepdim=True)
    none = most < 2.0 ** -100
    codes = torch.round(x * (127.0 / torch.where(none, 1.0, most))).clamp(-127, 127)
    return torch.where(none, 0.0, codes), torch.where(none, 2.0 ** -31, most / 127.0)


def _store(case, cache, slots, k, v):
    """Writes fp32 keys and values [tokens, kv_heads, head_dim] to their slots."""
    d = case["head_dim"]
    page, block, r, s, jh, h, jl = _places(case, slots)
    at_k, at_v, scales = _views(case, cache)
    if case["bits"] == 16:
        at_k[page, :, block, :, :, r] = k.half().unflatten(-1, (d // 16, 2, 8))
        at_v[page, :, block, :, s, h, :, jh, jl] = v.half().unflatten(-1, (d // 32, 32))
        return
    k, scale_k = _quantize(k)
    v, scale_v = _quantize(v)
    at_k[page, :, block, :, :, r] = (k + 128).to(torch.uint8).unflatten(-1, (d // 32, 2, 16))
    at_v[page, :, block, :, h, :, s, jh, jl] = (v + 128).to(torch.uint8).unflatten(-1, (d // 32, 32))
    scales[page, :, block, :, r] = torch.cat([scale_k, scale_v, torch.log2(scale_v), 1.0 / scale_v], -1)


def _rotated(case, x, cos, sin):
    """x fp32 [tokens, heads, head_dim]: channels i and i + rotary / 2 are turned by the angle of position and i."""
    half = case["rotary"] // 2
    a, b, rest = x[..., :half], x[..., half:2 * half], x[..., 2 * half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)


def _plain_append(s):
    c = s["case"]
    tokens, d, half = s["q"].shape[0], c["head_dim"], c["rotary"] // 2
    row = s["cos_sin"][s["positions"].long()][:, None]
    cos, sin = row[..., :half], row[..., half:]
    s["q_out"].copy_(_rotated(c, s["q"].float().view(tokens, -1, d), cos, sin).view(tokens, -1))
    _store(c, s["cache"], s["slots"], _rotated(c, s["k"].float().view(tokens, -1, d), cos, sin), s["v"].float().view(tokens, -1, d))
    page, block, r, hi, jh, h, jl = _places(c, s["slots"])
    at_k, at_v, scales = _views(c, s["cache"])
    if c["bits"] == 16:
        k, v = at_k[page, :, block, :, :, r].float(), at_v[page, :, block, :, hi, h, :, jh, jl].float()
    else:
        of = scales[page, :, block, :, r]
        k = (at_k[page, :, block, :, :, r].float() - 128).flatten(2) * of[:, :, 0, None]
        v = (at_v[page, :, block, :, h, :, hi, jh, jl].float() - 128).flatten(2) * of[:, :, 1, None]
    s["k_back"].copy_(k.reshape(tokens, -1))
    s["v_back"].copy_(v.reshape(tokens, -1))
    return s["q_out"], s["k_back"], s["v_back"]


def _plain_attend(s):
    c = s["case"]
    n, d, kv_heads, most = c["requests"], c["head_dim"], c["kv_heads"], s["most"]
    group, tokens = c["heads"] // kv_heads, s["q"].shape[0]
    columns = _pages(s["longest"], c["page"])
    length = columns * c["page"]
    pages = s["cache"][s["table"][:, :columns].long().clamp(min=0)]                  # [n, columns, kv_heads, blocks, bytes]
    k, v, scales = _views(c, pages)
    k = k.permute(0, 2, 4, 5, 7, 1, 3, 6).reshape(n, kv_heads, d, length).float()
    v = v.permute((0, 2, 1, 3, 5, 8, 6, 9, 4, 7) if c["bits"] == 16 else (0, 2, 1, 3, 7, 8, 5, 9, 4, 6)).reshape(n, kv_heads, length, d).float()
    if c["bits"] == 8:
        of = scales.permute(4, 0, 2, 1, 3, 5).reshape(4, n, kv_heads, length)
        k.sub_(128).mul_(of[0][:, :, None])
        v.sub_(128).mul_(of[1][..., None])
    cu, ctx, kv = s["cu"].long(), s["ctx"].long(), s["kv_len"].long()
    i = torch.arange(most, device=DEV)
    rows = (cu[:-1, None] + i).clamp(max=tokens - 1)                                  # [n, most], past the request's end as well
    q = s["q"].view(tokens, kv_heads, group, d)[rows].permute(0, 2, 3, 1, 4).reshape(n, kv_heads, group * most, d).float()
    at, j = ctx[:, None] + i, torch.arange(length, device=DEV)
    seen = (j < kv[:, None])[:, None].expand(n, most, length)
    if c["causal"]:
        seen = seen & (j <= at[..., None])
        if c["window"]:
            seen = seen & (j > at[..., None] - c["window"])
    p = torch.matmul(q, k).mul_(d ** -0.5).view(n, kv_heads, group, most, length)
    p.masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, kv_heads, group * most, length), v).view(n, kv_heads, group, most, d)
    o = torch.where(total > 0, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n * most, -1)
    t = torch.arange(tokens, device=DEV)
    whose = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    s["y"].copy_(o[whose * most + t - cu[whose]])
    return s["y"]


# ---- in 64 bits --------------------------------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "resize":
        return None                                   # whole numbers
    s = prepare(case, seed)
    d = case["head_dim"]
    if case["op"] == "append":
        half, t = case["rotary"] // 2, s["q"].shape[0]
        turn = s["cos_sin"].double()[s["positions"].long()]
        turned = []
        for x in (s["q"], s["k"]):
            x = x.double().view(t, -1, d)
            y = x.clone()
            y[..., :half] = x[..., :half] * turn[:, None, :half] - x[..., half:2 * half] * turn[:, None, half:]
            y[..., half:2 * half] = x[..., half:2 * half] * turn[:, None, :half] + x[..., :half] * turn[:, None, half:]
            turned.append(y)
        back = []
        for x in (turned[1], s["v"].double().view(t, -1, d)):
            if case["bits"] == 8:
                # a code is a decision of the operator's fp32 steps, which are stated: the products of the rotation rounded, then their sum
                f = x.float()
                if x is turned[1]:
                    a, b = s["k"].float().view(t, -1, d)[..., :half], s["k"].float().view(t, -1, d)[..., half:2 * half]
                    co, si = turn[:, None, :half].float(), turn[:, None, half:].float()
                    f[..., :half] = torch.sub(torch.mul(a, co), torch.mul(b, si))
                    f[..., half:2 * half] = torch.add(torch.mul(b, co), torch.mul(a, si))
                most = f.abs().amax(-1, keepdim=True)
                x = torch.round(f * torch.div(127.0, most)).double() * torch.div(most, 127.0).double()
            back.append(x.view(t, -1))
        return turned[0].view(t, -1), back[0], back[1]
    heads, kv_heads, page = case["heads"], case["kv_heads"], case["page"]
    group, wide = heads // kv_heads, case["bits"] == 16
    ctx, new = _lengths(case)
    raw = s["cache"].view(-1)
    size = _block_bytes(case)
    y = torch.zeros((s["q"].shape[0], heads, d), dtype=torch.float64, device=DEV)
    channel = torch.arange(d, device=DEV)
    row = 0
    for b in range(case["requests"]):
        kv = ctx[b] + new[b]
        j = torch.arange(kv, device=DEV)
        block = s["table"][b].long()[j // page] * kv_heads * (page // 32) + j % page // 32
        r = j % 32
        for h in range(kv_heads):
            at = (block + h * (page // 32)) * size                       # first byte of every token's block
            if wide:
                in_k = (channel // 16) * 512 + (channel % 16 // 8) * 256 + channel % 8
                in_v = (channel // 32) * 1024 + (channel % 32) * 8
                of_v = (r // 16) * 512 + (r // 4 % 2) * 256 + (r // 8 % 2) * 4 + r % 4
                data = raw.view(torch.float16)
                k = data[(at // 2 + r * 8)[:, None] + in_k].double()
                v = data[(at // 2 + 32 * d + of_v)[:, None] + in_v].double()
            else:
                in_k = (channel // 32) * 1024 + (channel % 32 // 16) * 512 + channel % 16
                in_v = (channel // 32) * 1024 + (channel % 32) * 16
                of_v = (r // 4 % 2) * 512 + (r // 16) * 8 + (r // 8 % 2) * 4 + r % 4
                scale = raw.view(torch.float32)
                k = (raw[(at + r * 16)[:, None] + in_k].double() - 128) * scale[(at + 64 * d) // 4 + r].double()[:, None]
                v = (raw[(at + 32 * d + of_v)[:, None] + in_v].double() - 128) * scale[(at + 64 * d) // 4 + 32 + r].double()[:, None]
            kt = k.t().contiguous()
            for i in range(0, new[b], 4096):
                m = min(4096, new[b] - i)
                q = s["q"][row + i:row + i + m].view(m, kv_heads, group, d)[:, h].double()
                w = torch.matmul(q.reshape(m * group, d), kt).view(m, group, kv) * (1.0 / math.sqrt(d))
                pos = (ctx[b] + i + torch.arange(m, device=DEV))[:, None]
                if case["causal"]:
                    hidden = j[None] > pos
                    if case["window"]:
                        hidden = hidden | (j[None] <= pos - case["window"])
                    w.masked_fill_(hidden[:, None], -math.inf)
                w = torch.softmax(w, -1)
                y[row + i:row + i + m, h * group:(h + 1) * group] = torch.matmul(w.view(m * group, kv), v).view(m, group, d)
        row += new[b]
    return y.view(-1, heads * d)
