"""The paged cache's operators together, as a serving loop uses them: PagedRequests and PagedDecoderLayer over steps of prompts, decoded
tokens, ended and new requests, against the oracle stage by stage (what a stage is fed is what the GPU's stage before gave it), and the
same calls captured into graphs, on other streams and with shared workspaces."""
import numpy as np
import pytest
import torch

from oracle import kv
from paper_2512_23367_amd import binding as ql, synth
from paper_2512_23367_amd.layer import DecoderLayerLinears, PagedDecoderLayer, PagedRequests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def U():
    import kv_util
    return kv_util


def _layer(U, fmt, q_heads, d, F, bits, max_tokens, max_requests):
    ws = [synth.weights((q_heads + 2 * fmt.heads) * fmt.head_dim, d, 1, "qkv"), synth.weights(d, q_heads * fmt.head_dim, 1, "o"), synth.weights(2 * F, d, 1, "gate_up"),
          synth.weights(d, F, 1, "down")]
    angle = np.arange(600)[:, None] * 10000.0 ** (-np.arange(fmt.head_dim // 2) / (fmt.head_dim // 2))
    cos_sin = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    return PagedDecoderLayer(*(U.dev(w) for w in ws), bits, max_tokens, fmt, U.dev(cos_sin), max_requests), cos_sin, ws


@pytest.mark.parametrize("bits,kv_bits,D,q_heads,heads,page", [(8, 8, 64, 4, 2, 32), (8, 16, 128, 4, 4, 64), (4, 8, 128, 6, 2, 64), (8, 16, 256, 2, 1, 32)])
def test_steps_of_a_serving_loop(U, bits, kv_bits, D, q_heads, heads, page):
    rng = np.random.default_rng(D + page)
    d, F, n, most = 256, 384, 4, 300
    fmt = ql.QlKvFormat(heads=heads, head_dim=D, page_size=page, pages=2 + 900 // page, bits=kv_bits)
    layer, cos_sin, _ = _layer(U, fmt, q_heads, d, F, bits, most, n)
    requests = PagedRequests(fmt, n, 300 // page, most, U.DEV)
    cache = torch.full((ql.ql_kv_cache_bytes(fmt),), 0xFF, dtype=torch.uint8, device=U.DEV)
    keys, values, length = [np.zeros((0, heads, D))] * n, [np.zeros((0, heads, D))] * n, [0] * n
    # prompts of three requests; tokens; one ends, one begins; tokens and a draft of five; all but one end
    for want in ([37, 5, 0, 200], [38, 6, 0, 201], [39, 0, 70, 202], [40, 0, 71, 207], [40, 33, 72, 207], [0, 34, 0, 0]):
        new = [max(0, w - o) for w, o in zip(want, length)]
        T = sum(new)
        pad = 3                                                        # rows of a padded batch
        x = U.dev(synth.activations(T + pad, d, 0, "single"))
        requests.step(U.ints(want), max_new=max(new))
        y = layer.forward(x, requests, cache)
        torch.cuda.synchronize()
        assert requests.kv_len.cpu().tolist() == want and requests.pool.cpu().tolist()[2] == 0
        cu = requests.cu_new.cpu().numpy()
        assert cu.tolist() == np.concatenate([[0], np.cumsum(new)]).tolist()

        # the QKV projection once more: its queries were turned in place
        qkv = torch.empty_like(layer.y_qkv[:T + pad])
        layer._linear(x, "qkv", qkv)
        rows = qkv.cpu().numpy()[:T].astype(np.float16)
        pos = np.concatenate([np.arange(o, w) for o, w in zip(length, want) if w > o] or [[]]).astype(int)
        assert (requests.positions.cpu().numpy()[:T] == pos).all()
        q = kv.rotate(rows[:, :q_heads * D].reshape(T, q_heads, D), cos_sin, pos, D).astype(np.float16)
        assert (layer.y_qkv[:T, :q_heads * D].cpu().numpy() == q.reshape(T, -1)).all()
        k = kv.rotate(rows[:, q_heads * D:(q_heads + heads) * D].reshape(T, heads, D), cos_sin, pos, D)
        v = rows[:, (q_heads + heads) * D:].reshape(T, heads, D).astype(np.float32)
        ks, vs = kv.stored(k, v, kv_bits) if T else (k, v)
        r = object.__new__(U.Requests)                                 # the oracle's view of the step
        r.ctx, r.new, r.len, r.D, r.heads, r.q, r.cu = length, new, want, D, q_heads, q.reshape(T, -1), cu
        for b in range(n):
            keys[b] = np.concatenate([keys[b][:want[b]], ks[cu[b]:cu[b + 1]]])
            values[b] = np.concatenate([values[b][:want[b]], vs[cu[b]:cu[b + 1]]])
        r.k, r.v = keys, values
        r.check(layer.y_attention[:T])
        # what lies behind is the linears' own path, on the rows that attention gave it
        plain = layer._behind_attention(layer.y_attention[:T + pad].clone()).clone()
        assert torch.equal(plain[:T], y[:T]) and torch.isfinite(y[:T]).all()
        length = want


def test_the_linears_alone_are_what_they_were(U):
    ws = [synth.weights(3 * 256, 256, 1, "qkv"), synth.weights(256, 256, 1, "o"), synth.weights(768, 256, 1, "gate_up"), synth.weights(256, 384, 1, "down")]
    layer = DecoderLayerLinears(*(U.dev(w) for w in ws), 8, 40)
    x = U.dev(synth.activations(40, 256, 0, "single"))
    y = layer.forward(x).clone()
    qkv = torch.empty((40, 768), dtype=torch.float16, device=U.DEV)
    layer._linear(x, "qkv", qkv)
    assert torch.equal(qkv, layer.y_qkv) and torch.equal(layer._behind_attention(qkv[:, :256]), y)


@pytest.mark.parametrize("kv_bits", [8, 16])
def test_a_captured_step_replays_with_other_lengths(U, kv_bits):
    """The whole step -- lengths, cache, attention, linears -- in one graph: every replay decodes one token per request, as the eager layer
    does on a copy of the state, bit for bit."""
    D, q_heads, heads, page, d, n = 64, 4, 2, 32, 256, 3
    fmt = ql.QlKvFormat(heads=heads, head_dim=D, page_size=page, pages=60, bits=kv_bits)
    layer, _, _ = _layer(U, fmt, q_heads, d, 384, 8, 200, n)
    caches = [torch.zeros(ql.ql_kv_cache_bytes(fmt), dtype=torch.uint8, device=U.DEV) for _ in range(2)]
    states = [PagedRequests(fmt, n, 16, 200, U.DEV) for _ in range(2)]
    prompt = U.dev(synth.activations(131, d, 0, "single"))
    for s, c in zip(states, caches):
        s.step(U.ints([30, 1, 100]))
        layer.forward(prompt, s, c)
    x = U.dev(synth.activations(n, d, 1, "qkv"))
    one = U.ints([1] * n)

    def step(s, c):
        s.step(s.kv_len + one, max_new=1)
        return layer.forward(x, s, c)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    kept = {k: getattr(states[1], k).clone() for k in ("kv_len", "ctx_len", "block_table", "ring", "pool")}
    step(states[1], caches[1])                                          # (the first launch of a kernel sets its attributes)
    torch.cuda.synchronize()
    for k, v in kept.items():
        getattr(states[1], k).copy_(v)
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            out = step(states[1], caches[1])
    torch.cuda.synchronize()
    for rep in range(70):                                               # over the ends of two pages
        want = step(states[0], caches[0]).clone()
        torch.cuda.synchronize()
        layer.y.fill_(7)                                                # eager work between the replays
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), rep
        for k in ("kv_len", "pool", "slots", "block_table"):
            assert torch.equal(getattr(states[0], k), getattr(states[1], k)), (rep, k)
    assert states[1].kv_len.cpu().tolist() == [100, 71, 170]


def test_two_graphs_that_share_a_workspace(U):
    """Captured one after the other with the same workspace and replayed in turn: each gives what it gives alone."""
    a = U.Requests(1, [3000, 40], [1, 1], 8, 2, 128, 8, 64)
    b = U.Requests(2, [700], [60], 4, 1, 64, 16, 32)
    need = max(ql.ql_paged_attention_bytes(r.fmt, r.T, len(r.ctx), r.heads, 0) for r in (a, b))
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=U.DEV)
    graphs = []
    side = torch.cuda.Stream()
    for r in (a, b):
        args = (U.dev(r.q), r.cache, r.fmt, U.ints(r.table), U.ints(r.cu), U.ints(r.ctx), U.ints(r.len), r.D ** -0.5)
        y = torch.zeros_like(args[0])
        ql.ql_paged_attention(*args, y, ws)
        torch.cuda.synchronize()
        want, g = y.clone(), torch.cuda.CUDAGraph()
        r.check(want)
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                ql.ql_paged_attention(*args, y, ws)
        graphs.append((g, y, want, args))
    for _ in range(3):
        for g, y, want, _ in graphs:
            y.fill_(7)
            ws.fill_(0xEE)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)


def test_calls_on_two_streams_with_workspaces_of_their_own(U):
    rs = [U.Requests(3, [2500, 900], [1, 1], 8, 2, 128, 8, 64), U.Requests(4, [100], [300], 4, 4, 128, 16, 32)]
    want = [r.call() for r in rs]
    for r, w in zip(rs, want):
        r.check(w)
    sets = [(U.dev(r.q), r.cache, r.fmt, U.ints(r.table), U.ints(r.cu), U.ints(r.ctx), U.ints(r.len), r.D ** -0.5) for r in rs]
    ws = [torch.empty(max(1, ql.ql_paged_attention_bytes(r.fmt, r.T, len(r.ctx), r.heads)), dtype=torch.uint8, device=U.DEV) for r in rs]
    ys = [torch.zeros_like(s[0]) for s in sets]
    streams = [torch.cuda.Stream() for _ in rs]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, w, y, st in zip(sets, ws, ys, streams):
            with torch.cuda.stream(st):
                y.fill_(7)
                ql.ql_paged_attention(*s, y, w)
    torch.cuda.synchronize()
    for y, w in zip(ys, want):
        assert torch.equal(y, w)


def test_a_smaller_workspace_serves_smaller_calls(U):
    """ql_paged_attention_bytes of the largest sizes is enough for every smaller call."""
    fmt = ql.QlKvFormat(heads=2, head_dim=128, page_size=64, pages=10, bits=8)
    for heads in (2, 8, 14):
        for T, n, new in ((1, 1, 1), (64, 64, 1), (300, 20, 0), (5000, 70, 7), (5000, 70, 0), (9000, 9000, 1)):
            most = ql.ql_paged_attention_bytes(fmt, T, n, heads, new)
            for t in {1, 2, 3, 5, 17, 33, 64, 100, 299, 1000, 4000, T}:
                for m in {1, 5, 64, n}:
                    for k in {1, 2, 3, 9, 65, new}:
                        if t <= T and m <= n and (new == 0 or 0 < k <= new):
                            assert ql.ql_paged_attention_bytes(fmt, t, m, heads, k) <= most
    r = U.Requests(5, [40, 3, 700], [1, 1, 9], 8, 2, 128, 8, 64)
    ws = torch.full((ql.ql_paged_attention_bytes(r.fmt, 500, 30, 8),), 0xFF, dtype=torch.uint8, device=U.DEV)
    for max_new in (0, 1, 9, 400):
        r.check(r.call(ws=ws, max_new=max_new))


def test_a_step_without_new_tokens_and_formats_that_differ(U):
    fmt = ql.QlKvFormat(heads=2, head_dim=64, page_size=32, pages=8, bits=8)
    layer, _, _ = _layer(U, fmt, 4, 256, 512, 8, 16, 3)
    cache = torch.empty(ql.ql_kv_cache_bytes(fmt), dtype=torch.uint8, device=U.DEV)
    requests = PagedRequests(fmt, 3, 4, 16)
    requests.step(U.ints([0, 0, 0]))
    assert layer.forward(torch.empty((0, 256), dtype=torch.float16, device=U.DEV), requests, cache).shape == (0, 256)
    assert requests.kv_len.tolist() == [0, 0, 0] and requests.pool.tolist() == [0, 8, 0, 0]
    other = PagedRequests(ql.QlKvFormat(heads=2, head_dim=64, page_size=64, pages=4, bits=8), 3, 4, 16)
    with pytest.raises(AssertionError):
        layer.forward(torch.empty((1, 256), dtype=torch.float16, device=U.DEV), other, cache)
