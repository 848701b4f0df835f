"""The four quantized linears of a decoder layer, chained on the device (buffer management and call order only:
every step runs in the library's kernels).

    x [M,d] --qkv--> [M,3d] --(first d columns stand in for the attention output)--> o --> [M,d]
      --gate_up--> [M,2F] --SwiGLU + per-token quantizer (ql_quant_act_swiglu)--> int8 [M,F] --down--> [M,d]

This is the prefill workload whose latency and weight memory the paper tabulates by batch size (Efficiency
Evaluation, Table 3: INT8 against FP16); attention itself, the normalisations and the residual adds are not part of
the quantized-linear path and are left out (the slice of the QKV output only makes the four GEMMs depend on each
other the way a layer's do).

    PagedDecoderLayer puts attention there: rotary embedding, the paged key/value cache and attention of the step's new
    tokens over it.  PagedRequests keeps the books of the requests that share the cache's pages; it serves all layers of a
    model, each of which has a cache of its own:

        requests = PagedRequests(fmt, max_requests, columns, max_tokens)
        requests.step(want_len, max_new)                           # tokens per request after this step, int32 on the device
        for layer, cache in zip(layers, caches): x = layer.forward(x, requests, cache)
"""
from __future__ import annotations

import torch

from . import binding as ql


class DecoderLayerLinears:
    def __init__(self, w_qkv, w_o, w_gate_up, w_down, bits: int, max_tokens: int, biases=None):
        """w_*: fp16 device tensors [N,K] (qkv [3d,d], o [d,d], gate_up [2F,d], down [d,F]); bits 8 (per-channel
        int8) or 4 (int4, groups of 128); biases: optional dict name -> fp16 [N]."""
        self.bits, self.group = bits, (0 if bits == 8 else 128)
        self.d = w_o.shape[0]
        self.F = w_down.shape[1]
        assert w_qkv.shape == self._qkv_shape(w_o) and w_gate_up.shape == (2 * self.F, self.d) and w_down.shape == (self.d, self.F)
        dev = w_o.device
        self.w = {}
        self.weight_bytes = 0
        for name, w in (("qkv", w_qkv), ("o", w_o), ("gate_up", w_gate_up), ("down", w_down)):
            N, K = w.shape
            _, sb, kb = ql.ql_weight_bytes(N, K, bits, self.group)
            scales = torch.empty(sb, dtype=torch.uint8, device=dev)
            kern = torch.empty(kb, dtype=torch.uint8, device=dev)
            ql.ql_quant_weight(w.contiguous(), bits, self.group, None, scales, kern)
            self.w[name] = (kern, scales.view(torch.float32) if bits == 8 else None, (biases or {}).get(name), N, K)
            self.weight_bytes += kb + (sb if bits == 8 else 0)
        M = max_tokens
        self.max_tokens = M
        self.y_qkv = torch.empty((M, w_qkv.shape[0]), dtype=torch.float16, device=dev)
        self.y_o = torch.empty((M, self.d), dtype=torch.float16, device=dev)
        self.y_gu = torch.empty((M, 2 * self.F), dtype=torch.float16, device=dev)
        self.y = torch.empty((M, self.d), dtype=torch.float16, device=dev)
        self.xq = torch.empty(ql.ql_act_kernel_bytes(M, self.F), dtype=torch.uint8, device=dev)
        self.sx = torch.empty(M, dtype=torch.float32, device=dev)
        ws = max(ql.ql_workspace_bytes(M, N, K, bits) for (_, _, _, N, K) in self.w.values())
        self.ws = torch.empty(ws, dtype=torch.uint8, device=dev)

    def _qkv_shape(self, w_o):
        return (3 * self.d, self.d)

    def _linear(self, x, name, y):
        kern, sw, bias, N, _ = self.w[name]
        if self.bits == 8:
            ql.ql_w8a8_linear(x, kern, sw, bias, N, y, self.ws)
        else:
            ql.ql_w4a8_linear(x, kern, self.group, bias, N, y, self.ws)

    def forward(self, x):
        """x fp16 [M,d], M <= max_tokens; returns the fp16 [M,d] output of the down projection (a view of an
        internal buffer, overwritten by the next call).  Everything is enqueued on torch's current stream."""
        M = x.shape[0]
        assert M <= self.max_tokens and x.shape[1] == self.d
        y_qkv = self.y_qkv[:M]
        self._linear(x, "qkv", y_qkv)
        return self._behind_attention(y_qkv[:, :self.d])

    def _behind_attention(self, y_attention):
        M = y_attention.shape[0]
        y_o, y_gu, y = self.y_o[:M], self.y_gu[:M], self.y[:M]
        self._linear(y_attention, "o", y_o)
        self._linear(y_o, "gate_up", y_gu)
        ql.ql_quant_act_swiglu(y_gu, None, self.xq, self.sx)
        kern, sw, bias, N, K = self.w["down"]
        if self.bits == 8:
            ql.ql_w8a8_gemm(self.xq, self.sx, M, K, kern, sw, bias, N, y, self.ws)
        else:
            ql.ql_w4a8_gemm(self.xq, self.sx, M, K, kern, self.group, bias, N, y, self.ws)
        return y


class PagedRequests:
    """The requests that share a cache's pages: block table, ring of free pages, and for the step at hand the slots and
    positions of the new tokens.  All on the device; step() only enqueues, so a step can be captured into a HIP graph."""

    def __init__(self, fmt: ql.QlKvFormat, max_requests: int, columns: int, max_tokens: int, device="cuda"):
        """columns: pages that one request can have; max_tokens: new tokens of one step."""
        ints = lambda *s: torch.zeros(s, dtype=torch.int32, device=device)  # noqa: E731
        self.fmt, self.max_requests, self.max_tokens = fmt, max_requests, max_tokens
        self.block_table = ints(max_requests, columns)
        self.ring = torch.arange(fmt.pages, dtype=torch.int32, device=device)
        self.pool = torch.tensor([0, fmt.pages, 0, 0], dtype=torch.int32, device=device)   # [2]: tokens that found no page or row
        self.ctx_len, self.kv_len, self.cu_new = ints(max_requests), ints(max_requests), ints(max_requests + 1)
        self.slots, self.positions = ints(max_tokens), ints(max_tokens)
        self.max_new = 0

    def step(self, want_len, max_new: int = 0):
        """want_len int32 [max_requests]: tokens of every request after this step (0: none, its pages are free again; the
        new tokens are the rows of the step's x, request after request).  max_new: the most new tokens of one request; 0: not
        known.  It chooses the kernel of the attention, never its result: a decode step that does not pass 1 takes the one for
        prompts, 47 us for 34 with 32 requests of 32 + 8 heads, int8, on 200 to 4096 tokens.  Rows behind the last new token (a padded
        batch) are computed, but neither stored nor attended to."""
        self.max_new = max_new
        self.ctx_len.copy_(self.kv_len)
        self.slots.fill_(-1)
        ql.ql_kv_resize(self.fmt.page_size, self.ctx_len, want_len, self.ring, self.pool, self.pool, self.block_table, self.kv_len,
                        self.cu_new, self.slots, self.positions)


class PagedDecoderLayer(DecoderLayerLinears):
    """The four linears with attention over a paged cache between the QKV and the O projection."""

    def __init__(self, w_qkv, w_o, w_gate_up, w_down, bits: int, max_tokens: int, fmt: ql.QlKvFormat, cos_sin, max_requests: int,
                 biases=None, scale=None):
        """w_qkv fp16 [(q_heads + 2 heads) head_dim, d], w_o [d, q_heads head_dim], the others as in DecoderLayerLinears; cos_sin:
        rotary table of ql_kv_append (None: a layer without rotary embedding); scale: of the scores, head_dim ** -0.5 by default."""
        self.fmt, self.cos_sin = fmt, cos_sin
        self.q_heads = w_o.shape[1] // fmt.head_dim
        self.scale = fmt.head_dim ** -0.5 if scale is None else scale
        super().__init__(w_qkv, w_o, w_gate_up, w_down, bits, max_tokens, biases)
        self.y_attention = torch.zeros((max_tokens, self.q_heads * fmt.head_dim), dtype=torch.float16, device=w_o.device)
        # for any step; layers that run one after the other may be given one of them
        self.attention_ws = torch.empty(ql.ql_paged_attention_bytes(fmt, max_tokens, max_requests, self.q_heads), dtype=torch.uint8, device=w_o.device)
        self.max_requests = max_requests

    def _qkv_shape(self, w_o):
        assert w_o.shape[1] == self.q_heads * self.fmt.head_dim
        return ((self.q_heads + 2 * self.fmt.heads) * self.fmt.head_dim, self.d)

    def forward(self, x, requests: PagedRequests, cache):
        """x fp16 [M,d]: the new tokens of requests.step(), in its order; cache: this layer's, ql_kv_cache_bytes(fmt) bytes.
        Returns fp16 [M,d], a view of an internal buffer that the next call overwrites."""
        M, D = x.shape[0], self.fmt.head_dim
        assert M <= min(self.max_tokens, requests.max_tokens) and requests.max_requests <= self.max_requests and x.shape[1] == self.d
        assert (requests.fmt.page_size, requests.fmt.pages) == (self.fmt.page_size, self.fmt.pages)
        if M == 0:
            return self.y[:0]
        y_qkv, y_attention = self.y_qkv[:M], self.y_attention[:M]
        self._linear(x, "qkv", y_qkv)
        nq, nk = self.q_heads * D, self.fmt.heads * D
        q, k, v = y_qkv[:, :nq], y_qkv[:, nq:nq + nk], y_qkv[:, nq + nk:]
        turned = q if self.cos_sin is not None else None                 # (ql_kv_append takes queries only to turn them)
        ql.ql_kv_append(turned, k, v, self.cos_sin, requests.positions[:M], requests.slots[:M], turned, cache, self.fmt)
        ql.ql_paged_attention(q, cache, self.fmt, requests.block_table, requests.cu_new, requests.ctx_len, requests.kv_len, self.scale, y_attention,
                              self.attention_ws, max_new=requests.max_new)
        return self._behind_attention(y_attention)
