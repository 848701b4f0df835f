// Attention over the paged cache: which kernel takes a call, and the sum of partial results (include/qlinear.h).
#include <cmath>

#include "attention.h"

namespace ql {
namespace {

// Joins the parts of the rows whose tokens several workgroups shared: one workgroup per new token, a wavefront per query head in turn.
template <int D>
__global__ __launch_bounds__(ATTN_THREADS) void attn_join_kernel(AttnArgs a, AttnPlan plan)
{
    constexpr int N = D / 64;
    __shared__ AttnScratch scratch;
    __shared__ int owner;
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t tiles;
    const int64_t work = attn_work<ATTN_THREADS>(a, plan.bm, scratch.part, tiles);
    const int c = attn_part_units(work, plan.target);
    // t's request, and the items before it
    if (tid == 0) owner = -1;
    __syncthreads();
    for (int b = tid; b < a.requests; b += ATTN_THREADS) {
        const AttnSpan r = attn_span(a, b);
        if (t >= r.cu && t < r.cu + r.rows / a.group) owner = b;
    }
    __syncthreads();
    const int b = owner;
    if (b < 0) return;
    const AttnSpan r = attn_span(a, b);
    const int parts = attn_parts(r, c);
    if (parts == 1) return;
    int64_t n = 0, before;
    for (int i = tid; i < b; i += ATTN_THREADS) {
        const AttnSpan s = attn_span(a, i);
        n += (int64_t)attn_tiles(s, plan.bm) * attn_parts(s, c);
    }
    block_sum_before<ATTN_THREADS>(n, scratch.part, before);

    const size_t size = attn_partial_floats(plan.bm, D);
    for (int head = wave; head < a.q_heads; head += ATTN_THREADS / 64) {
        const int kvh = head / a.group, row = (t - r.cu) * a.group + head % a.group;
        const int64_t item = before + (int64_t)(row / plan.bm) * parts;
        if (item + parts > plan.items) continue;             // (lengths that contradict each other)
        const float *p0 = static_cast<const float *>(a.ws) + ((size_t)item * a.kv.heads + kvh) * size;
        const size_t step = (size_t)a.kv.heads * size;
        const int at = row % plan.bm;
        float m = -INFINITY;
        for (int k = 0; k < parts; ++k) m = fmaxf(m, p0[k * step + (size_t)plan.bm * D + at]);
        float l = 0, o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = 0;
        for (int k = 0; k < parts; ++k) {
            const float *p = p0 + k * step;
            const float mk = p[(size_t)plan.bm * D + at], lk = p[(size_t)plan.bm * (D + 1) + at];
            const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(mk - m);
            l += lk * w;
#pragma unroll
            for (int i = 0; i < N; ++i) o[i] = fmaf(lk == 0.f ? 0.f : p[(size_t)at * D + lane + 64 * i], w, o[i]);
        }
        const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
        for (int i = 0; i < N; ++i) a.y[(int64_t)t * a.ldy + (int64_t)head * D + lane + 64 * i] = __float2half(o[i] * inv);
    }
}

}  // namespace

AttnPlan attention_plan(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    AttnPlan p = {};
    const int group = q_heads / kv.heads;
    const int64_t rows = (int64_t)(max_new && max_new < T ? max_new : T) * group;   // most of a request
    p.step = rows <= (kv.D == 256 ? 16 : 32);
    p.bm = !p.step ? 128 : rows <= 16 ? 16 : 32;
    const int64_t tiles = (int64_t)T * group / p.bm + requests;
    p.target = !p.step && tiles * kv.heads >= 512 ? 0 : ceil_div(512, kv.heads);
    p.items = (int)(tiles + p.target);
    p.ws_bytes = p.target ? (size_t)p.items * kv.heads * attn_partial_floats(p.bm, kv.D) * 4 : 0;
    return p;
}

size_t attention_workspace_bytes(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    return attention_plan(kv, T, requests, q_heads, max_new).ws_bytes;
}

int launch_attention(const AttnArgs &a, hipStream_t st)
{
    const AttnPlan p = attention_plan(a.kv, a.T, a.requests, a.q_heads, a.max_new);
    if ((int64_t)p.items * a.kv.heads >= (int64_t)1 << 31)
        return fail(QL_ERR_UNSUPPORTED, "%d tokens of %d query heads are more than a launch holds", a.T, a.q_heads);
    // exp(scale s) = exp2(c s); a scale of nothing keeps masked scores apart from the others (-inf times 0 would be NaN)
    const float c = fmaxf(std::fabs(a.scale) * 1.44269504088896341f, 1e-30f);
    QL_TRY(p.step ? launch_attention_steps(a, p, c, st) : launch_attention_tiles(a, p, c, st));
    if (!p.target) return QL_OK;
    if (a.kv.D == 64) attn_join_kernel<64><<<a.T, ATTN_THREADS, 0, st>>>(a, p);
    else if (a.kv.D == 128) attn_join_kernel<128><<<a.T, ATTN_THREADS, 0, st>>>(a, p);
    else attn_join_kernel<256><<<a.T, ATTN_THREADS, 0, st>>>(a, p);
    return check_hip(hipGetLastError(), "attn_join_kernel");
}

}  // namespace ql
