// Attention over the paged cache: which kernel takes a call, and the sum of partial results (include/qlinear.h).
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace ql {
namespace {

// Joins the parts of the rows whose tokens several workgroups shared: a wavefront takes `rows` / 4 rows of an item and key/value head in
// turn, its lanes the channels; the weights of the parts (lane k: part k) first, so that the loads of the sums wait for nothing.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, AttnPlan plan, int rows)
{
    constexpr int N = D / 64;
    typedef float fn __attribute__((ext_vector_type(N)));
    const int kvh = blockIdx.x % a.kv.heads, item = blockIdx.x / a.kv.heads, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t step = (size_t)a.kv.heads * attn_partial_floats(plan.bm, D);
    const float *p0 = attn_partial(a, plan, item, kvh);
    // maximum and sum of part `lane` of the first row: asked for together with the note, which says whether there is one (one token on
    // 8000 14.4 -> 14.0 us)
    const int first = blockIdx.y * rows + wave;
    const float *pf = p0 + (size_t)plan.bm * D + first + min(lane, plan.items - 1 - item) * step;
    const float m0 = pf[0], l0 = pf[plan.bm];
    const int4 note = static_cast<const int4 *>(a.ws)[item];
    const int parts = min(note.x, plan.items - item);
    if (parts < 2) return;
    for (int at = first; at < min((int)(blockIdx.y + 1) * rows, plan.bm); at += 4) {
        const int row = note.z + at;
        if (row >= note.w) return;
        const float *pm = p0 + (size_t)plan.bm * D + at, *ps = p0 + (size_t)at * D + lane * N;
        auto most = [&](int k) { return k == lane && at == first ? m0 : pm[k * step]; };
        auto sum = [&](int k) { return k == lane && at == first ? l0 : pm[k * step + plan.bm]; };
        float m = -INFINITY;
        for (int k = lane; k < parts; k += 64) m = fmaxf(m, most(k));
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m = fmaxf(m, __shfl_xor(m, d));
        float l = 0, o[N];
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] = 0;
        for (int k0 = 0; k0 < parts; k0 += 64) {
            const int k = k0 + lane;
            const float lk = k < parts ? sum(k) : 0.f;
            const float w = lk == 0.f ? 0.f : __builtin_amdgcn_exp2f(most(k) - m);   // (lk 0: nothing seen, its sums are 0; NaN stays)
            l += lk * w;
            for (int i0 = 0; i0 < min(parts - k0, 64); i0 += 8) {             // (behind the last part: the last one again, with weight 0)
                fn v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const fn *>(ps + min(k0 + i0 + i, parts - 1) * step);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float wi = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), i0 + i));
#pragma unroll
                    for (int c = 0; c < N; ++c) o[c] = fmaf(v[i][c], wi, o[c]);
                }
            }
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) l += __shfl_xor(l, d);
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const int token = attn_token(a, row);
        __half *dst = a.y + (int64_t)(note.y + token) * a.ldy + (int64_t)(kvh * a.group + row - token * a.group) * D + lane * N;
#pragma unroll
        for (int c = 0; c < N; ++c) dst[c] = __float2half(o[c] * inv);
    }
}

constexpr int SHORT = 1024;

}  // namespace

// Rows of a tile for requests of at most `rows` rows.  Fewer than 128: the kernel for few rows.  D = 256 leaves it registers for 16.
// 256 rows: keys and values come to a CU once for all eight of its wavefronts instead of once for every four, whose every load costs
// the instruction issue of ten vector operations; where there are such tiles for three CUs in four.
// us, 128 / 256 rows, 32 + 8 heads: 16384 tokens fp16 2190 / 2080; 2 x 1000 on 9000 and 17000 int8 680 / 627; 4096, 32 + 32 heads, 171 / 151, int8 191 / 165;
// 2048, 12 + 12 heads (108 tiles of 256) 52 / 52; D = 64, 8192 tokens int8 398 / 430.
static int tile_rows(const KvView &kv, int T, int group, int max_new)
{
    const int64_t rows = (int64_t)(max_new && max_new < T ? max_new : T) * group;
    if (rows <= 16) return 16;
    if (rows <= 32 && kv.D < 256) return 32;
    return kv.D == 128 && rows >= 256 && (int64_t)T * group / 256 * kv.heads >= 192 ? 256 : 128;
}

// Tiles of a call that is cut into parts, at most: where they are more, there is enough of them for every CU; tiles of few rows, whose
// time a single long request may be, as far as the partial results stay small.  (Tiles of 256 rows cut into one to four parts for every
// CU, against whole ones: 2 x 1000 tokens on 9000 and 17000 654 us, 647; 4096 tokens, 32 + 32 heads, 164, 155.)
static int64_t most_tiles(int bm) { return bm == 256 ? 0 : bm == 128 ? 511 : 4095; }

static AttnPlan plan_of(const KvView &kv, int64_t tiles, int bm)
{
    AttnPlan p = {};
    p.bm = bm, p.step = bm < 128;
    p.slots = tiles * kv.heads > most_tiles(bm) ? 0 : std::max(1, 512 / kv.heads);
    p.items = (int)(tiles + p.slots);                                // tiles cut into c = work / slots units, or fewer
    p.far_first = !p.step && !p.slots && (int64_t)p.items * kv.heads <= 2048;
    p.ws_bytes = p.slots ? attn_notes_bytes(p.items) + (size_t)p.items * kv.heads * attn_partial_floats(bm, kv.D) * 4 : 0;
    return p;
}

AttnPlan attention_plan(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    const int group = q_heads / kv.heads, bm = tile_rows(kv, T, group, max_new);
    return plan_of(kv, (int64_t)T * group / bm + requests, bm);
}

// The most that a call with these sizes or smaller ones asks for.
size_t attention_workspace_bytes(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    const int group = q_heads / kv.heads, largest = tile_rows(kv, T, group, max_new);
    size_t most = 0;
    for (int bm : {16, 32, 128}) {
        if (bm > largest) break;
        const int64_t limit = most_tiles(bm) / kv.heads;             // of the largest call that is cut
        most = std::max(most, plan_of(kv, std::min((int64_t)T * group / bm + requests, limit), bm).ws_bytes);
    }
    return most;
}

int launch_attention(const AttnArgs &a, hipStream_t st)
{
    AttnPlan p = attention_plan(a.kv, a.T, a.requests, a.q_heads, a.max_new);
    if (p.ws_bytes) {
        if (!a.ws) return fail(QL_ERR_NULL, "ws is NULL");
        if (a.ws_bytes < p.ws_bytes) return fail(QL_ERR_WORKSPACE, "workspace has %zu bytes, this call needs %zu (see ql_paged_attention_bytes)", a.ws_bytes, p.ws_bytes);
    }
    if (p.step && (int64_t)a.columns << a.kv.page_shift <= SHORT) p.slots = 0, p.items = (int)((int64_t)a.T * a.group / p.bm + a.requests);
    if ((int64_t)p.items * a.kv.heads >= (int64_t)1 << 31)
        return fail(QL_ERR_UNSUPPORTED, "%d tokens of %d query heads are more than a launch holds", a.T, a.q_heads);
    // exp(scale s) = exp2(c s); a scale of nothing keeps masked scores apart from the others (-inf times 0 would be NaN)
    const float c = fmaxf(std::fabs(a.scale) * 1.44269504088896341f, 1e-30f);
    QL_TRY(p.step ? launch_attention_steps(a, p, c, st) : launch_attention_tiles(a, p, c, st));
    if (!p.slots) return QL_OK;
    const int rows = p.step ? 4 : 8;                                 // (tiles of 128 rows, 40 of them there: 4 rows 76.0 us, 8 75.5, 16 78, 32 83)
    const dim3 grid(p.items * a.kv.heads, p.bm / rows);
    if (a.kv.D == 64) attn_join_kernel<64><<<grid, 256, 0, st>>>(a, p, rows);
    else if (a.kv.D == 128) attn_join_kernel<128><<<grid, 256, 0, st>>>(a, p, rows);
    else attn_join_kernel<256><<<grid, 256, 0, st>>>(a, p, rows);
    return check_hip(hipGetLastError(), "attn_join_kernel");
}

}  // namespace ql
