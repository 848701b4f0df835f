// Attention over the paged cache: which kernel takes a call, and the sum of partial results (include/qlinear.h).
#include <algorithm>
#include <cmath>

#include "attention.h"

namespace ql {
namespace {

// Joins the parts of the rows whose tokens several workgroups shared: a thread takes 4 channels of a row, eight parts at a time with their
// weights, all asked for at once.  Bound by latency: the note, then the parts.
template <int D>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, AttnPlan plan, float factor)
{
    constexpr int LANES = D / 4, ROWS = 256 / LANES;
    const int kvh = blockIdx.x % a.kv.heads, at = blockIdx.y * ROWS + threadIdx.x / LANES, channel = threadIdx.x % LANES * 4;
    const AttnNote note = static_cast<const AttnNote *>(a.ws)[blockIdx.x / a.kv.heads];
    // (where cu_new decreases a tile may have left no note: whatever is there stays inside the workspace and y)
    const int row = note.row0 + at;
    if (note.parts < 2 || (unsigned)note.item >= (unsigned)plan.items || row < 0 || row >= note.rows) return;
    const int token = attn_token(a, row), parts = min(note.parts, plan.items - note.item);
    const int64_t t = (int64_t)note.cu + token;
    if (t < 0 || t >= a.T) return;
    const size_t step = (size_t)a.kv.heads * attn_partial_floats(plan.bm, D);
    const float *p0 = attn_partial(a, plan, note.item, kvh), *pm = p0 + (size_t)plan.bm * D + at, *ps = p0 + (size_t)at * D + channel;
    float m = -INFINITY, l = 0;
    f4 o = {0, 0, 0, 0};
    for (int k0 = 0; k0 < parts; k0 += 8) {
        float mk[8], lk[8];
        f4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {                                // (behind the last part: the last one again, with weight 0)
            const size_t off = min(k0 + i, parts - 1) * step;
            mk[i] = pm[off], lk[i] = pm[off + plan.bm], v[i] = *reinterpret_cast<const f4 *>(ps + off);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lk[i] = k0 + i < parts ? lk[i] : 0.f;
            top = fmaxf(top, mk[i]);
        }
        const float keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * factor);
        l *= keep, o *= keep, m = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = lk[i] == 0.f ? 0.f : __builtin_amdgcn_exp2f((mk[i] - top) * factor);   // (lk 0: nothing seen, its sums are 0; NaN stays)
            l += lk[i] * w;
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(v[i][c], w, o[c]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    __half *dst = a.y + t * a.ldy + (int64_t)(kvh * a.group + row - token * a.group) * D + channel;
    *reinterpret_cast<h4 *>(dst) = h4{(_Float16)(o[0] * inv), (_Float16)(o[1] * inv), (_Float16)(o[2] * inv), (_Float16)(o[3] * inv)};
}

// Tokens that a block table can hold up to which requests of few rows are not cut into parts, which takes a second launch (tiles of 128 rows: half
// of it).  us, whole / parts: 32 requests of one token, 8 heads, int8: on 400 tokens 8.4 / 10.3, 700 12.3 / 14.4, 1000 17.9 / 17.8; one, 12 heads:
// 400 7.1 / 8.9, 1000 9.3 / 9.1; one of 64 new tokens, 32 + 8 heads: 60 8.5 / 10.5, 200 12.0 / 13.9, 350 15.3 / 15.0.
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
    p.tiles = (int)tiles, p.items = (int)(tiles + p.slots);          // (no more items than that: see attn_part_units)
    p.far_first = !p.step && !p.slots && (int64_t)p.items * kv.heads <= 2048;
    p.ws_bytes = p.slots ? attn_notes_bytes(p.tiles) + (size_t)p.items * kv.heads * attn_partial_floats(bm, kv.D) * 4 : 0;
    return p;
}

AttnPlan attention_plan(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    const int group = q_heads / kv.heads, bm = tile_rows(kv, T, group, max_new);
    return plan_of(kv, (int64_t)T * group / bm + requests, bm);
}

// The most that a call with these sizes or smaller ones asks for: of every size of tiles that they have, the largest call that is cut.  With more
// heads than most_tiles none is.  Over all sizes 135.1 MB in tiles of 128 rows (D = 256), 135.2 of 16 (D = 256), 136.3 of 32 (D = 128, 4095 heads).
size_t attention_workspace_bytes(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    const int group = q_heads / kv.heads, largest = tile_rows(kv, T, group, max_new);
    size_t most = 0;
    for (int bm : {16, 32, 128}) {
        if (bm > largest) break;
        if (bm == 32 && kv.D == 256) continue;                       // (as tile_rows)
        const int64_t limit = most_tiles(bm) / kv.heads;
        if (limit) most = std::max(most, plan_of(kv, std::min((int64_t)T * group / bm + requests, limit), bm).ws_bytes);
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
    if ((int64_t)a.columns << a.kv.page_shift <= (p.step ? SHORT : SHORT / 2)) p.slots = 0, p.items = p.tiles, p.far_first = !p.step, p.step *= 2;
    if ((int64_t)p.items * a.kv.heads >= (int64_t)1 << 31)
        return fail(QL_ERR_UNSUPPORTED, "%d tokens of %d query heads are more than a launch holds", a.T, a.q_heads);
    // exp(scale s) = exp2(c s); a scale of nothing keeps masked scores apart from the others (-inf times 0 would be NaN)
    const float c = fmaxf(std::fabs(a.scale) * 1.44269504088896341f, 1e-30f);
    QL_TRY(p.step ? launch_attention_steps(a, p, c, st) : launch_attention_tiles(a, p, c, st));
    if (!p.slots) return QL_OK;
    const dim3 grid(p.tiles * a.kv.heads, p.bm * a.kv.D / 1024);
    const float factor = a.kv.bits == 16 ? c : 1.0f;                 // (int8: in the scores already, with the keys' scales)
    if (a.kv.D == 64) attn_join_kernel<64><<<grid, 256, 0, st>>>(a, p, factor);
    else if (a.kv.D == 128) attn_join_kernel<128><<<grid, 256, 0, st>>>(a, p, factor);
    else attn_join_kernel<256><<<grid, 256, 0, st>>>(a, p, factor);
    return check_hip(hipGetLastError(), "attn_join_kernel");
}

}  // namespace ql
