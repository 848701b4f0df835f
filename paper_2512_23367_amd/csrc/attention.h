// What the attention kernels share: which work a workgroup takes, and how parts of a row's tokens are joined.
//
// A row is one new token of one query head.  The G query heads that share a key/value head are rows of one problem: row r of a
// request is token r / G, head r % G of the group, so that keys and values are fetched once for all of them.  A workgroup takes
// a tile of `bm` consecutive rows of one request and key/value head, and all of the tokens that they see, or a part of them.
//
// Lengths are known on the device only (a captured step is replayed with others).  The host launches as many workgroups as the sizes
// that it knows allow for, and each finds its work from the lengths: request b has tiles_b = ceil(new_b G / bm) tiles and
// parts_b = ceil(units_b / c) parts of each (units of 64 tokens); see attn_part_units for c.  Without parts (slots 0): one per tile.
#pragma once

#include <type_traits>

#include "kv_cache.h"
#include "quant_math.h"

namespace ql {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr int ATTN_UNIT = 64;            // tokens that tiles of keys are aligned to, and parts of a row's tokens
constexpr int ATTN_THREADS = 512;

// Weights are 2^(score - maximum + ATTN_LEAD): fp16 reaches 2^16, the maximum that the kernels keep may be 2^8 behind, and what is left goes to the
// small ones.  Rounded to fp16 they lose 2^-11 of themselves down to 2^-21 of the maximum's weight, below it 2^-32 of that (without the lead 2^-25: of
// 120000 tokens of 2^-25 each behind one far ahead nothing was left, 0.3 % of the sum).
constexpr float ATTN_LEAD = 7.0f;
// Maxima beyond this (in powers of two) are subtracted from the scores before the factor is applied: 2^(fma(s, c, 7 - m c)) takes fewer operations, but what is lost
// in rounding m c is a factor of all of a row's weights, which takes them out of fp16 from 2^24 on (a row of NaN).  The branch costs 0.5 % (16384 tokens
// 1996 us, 2001; decode steps 33.9 as without it), small prompts of D = 64 1.5 %.
constexpr float ATTN_FAR = 1024.0f;
__device__ inline bool attn_far(float m, float factor) { return m != -INFINITY && __builtin_fabsf(m) * factor > ATTN_FAR; }

// r / group: see AttnArgs::group_mul
__device__ inline int attn_token(const AttnArgs &a, int r) { return (int)((__umulhi((unsigned)r, a.group_mul) + (unsigned)r) >> a.group_shift); }

// Eight channels of a query: an infinity becomes NaN (inf * 0), all else stays.  An infinite channel makes every score of its row infinite or NaN, and the
// softmax of those NaN; by the running maximum alone a row whose scores are all -inf would come out as one that sees nothing.
__device__ inline h8 attn_query(h8 x)
{
    const h8 zero = {};
    return __builtin_elementwise_fma(x, zero, x);
}

struct AttnSpan {                        // a request as the kernels see it
    int cu, rows, ctx, len;              // first row of q, rows (new tokens x heads of the group), position of the first new token, tokens
    int low, high;                       // tokens that any of its rows sees; low is a multiple of ATTN_UNIT
};

struct AttnItem {
    AttnSpan r;
    int b, tile, part, parts;
    int item;                            // its number: parts of a tile follow each other
    int ordinal;                         // of the tile, over all requests (with parts only); where there is no item left, one behind the last
                                         // for each workgroup too many
};

__device__ inline AttnSpan attn_span(const AttnArgs &a, int b)
{
    AttnSpan r;
    const int c0 = min(max(a.cu[b], 0), a.T), c1 = min(max(a.cu[b + 1], 0), a.T);
    r.cu = c0;
    r.rows = max(0, c1 - c0) * a.group;
    r.len = (int)min((int64_t)max(a.len[b], 0), (int64_t)a.columns << a.kv.page_shift);
    r.low = 0, r.high = r.len, r.ctx = 0;
    if (a.causal) {
        r.ctx = a.ctx[b];
        r.high = (int)max((int64_t)0, min((int64_t)r.len, (int64_t)r.ctx + max(0, c1 - c0)));
        if (a.window) r.low = (int)min((int64_t)r.high, max((int64_t)0, (int64_t)r.ctx - a.window + 1)) & -ATTN_UNIT;
    }
    return r;
}

__device__ inline int attn_units(int low, int high) { return (max(high - low, 0) + ATTN_UNIT - 1) / ATTN_UNIT; }

__device__ inline int attn_tiles(const AttnSpan &r, int bm) { return (r.rows + bm - 1) / bm; }

// Units that a tile of the request sees, at most.
template <int bm>
__device__ inline int attn_tile_units(const AttnArgs &a, const AttnSpan &r)
{
    const int units = attn_units(r.low, r.high);
    return a.window ? (int)min((int64_t)units, ((int64_t)a.window + attn_token(a, bm - 1) + 2 * ATTN_UNIT) / ATTN_UNIT) : units;
}

// Parts of a tile's units, of about c each (any number covers them: see attn_part_range).
constexpr int ATTN_LEAST = 4;
__device__ inline int attn_parts(int units, float c) { return max(1, (int)(units * __builtin_amdgcn_rcpf(c) + 0.9999f)); }

// over a wavefront, the same in every lane
template <typename T, typename OP>
__device__ inline T wave_all(T v, OP op)
{
    static_assert(sizeof(T) == 4, "one register");
    auto step = [&](auto off) {
        unsigned a, b;
        lane_pair<decltype(off)::value>(__builtin_bit_cast(unsigned, v), a, b);
        v = op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    };
    step(std::integral_constant<int, 1>{}), step(std::integral_constant<int, 2>{}), step(std::integral_constant<int, 4>{});
    step(std::integral_constant<int, 8>{}), step(std::integral_constant<int, 16>{}), step(std::integral_constant<int, 32>{});
    return v;
}
template <typename T>
__device__ inline T wave_total(T v) { return wave_all(v, [](T a, T b) { return a + b; }); }
__device__ inline int wave_most(int v) { return wave_all(v, [](int a, int b) { return max(a, b); }); }

// Units of a part.  `slots`: workgroups of a key/value head that two for every CU come to.
// A CU streams keys and values at about 36 GB/s with two workgroups or more, at 27 with one of 16 rows, at 16 with one of more
// rows; 256 CUs together no more than 6.2 TB/s: in units of a CU's 36 GB/s the time is the larger of 1.5 work / 256 and of (workgroups per
// CU, rounded up) x (units of a part).  So their number is kept just below one or two for every CU, in as long parts as that gives; where
// the tiles alone are more, none is longer than the average.
// Decode steps, 8 heads, int8, cut into work / slots units for 512 and for 256 workgroups (a few CUs get one more than the others): four
// requests of 60000..131072 tokens 184, 193 us, this way 157; 32 requests of 200..4096 tokens 40, 37 us, this way 35; four new tokens
// each (32 rows) on four requests of 30000..60000: one workgroup a CU 139 us, two 114.
// Tiles of 128 rows wait for themselves rather than for memory, and their partial results weigh more: they are cut where that is faster by
// times fitted to parts (a unit 1.3 us at D = 64, 1.9 at 128, 3.7 at 256, with what writing the part costs).  Over 120 mixed prompts and chunks 0.8 %
// slower than the better of cutting and not cutting for each, always cutting 1.4 %, never 26 %.
template <int bm, typename COUNT>
__device__ inline float attn_part_units(const KvView &kv, float tiles, float work, float most, int slots, COUNT parts_of_all)
{
    const float least = (float)ATTN_LEAST, half = (float)max(slots / 2, 1);
    auto average = [&](float n) { return fmaxf(work * __builtin_amdgcn_rcpf(n) * 1.00001f, least); };
    const float D = (float)kv.D, unit = fmaxf(1.3f, 0.0145f * D);
    auto tile_time = [&](float units, float n) {                     // us
        const bool one = n <= half;
        return kv.D == 256 ? (one ? 1.0f : 2.0f) * (4 + unit * units) : 4 + unit * (one ? 1.0f : 1.2f) * units;
    };
    float best = bm >= 128 ? most : average((float)slots), best_time = bm >= 128 ? tile_time(most, tiles) : INFINITY;
    for (int r = 1; r <= 2; ++r) {
        const float room = r * half;
        if (tiles > room) continue;
        float c = average(room), n = 0;
        for (int i = 0; i < 6; ++i) {                                // (parts are whole ones: the average gives too many)
            n = (float)parts_of_all(c);
            if (n <= room) break;
            c *= fmaxf(n * __builtin_amdgcn_rcpf(room), 1.04f);
        }
        const float per = fminf(c, most);
        const float time = bm >= 128 ? tile_time(per, n) + 2.5f + 1.2e-4f * D * n * (float)kv.heads
                                     : fmaxf(1.5f * work, (r == 2 ? 2.0f : bm == 16 ? 1.33f : 2.25f) * per * half) + 2 * r * half;
        if (n <= room && time < best_time) best = c, best_time = time;
    }
    return best;
}

__device__ inline int64_t wave_sum_before(int64_t v, int lane)    // inclusive prefix sum over a wavefront
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}
__device__ inline int wave_sum_before(int v, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

struct AttnScratch {
    int64_t part[ATTN_THREADS / 64], tiles[ATTN_THREADS / 64];
    float work[ATTN_THREADS / 64];
    int64_t found[3];
};

// The workgroup's tile (and part): the last of all requests first, as causal tiles get longer towards the end of a request and the longest
// should not start last (with more than 64 requests and parts, the first first); false if there are fewer.
// Up to 64 requests every wavefront finds it by itself, a request per lane; more are shared out over the workgroup.
template <int THREADS, int bm>
__device__ inline bool attn_item(const AttnArgs &a, int slots, bool far_first, int item, AttnScratch &s, AttnItem &out)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int NW = THREADS / 64;
    if (a.requests == 1) {                                   // the same without sums over lanes (one token on 300 7.0 -> 6.6 us, on 8000 14.4 -> 13.6)
        out.r = attn_span(a, 0), out.b = 0, out.parts = 1;
        const int tiles = attn_tiles(out.r, bm), units = attn_tile_units<bm>(a, out.r);
        if (slots) {
            auto count = [&](float c) { return (float)tiles * (float)attn_parts(units, c); };
            out.parts = attn_parts(units, attn_part_units<bm>(a.kv, (float)tiles, (float)tiles * (float)units, (float)units, slots, count));
        }
        const int all = (int)min((int64_t)tiles * out.parts, (int64_t)1 << 24);
        out.item = all - 1 - item;
        out.tile = out.item / out.parts, out.part = out.item % out.parts;
        out.ordinal = out.item >= 0 ? out.tile : tiles + item - all;
        return out.item >= 0;
    }
    if (a.requests <= 64) {
        AttnSpan r = {};
        if (lane < a.requests) r = attn_span(a, lane);
        const int tiles = attn_tiles(r, bm), units = attn_tile_units<bm>(a, r);
        auto of = [&](int v) { return __builtin_amdgcn_readlane(v, out.b); };
        if (bm >= 128 && far_first) {
            // By the last token that they see, counted in tiles, the farthest first: the short ones fill the end.  (Six prompts of
            // 700..1900 tokens, D = 64, window 1024, 1292 workgroups: request after request 56.5 us, this way 51.8; eight prompts of 100..1900,
            // 32 + 8 heads, 173, 164; the search costs, and 60 of 100..500, 4700 workgroups, go from 147 to 151 us.)
            const int from = a.causal ? (int)min((int64_t)max(r.ctx, 0) * a.group / bm, (int64_t)1 << 24) : units;
            auto from_level = [&](int level) { return a.causal ? min(max(from + tiles - level, 0), tiles) : from >= level ? tiles : 0; };
            int level = 0, end = wave_most(from + tiles), before = 0;        // tiles at `end` and beyond: `before`
            if (item >= wave_total(tiles)) return false;
            while (end - level > 1) {
                const int mid = (level + end) / 2, n = wave_total(from_level(mid));
                if (n > item) level = mid;
                else end = mid, before = n;
            }
            const int n = from_level(level) - from_level(level + 1), upto = wave_sum_before(n, lane), want = item - before;
            out.b = __builtin_ctzll(__ballot(want >= upto - n && want < upto));
            out.r = {of(r.cu), of(r.rows), of(r.ctx), of(r.len), of(r.low), of(r.high)};
            out.parts = 1, out.part = 0, out.item = item;
            out.tile = a.causal ? level - of(from) : want - (of(upto) - of(n));
            return true;
        }
        int parts = 1;
        if (slots) {
            const int all = wave_total(tiles);               // (2^24 each at most)
            auto count = [&](float c) { return wave_total((float)tiles * (float)attn_parts(units, c)); };
            const float c = attn_part_units<bm>(a.kv, (float)all, wave_total((float)tiles * (float)units), (float)wave_most(units), slots, count);
            parts = attn_parts(units, c);
        }
        // (at most 2^24 each: more is a cu_new that decreases somewhere)
        const int n = lane < a.requests ? (int)min((int64_t)tiles * parts, (int64_t)1 << 24) : 0;
        const int upto = wave_sum_before(n, lane), tiles_upto = slots ? wave_sum_before(tiles, lane) : 0;
        item = __builtin_amdgcn_readlane(upto, 63) - 1 - item;
        const uint64_t owner = __ballot(item >= 0 && item < upto);
        out.ordinal = __builtin_amdgcn_readlane(tiles_upto, 63) - 1 - item;
        if (!owner) return false;
        out.b = __builtin_ctzll(owner);
        out.r = {of(r.cu), of(r.rows), of(r.ctx), of(r.len), of(r.low), of(r.high)};
        out.parts = of(parts);
        const int k = item - (of(upto) - of(n));
        out.tile = k / out.parts, out.part = k % out.parts, out.item = item;
        out.ordinal = of(tiles_upto) - of(tiles) + out.tile;
        return true;
    }
    int64_t tiles = 0;
    float work = 0;
    for (int b = threadIdx.x; b < a.requests; b += THREADS) {
        const AttnSpan r = attn_span(a, b);
        const int n = attn_tiles(r, bm);
        tiles += n, work += (float)n * (float)attn_tile_units<bm>(a, r);
    }
    tiles = __shfl(wave_sum_before(tiles, lane), 63), work = wave_total(work);
    if (lane == 0) s.part[wave] = tiles, s.work[wave] = work;
    if (threadIdx.x == 0) s.found[0] = -1;
    __syncthreads();
    tiles = 0, work = 0;
#pragma unroll
    for (int w = 0; w < NW; ++w) tiles += s.part[w], work += s.work[w];
    const float c = slots ? fmaxf(work * __builtin_amdgcn_rcpf((float)slots) * 1.00001f, (float)(bm >= 128 ? 4 * ATTN_LEAST : ATTN_LEAST)) : 0.f;   // the average
    int64_t want = item, before = 0, tiles_before = 0;
    if (slots == 0) want = tiles - 1 - item;
    for (int base = 0; base < a.requests && before <= want; base += THREADS) {
        const int b = base + threadIdx.x;
        int64_t n = 0, own = 0;
        int parts = 1;
        if (b < a.requests) {
            const AttnSpan r = attn_span(a, b);
            if (slots) parts = attn_parts(attn_tile_units<bm>(a, r), c);
            own = attn_tiles(r, bm), n = own * parts;
        }
        const int64_t upto = wave_sum_before(n, lane), own_upto = slots ? wave_sum_before(own, lane) : 0;
        __syncthreads();                                     // the sums of the round before have been read
        if (lane == 63) s.part[wave] = upto, s.tiles[wave] = own_upto;
        __syncthreads();
        int64_t at = before + upto - n, tile = tiles_before + own_upto - own;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) at += s.part[w], tile += s.tiles[w];
            before += s.part[w], tiles_before += s.tiles[w];
        }
        if (want >= at && want < at + n) s.found[0] = b, s.found[1] = want - at, s.found[2] = tile;
    }
    __syncthreads();
    out.b = __builtin_amdgcn_readfirstlane((int)s.found[0]);
    out.ordinal = (int)min(tiles + item - before, (int64_t)INT32_MAX);
    if (out.b < 0) return false;
    const int k = __builtin_amdgcn_readfirstlane((int)s.found[1]);
    const AttnSpan r = attn_span(a, out.b);
    auto same = [&](int v) { return __builtin_amdgcn_readfirstlane(v); };
    out.r = {same(r.cu), same(r.rows), same(r.ctx), same(r.len), same(r.low), same(r.high)};
    out.parts = same(slots ? attn_parts(attn_tile_units<bm>(a, r), c) : 1);
    out.tile = k / out.parts, out.part = k % out.parts, out.item = (int)want;
    out.ordinal = __builtin_amdgcn_readfirstlane((int)s.found[2]) + out.tile;
    return true;
}

// Tokens that rows row0 .. row1 - 1 of the request see: [low, high), low a multiple of ATTN_UNIT.
__device__ inline void attn_range(const AttnArgs &a, const AttnSpan &r, int row0, int row1, int &low, int &high)
{
    low = r.low, high = r.high;
    if (a.causal) {
        high = (int)max((int64_t)0, min((int64_t)r.len, (int64_t)r.ctx + attn_token(a, row1 - 1) + 1));
        if (a.window) low = (int)min((int64_t)high, max((int64_t)0, (int64_t)r.ctx + attn_token(a, row0) - a.window + 1)) & -ATTN_UNIT;
    }
}

// Range of a part of [low, high), in whole units.
__device__ inline void attn_part_range(int &low, int &high, int part, int parts)
{
    if (parts == 1) return;
    const int each = (attn_units(low, high) + parts - 1) / parts * ATTN_UNIT, end = high;
    low = (int)min((int64_t)low + (int64_t)part * each, (int64_t)end), high = (int)min((int64_t)low + each, (int64_t)end);
}

// Workspace: for every tile a note of what there is to join, then for every item and key/value head bm rows of D fp32 sums, bm maxima (as the
// kernels keep them: times `factor`, in powers of two) and bm sums of the weights.
struct alignas(16) AttnNote {
    int parts, item;                     // of the tile (0 or 1: nothing to join), the first one's number
    int cu, row0, rows, unused[3];       // first row of q, first row of the tile, rows of the request
};
__host__ __device__ inline size_t attn_partial_floats(int bm, int D) { return (size_t)bm * (D + 2); }
__host__ __device__ inline size_t attn_notes_bytes(int tiles) { return ((size_t)tiles * sizeof(AttnNote) + 255) & ~(size_t)255; }

struct AttnPlan {
    int bm;              // rows of a tile
    int step;            // 1: the kernel for few rows, whose wavefronts share a tile's tokens; 2: requests are short
    int slots;           // see attn_part_units (0: a workgroup per tile, no parts)
    int tiles, items;    // tiles of a key/value head, at most, and workgroups
    int far_first;       // whole tiles in the order of what they see, over all requests: at most eight workgroups for every CU
    size_t ws_bytes;
};
AttnPlan attention_plan(const KvView &kv, int T, int requests, int q_heads, int max_new);

__device__ inline float *attn_partial(const AttnArgs &a, const AttnPlan &p, int64_t item, int kvh)
{
    return reinterpret_cast<float *>(static_cast<char *>(a.ws) + attn_notes_bytes(p.tiles)) + (item * a.kv.heads + kvh) * attn_partial_floats(p.bm, a.kv.D);
}

// Finds the workgroup's item and leaves the note of it.
template <int THREADS, int BM>
__device__ inline bool attn_take(const AttnArgs &a, const AttnPlan &p, int index, int kvh, AttnScratch &s, AttnItem &it)
{
    bool there = attn_item<THREADS, BM>(a, p.slots, p.far_first, index, s, it);
    if (p.slots && there && it.item >= p.items) there = false;       // (a cu_new that decreases: more than the workspace has room for)
    if (p.slots && kvh == 0 && threadIdx.x == 0 && (unsigned)it.ordinal < (unsigned)p.tiles && (!there || it.part == 0))
        static_cast<AttnNote *>(a.ws)[it.ordinal] = there ? AttnNote{it.parts, it.item, it.r.cu, it.tile * BM, it.r.rows, {}} : AttnNote{};
    return there;
}

int launch_attention_steps(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st);
int launch_attention_tiles(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st);

}  // namespace ql
