// What the attention kernels share: which work a workgroup takes, and how parts of a row's tokens are joined.
//
// A row is one new token of one query head.  The G query heads that share a key/value head are rows of one problem: row r of a
// request is token r / G, head r % G of the group, so that keys and values are fetched once for all of them.  A workgroup takes
// a tile of `bm` consecutive rows of one request and key/value head, and all of the tokens that they see, or a part of them.
//
// Lengths are known on the device only (a captured step is replayed with others).  The host launches as many workgroups as the sizes
// that it knows allow for, and each finds its work from the lengths: request b has tiles_b = ceil(new_b G / bm) tiles and
// parts_b = ceil(units_b / C) parts of each (units of 64 tokens), C chosen so that all tiles and heads together have about `target`
// parts: sum tiles_b parts_b <= target + sum tiles_b <= target + floor(T G / bm) + requests.  Without parts (target 0): one per tile.
#pragma once

#include "kv_cache.h"

namespace ql {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr int ATTN_UNIT = 64;            // tokens that tiles of keys are aligned to, and parts of a row's tokens
constexpr int ATTN_THREADS = 256;

struct AttnSpan {                        // a request as the kernels see it
    int cu, rows, ctx, len;              // first row of q, rows (new tokens x heads of the group), position of the first new token, tokens
    int low, high;                       // tokens that any of its rows sees; low is a multiple of ATTN_UNIT
};

struct AttnItem {
    AttnSpan r;
    int b, tile, part, parts;
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

__device__ inline int64_t wave_sum_before(int64_t v, int lane)    // inclusive prefix sum over a wavefront
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

struct AttnScratch {
    int64_t part[ATTN_THREADS / 64];
    int64_t found[3];
};

// exclusive prefix sum over the workgroup's THREADS threads, and its total
template <int THREADS>
__device__ inline int64_t block_sum_before(int64_t v, int64_t *part, int64_t &sum)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t inc = wave_sum_before(v, lane);
    __syncthreads();
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int64_t before = 0;
    sum = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before += part[w];
        sum += part[w];
    }
    return before + inc - v;
}

__device__ inline int attn_tiles(const AttnSpan &r, int bm) { return (r.rows + bm - 1) / bm; }

// units of a part, from the sum over all requests of tiles x units
__device__ inline int attn_part_units(int64_t work, int target)
{
    const int64_t c = target ? (work + target - 1) / target : (int64_t)1 << 30;
    return (int)min(max(c, (int64_t)4), (int64_t)1 << 30);
}
__device__ inline int attn_parts(const AttnSpan &r, int part_units) { return max(1, (attn_units(r.low, r.high) + part_units - 1) / part_units); }

template <int THREADS>
__device__ inline int64_t attn_work(const AttnArgs &a, int bm, int64_t *part, int64_t &tiles)
{
    int64_t work = 0, n = 0, sum;
    for (int b = threadIdx.x; b < a.requests; b += THREADS) {
        const AttnSpan r = attn_span(a, b);
        n += attn_tiles(r, bm);
        work += (int64_t)attn_tiles(r, bm) * attn_units(r.low, r.high);
    }
    block_sum_before<THREADS>(n, part, tiles);
    block_sum_before<THREADS>(work, part, sum);
    return sum;
}

// The item-th tile (and part) of all requests; false if there are fewer.  Without parts the last tile of the last request comes first:
// causal tiles get longer towards the end of a request, and the longest should not start last.
template <int THREADS>
__device__ inline bool attn_item(const AttnArgs &a, int bm, int target, int64_t item, AttnScratch &s, AttnItem &out)
{
    int64_t tiles;
    const int64_t work = attn_work<THREADS>(a, bm, s.part, tiles);
    const int c = attn_part_units(work, target);
    if (target == 0) {
        if (item >= tiles) return false;
        item = tiles - 1 - item;
    }
    if (threadIdx.x == 0) s.found[0] = -1;
    int64_t before = 0;
    for (int base = 0; base < a.requests && before <= item; base += THREADS) {
        const int b = base + threadIdx.x;
        int64_t n = 0, sum;
        if (b < a.requests) {
            const AttnSpan r = attn_span(a, b);
            n = (int64_t)attn_tiles(r, bm) * (target ? attn_parts(r, c) : 1);
        }
        const int64_t at = before + block_sum_before<THREADS>(n, s.part, sum);
        if (item >= at && item < at + n) s.found[0] = b, s.found[1] = item - at;
        before += sum;
    }
    __syncthreads();
    out.b = __builtin_amdgcn_readfirstlane((int)s.found[0]);
    if (out.b < 0) return false;
    const int k = __builtin_amdgcn_readfirstlane((int)s.found[1]);
    out.r = attn_span(a, out.b);
    out.r.cu = __builtin_amdgcn_readfirstlane(out.r.cu), out.r.rows = __builtin_amdgcn_readfirstlane(out.r.rows);
    out.r.ctx = __builtin_amdgcn_readfirstlane(out.r.ctx), out.r.len = __builtin_amdgcn_readfirstlane(out.r.len);
    out.r.low = __builtin_amdgcn_readfirstlane(out.r.low), out.r.high = __builtin_amdgcn_readfirstlane(out.r.high);
    out.parts = __builtin_amdgcn_readfirstlane(target ? attn_parts(out.r, c) : 1);
    out.tile = k / out.parts, out.part = k % out.parts;
    return true;
}

// Tokens that rows row0 .. row1 - 1 of the request see: [low, high), low a multiple of ATTN_UNIT.
__device__ inline void attn_range(const AttnArgs &a, const AttnSpan &r, int row0, int row1, int &low, int &high)
{
    low = r.low, high = r.high;
    if (a.causal) {
        high = (int)max((int64_t)0, min((int64_t)r.len, (int64_t)r.ctx + (row1 - 1) / a.group + 1));
        if (a.window) low = (int)min((int64_t)high, max((int64_t)0, (int64_t)r.ctx + row0 / a.group - a.window + 1)) & -ATTN_UNIT;
    }
}

// Range of a part of [low, high), in whole units.
__device__ inline void attn_part_range(int &low, int &high, int part, int parts)
{
    const int u = attn_units(low, high), l0 = low;
    low = l0 + (int)((int64_t)u * part / parts) * ATTN_UNIT;
    high = min(high, l0 + (int)((int64_t)u * (part + 1) / parts) * ATTN_UNIT);
}

// Workspace: for every item a note of what there is to join (int4: parts, or 0 where this item is not the first of several; first row
// of q, first row of the tile, rows of the request), then for every item and key/value head bm rows of D fp32 sums, bm maxima (in powers
// of two) and bm sums of the weights.
__host__ __device__ inline size_t attn_partial_floats(int bm, int D) { return (size_t)bm * (D + 2); }
__host__ __device__ inline size_t attn_notes_bytes(int items) { return ((size_t)items * 16 + 255) & ~(size_t)255; }

struct AttnPlan {
    int bm;              // rows of a tile
    int step;            // 1: the kernel for few rows, whose wavefronts share a tile's tokens
    int target;          // parts that all tiles of a key/value head together are cut into (0: none)
    int items;           // workgroups of a key/value head
    size_t ws_bytes;
};
AttnPlan attention_plan(const KvView &kv, int T, int requests, int q_heads, int max_new);

__device__ inline float *attn_partial(const AttnArgs &a, const AttnPlan &p, int64_t item, int kvh)
{
    return reinterpret_cast<float *>(static_cast<char *>(a.ws) + attn_notes_bytes(p.items)) + (item * a.kv.heads + kvh) * attn_partial_floats(p.bm, a.kv.D);
}

// Finds the workgroup's item and leaves the note of it.
template <int THREADS>
__device__ inline bool attn_take(const AttnArgs &a, const AttnPlan &p, int64_t index, int kvh, AttnScratch &s, AttnItem &it)
{
    const bool there = attn_item<THREADS>(a, p.bm, p.target, index, s, it);
    if (p.target && kvh == 0 && threadIdx.x == 0)
        static_cast<int4 *>(a.ws)[index] = there && it.part == 0 && it.parts > 1 ? make_int4(it.parts, it.r.cu, it.tile * p.bm, it.r.rows) : make_int4(0, 0, 0, 0);
    return there;
}

int launch_attention_steps(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st);
int launch_attention_tiles(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st);

}  // namespace ql
