// Bookkeeping of the paged key/value cache, and what writes and reads it (layout: include/qlinear.h, kv_cache.h).
#include <type_traits>

#include "kv_cache.h"
#include "quant_math.h"

namespace ql {
namespace {

// ---- lengths -> pages, slots, positions ------------------------------------------------------------------------
// With n_b = new tokens, T_b = take_b pages, R_b = give_b pages of request b, everything follows from three prefix sums over the
// requests: row t belongs to the request whose range of cu holds it, the i-th page taken is ring[head + i], the i-th given
// back goes to ring[head + free + i].  No step waits for another, so one launch does it: every workgroup forms the sums itself (at most
// 4096 requests, from the caches), and every thread takes a token, a page taken or a page given back.  The places of the ring that a call
// reads and those that it writes are different ones, entries of the table that are looked up for tokens are not those that are written;
// only the pool's state is read by all and written at the end, where it is updated in place by the workgroup that finishes last.
// Bound by latency: lengths -> sums -> search in them -> table or ring.  1024 requests, 27000 tokens: 6.9 us (tokens, pages taken and
// pages given back one after the other in a thread: 11.2); 64 requests of a decode step: 4.8.
constexpr int RESIZE_THREADS = 256;
constexpr int RESIZE_MOST = 4096;

struct Sums {
    int64_t tokens, pages;                                    // pages taken, pages given << 32 (each sum below 2^31)
};

// exclusive prefix sums over the workgroup's threads, and the totals
__device__ inline Sums sums_before(Sums v, Sums *part, Sums &all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums inc = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t t = __shfl_up(inc.tokens, d), p = __shfl_up(inc.pages, d);
        if (lane >= d) inc.tokens += t, inc.pages += p;
    }
    __syncthreads();                                          // (of an earlier use of `part`)
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    Sums before = {inc.tokens - v.tokens, inc.pages - v.pages};
    all = {0, 0};
#pragma unroll
    for (int w = 0; w < RESIZE_THREADS / 64; ++w) {
        if (w < wave) before.tokens += part[w].tokens, before.pages += part[w].pages;
        all.tokens += part[w].tokens, all.pages += part[w].pages;
    }
    return before;
}

// the request whose range of the prefix sums holds i: the last b with sums[b] <= i (sums[n] > i, so ranges of length 0 are passed over)
__device__ inline int request_of(const int *sums, int n, int i)
{
    int lo = 0, hi = n;                                       // sums[lo] <= i < sums[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (sums[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

struct ResizeArgs {
    const int32_t *old_len, *want_len;
    int32_t *ring;
    const int32_t *pool;
    int32_t *pool_out, *table;
    int64_t ld_table;
    int32_t *kv_len, *cu_new, *slots, *positions;
    int requests, page_shift, pages, columns, max_tokens;
};

// PER: requests of a thread
template <int PER>
__global__ __launch_bounds__(RESIZE_THREADS) void kv_resize_kernel(ResizeArgs a)
{
    constexpr int MOST = PER * RESIZE_THREADS;
    __shared__ int cu[MOST + 1], takes[MOST + 1], gives[MOST + 1];
    __shared__ Sums part[RESIZE_THREADS / 64];
    __shared__ int64_t losses[RESIZE_THREADS / 64];
    const int tid = threadIdx.x, B = a.requests, page = 1 << a.page_shift, cap = a.columns << a.page_shift, pages = a.pages;
    const int first = tid * PER;

    int old_[PER], want[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) old_[i] = first + i < B ? a.old_len[first + i] : 0, want[i] = first + i < B ? a.want_len[first + i] : 0;
    int head = a.pool[0] % pages, free = a.pool[1];
    head = head < 0 ? head + pages : head;
    free = min(max(free, 0), pages);

    auto pages_of = [&](int len) { return (int)(((int64_t)len + page - 1) >> a.page_shift); };
    auto clip_old = [&](int len) { return min(max(len, 0), cap); };
    // the length that a request would have with pages for all of it; pages that it takes or gives
    auto target = [&](int o, int w, int n) { return w < o ? w : (int)min((int64_t)o + n, (int64_t)cap); };
    auto moved = [&](int o, int t) -> int64_t {
        const int d = pages_of(t) - pages_of(o);
        return d > 0 ? (int64_t)d : (int64_t)-d << 32;
    };
    Sums mine = {0, 0}, all;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int o = clip_old(old_[i]), w = max(want[i], 0);
        old_[i] = o, want[i] = w;
        mine.tokens += max(0, w - o), mine.pages += moved(o, target(o, w, max(0, w - o)));
    }
    Sums before = sums_before(mine, part, all);
    const bool fits = all.tokens <= a.max_tokens;
    auto clipped = [&](int64_t t) { return (int)min(t, (int64_t)a.max_tokens); };
    if (!fits) {                                              // fewer tokens than wanted: the pages once more
        int64_t t = before.tokens;
        mine.pages = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int n = max(0, want[i] - old_[i]);
            mine.pages += moved(old_[i], target(old_[i], want[i], clipped(t + n) - clipped(t)));
            t += n;
        }
        Sums ignored;
        before.pages = sums_before({0, mine.pages}, part, ignored).pages;
        all.pages = ignored.pages;
    }
    int64_t lost = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int b = first + i, o = old_[i], w = want[i], from = clipped(before.tokens), n = clipped(before.tokens + max(0, w - o)) - from;
        const int t = target(o, w, n), has = pages_of(o), taken = (int)(before.pages & 0xffffffff), d = pages_of(t) - has;
        const int got = d > 0 ? min(max(free - taken, 0), d) : 0;
        const int len = w < o ? w : (int)min((int64_t)t, (int64_t)(has + got) << a.page_shift);
        if (b <= B) cu[b] = from, takes[b] = taken, gives[b] = (int)(before.pages >> 32);
        if (b < B) {
            if (w >= o) lost += (int64_t)w - len;              // (for want of a page, a column of the table or a row of the step)
            if (blockIdx.x == 0) a.kv_len[b] = len, a.cu_new[b] = from;
        }
        before.tokens += max(0, w - o), before.pages += moved(o, t);
    }
    if (tid == RESIZE_THREADS - 1 && B == MOST) cu[B] = clipped(all.tokens), takes[B] = (int)(all.pages & 0xffffffff), gives[B] = (int)(all.pages >> 32);
    if (blockIdx.x == 0 && tid == 0) a.cu_new[B] = clipped(all.tokens);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) lost += __shfl_xor(lost, d);
    if ((tid & 63) == 0) losses[tid >> 6] = lost;
    __syncthreads();

    const int tokens = cu[B], taken = min(takes[B], free), given = min(gives[B], pages - free);   // (a pool that is in order has room for all of them)
    auto ring_at = [&](int64_t i) { return a.ring + (head + i) % pages; };
    const int64_t items = (int64_t)tokens + taken + given;
    for (int64_t at = blockIdx.x * RESIZE_THREADS + tid; at < items; at += gridDim.x * RESIZE_THREADS) {
        const bool is_token = at < tokens, is_take = !is_token && at < (int64_t)tokens + taken;
        const int i = (int)(is_token ? at : is_take ? at - tokens : at - tokens - taken);
        const int *sums = is_token ? cu : is_take ? takes : gives;
        const int b = request_of(sums, B, i), k = i - sums[b];
        int32_t *row = a.table + b * a.ld_table;
        if (is_token) {
            const int o = clip_old(a.old_len[b]), has = pages_of(o);
            const int64_t pos = (int64_t)o + k, j = pos >> a.page_shift;
            int p = -1;
            if (j < has) p = row[j];
            else if (pos < cap && takes[b] + j - has < free) p = *ring_at(takes[b] + j - has);
            a.slots[i] = p >= 0 && p < pages ? (p << a.page_shift) + (int)(pos & (page - 1)) : -1;
            a.positions[i] = (int)min(pos, (int64_t)INT32_MAX);
        } else if (is_take) {
            row[pages_of(clip_old(a.old_len[b])) + k] = *ring_at(i);
        } else {
            *ring_at((int64_t)free + i) = row[pages_of(max(a.want_len[b], 0)) + k];
        }
    }

    if (a.pool_out == a.pool && gridDim.x > 1) {              // all have read the pool's state once the last one arrives
        __shared__ int arrived;
        __syncthreads();
        if (tid == 0) arrived = __hip_atomic_fetch_add(a.pool_out + 3, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (int)gridDim.x - 1) return;
    } else if (blockIdx.x != 0) {
        return;
    }
    if (tid == 0) {
        int64_t sum = 0;
#pragma unroll
        for (int w = 0; w < RESIZE_THREADS / 64; ++w) sum += losses[w];
        a.pool_out[0] = (int)(((int64_t)head + taken) % pages);
        a.pool_out[1] = free - taken + given;
        a.pool_out[2] = (int)min(sum, (int64_t)INT32_MAX);
        __hip_atomic_store(a.pool_out + 3, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// ---- rows into the cache, and back -----------------------------------------------------------------------------
// Bound by memory: rows of 2 D bytes are read, blocks written (read back: the other way round).  A workgroup takes about 32 consecutive rows of one
// key/value head, 16 channels per thread: the rows and the keys' pieces are 16 bytes per lane on both sides.  Values lie transposed in
// a block: they go through LDS, and leave (arrive) 16 bytes at a time where the rows fill the piece of a channel -- 8 tokens in fp16, 16 in
// int8 --, else by groups of 4 tokens, else singly: a decode step's tokens are single ones, a prompt's rows have them at its ends only.
// 4096 tokens, 32 + 2 x 32 heads of 128, fp16, and 16001 tokens, 32 + 2 x 8 heads, int8; append / read back: 48 / 25 us and 78 / 28 us, 4.5 TB/s and more
// of 5.1 that a large copy reaches (with windows of 32 rows whatever their slots, pieces cut at the windows' ends: 57 / 37, 86 / 40).

__device__ inline bool finite(float x) { return __builtin_fabsf(x) <= 3.402823466e38f; }

// the D / 16 lanes that hold a token
template <int LANES, typename OP>
__device__ inline float over_lanes(float v, OP op)
{
    auto step = [&](auto off) {
        unsigned a, b;
        lane_pair<decltype(off)::value>(__builtin_bit_cast(unsigned, v), a, b);
        v = op(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
    };
    step(std::integral_constant<int, 1>{}), step(std::integral_constant<int, 2>{});
    if constexpr (LANES >= 8) step(std::integral_constant<int, 4>{});
    if constexpr (LANES >= 16) step(std::integral_constant<int, 8>{});
    return v;
}

// The rows of a workgroup.  Consecutive slots of one block are a run; a workgroup takes the runs that begin in its window of TILE rows,
// with what of the last one lies behind the window: so that blocks are written whole wherever the rows hold them whole, whatever place
// in the batch a request's rows have.  Every wavefront finds them by itself, a row per lane.
struct Rows {
    uint64_t cont;                                        // rows that continue the row before
    int slot, first, n;                                   // slot of this lane's row (-1: none); rows [first, first + n) from t0
};
template <int TILE>
__device__ inline Rows find_rows(const int32_t *slots, int t0, int T, const KvView &kv)
{
    static_assert(TILE + KV_BLOCK <= 64, "a row per lane");
    const int lane = threadIdx.x & 63;
    auto slot_of = [&](int t) {
        const int s = t >= 0 && t < T ? slots[t] : -1;
        return (unsigned)s < (unsigned)kv.pages << kv.page_shift ? s : -1;
    };
    Rows r;
    r.slot = slot_of(t0 + lane);
    const int before = slot_of(t0 + lane - 1);
    const bool cont = r.slot >= 0 && before >= 0 && r.slot == before + 1 && r.slot % KV_BLOCK != 0;
    r.cont = __ballot(cont);
    const uint64_t begins = __ballot(t0 + lane < T && !cont) & ((1ull << TILE) - 1);   // (a row without a slot is a run of its own)
    r.first = r.n = 0;
    if (begins) {
        const int last = 63 - __builtin_clzll(begins);
        r.first = __builtin_ctzll(begins);
        r.n = last + 1 + __builtin_ctzll(~(r.cont >> last >> 1)) - r.first;
    }
    return r;
}

// What to move of the rows' values, {row from `first`, kind}: whole pieces of a channel (fp16: tokens 4 h .. and 8 + 4 h .. of 16; int8:
// four such groups of 32), groups of 4 tokens, single ones.
enum { ONE = 1, FOUR = 2, WHOLE = 3 };
struct Pieces {
    int slot[64];                                         // by row from `first`
    int count, row[64], kind[64];
};
template <int ELEM>
__device__ inline void find_pieces(Pieces &p, const Rows &r)          // by one wavefront
{
    const int lane = threadIdx.x & 63, s = r.slot;
    auto follow = [&](int row, int n) { return ((r.cont >> row >> 1) & ((1ull << n) - 1)) == (1ull << n) - 1; };   // rows + 1 .. + n continue
    constexpr int REST = ELEM == 2 ? 11 : 27, SPAN = ELEM == 2 ? 16 : 32;
    const bool mine = lane >= r.first && lane < r.first + r.n && s >= 0;
    const bool four = s % 4 == 0 && follow(lane, 3), whole = four && s % SPAN < 8 && follow(lane, REST);
    const int in4 = s & 3, up = s & (SPAN - 8);                        // rows down to the group's, to the piece's first one
    const bool inside = in4 && lane >= in4 && follow(lane - in4, 3);
    const bool inside_whole = four && up && lane >= up && follow(lane - up, REST);
    const int kind = !mine || inside || inside_whole ? 0 : whole ? WHOLE : four ? FOUR : ONE;
    const uint64_t have = __ballot(kind != 0);
    if (kind) {
        const int n = __popcll(have & ((1ull << lane) - 1));
        p.row[n] = lane - r.first, p.kind[n] = kind;
    }
    if (lane >= r.first && lane < r.first + r.n) p.slot[lane - r.first] = s;
    if (lane == 0) p.count = __popcll(have);
}

// Rotation of 16 channels of a row: the thread's two runs of 8, (8 j, 8 j + half) among the channels that are turned, neighbours among
// the others.
struct Turn {
    int c0, c1;
    bool turned;
    __device__ Turn(int j, int rotary) : c0(8 * j), c1(8 * j + rotary / 2), turned(8 * j < rotary / 2)
    {
        if (!turned) c0 = rotary + 16 * (j - rotary / 16), c1 = c0 + 8;
    }
};
__device__ inline void widen8(const uint4 &v, float (&f)[8])
{
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = half_bits_to_float(w[i] & 0xffffu), f[2 * i + 1] = half_bits_to_float(w[i] >> 16);
}
__device__ inline uint4 narrow8(const float (&f)[8])
{
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(unsigned, h2{(_Float16)f[2 * i], (_Float16)f[2 * i + 1]});
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ inline void rotate(const Turn &u, const float *row, int rotary, float (&a)[8], float (&b)[8])
{
    if (!u.turned) return;
    const float4 c0 = *reinterpret_cast<const float4 *>(row + u.c0), c1 = *reinterpret_cast<const float4 *>(row + u.c0 + 4);
    const float4 s0 = *reinterpret_cast<const float4 *>(row + rotary / 2 + u.c0), s1 = *reinterpret_cast<const float4 *>(row + rotary / 2 + u.c0 + 4);
    const float co[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, si[8] = {s0.x, s0.y, s0.z, s0.w, s1.x, s1.y, s1.z, s1.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {                         // (no contraction: each product and each sum is rounded)
        const float x = a[i], y = b[i];
        a[i] = x * co[i] - y * si[i];
        b[i] = y * co[i] + x * si[i];
    }
}
__device__ inline uint2 codes8(const float (&f)[8], float inv, bool some)
{
    unsigned w[2] = {0x80808080u, 0x80808080u};           // codes are stored plus 128
    if (some) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int q = (int)fminf(fmaxf(rintf(f[i] * inv), -127.f), 127.f);
            w[i / 4] ^= (unsigned)(q & 255) << (8 * (i % 4));   // q + 128 = q ^ 128 in a byte
        }
    }
    return make_uint2(w[0], w[1]);
}

__device__ inline uint4 kept(const uint4 &v, bool keep, unsigned other) { return make_uint4(keep ? v.x : other, keep ? v.y : other, keep ? v.z : other, keep ? v.w : other); }

struct AppendArgs {
    const __half *q, *k, *v;
    int64_t ldq, ldk, ldv, ldqo;
    __half *q_out;
    const float *cos_sin;
    const int32_t *positions, *slots;
    int T, q_heads, rotary, max_positions, kv_groups;     // kv_groups: workgroups of keys and values (the first ones of the grid)
    KvView kv;
};

template <int ELEM, int D, int TILE>
__global__ __launch_bounds__(2 * D) void kv_append_kernel(AppendArgs a)
{
    constexpr int LANES = D / 16, ROW = ELEM * D + 16, MOST = TILE + KV_BLOCK - 1;   // lanes of a token; bytes of a row in LDS; rows
    const int tid = threadIdx.x;
    auto table_row = [&](int t) { return a.cos_sin + (int64_t)min(max(a.positions[t], 0), a.max_positions - 1) * a.rotary; };

    if ((int)blockIdx.x >= a.kv_groups) {                 // queries: 32 (token, head) pairs
        const unsigned pair = (blockIdx.x - (unsigned)a.kv_groups) * 32u + tid / LANES, t = pair / (unsigned)a.q_heads, head = pair - t * (unsigned)a.q_heads;
        if (t >= (unsigned)a.T) return;
        const Turn u(tid % LANES, a.rotary);
        const __half *src = a.q + t * a.ldq + (int64_t)head * D;
        __half *dst = a.q_out + t * a.ldqo + (int64_t)head * D;
        uint4 lo = *reinterpret_cast<const uint4 *>(src + u.c0), hi = *reinterpret_cast<const uint4 *>(src + u.c1);
        if (u.turned) {
            float x[8], y[8];
            widen8(lo, x), widen8(hi, y);
            rotate(u, table_row(t), a.rotary, x, y);
            lo = narrow8(x), hi = narrow8(y);
        }
        *reinterpret_cast<uint4 *>(dst + u.c0) = lo;
        *reinterpret_cast<uint4 *>(dst + u.c1) = hi;
        return;
    }

    __shared__ Pieces p;
    __shared__ __attribute__((aligned(16))) char values[MOST * ROW];
    const int head = blockIdx.x % a.kv.heads, t0 = blockIdx.x / a.kv.heads * TILE;
    const Rows rows = find_rows<TILE>(a.slots, t0, a.T, a.kv);
    if (tid < 64) find_pieces<ELEM>(p, rows);
    const int j = tid % LANES;
    const Turn u(j, a.rotary);
    for (int r = tid / LANES; r < rows.n; r += 32) {
        const int t = t0 + rows.first + r, slot = a.slots[t];
        const bool stored = (unsigned)slot < (unsigned)a.kv.pages << a.kv.page_shift;
        const __half *ks = a.k + t * a.ldk + (int64_t)head * D, *vs = a.v + t * a.ldv + (int64_t)head * D + 16 * j;
        const uint4 k0 = *reinterpret_cast<const uint4 *>(ks + u.c0), k1 = *reinterpret_cast<const uint4 *>(ks + u.c1);
        const uint4 v0 = *reinterpret_cast<const uint4 *>(vs), v1 = *reinterpret_cast<const uint4 *>(vs + 8);
        float x[8], y[8], z[8], w[8];
        widen8(k0, x), widen8(k1, y), widen8(v0, z), widen8(v1, w);
        if (a.rotary) rotate(u, table_row(t), a.rotary, x, y);
        uint4 kh0, kh1;
        if (ELEM == 2) {
            kh0 = narrow8(x), kh1 = narrow8(y);
            widen8(kh0, x), widen8(kh1, y);
        }
        float kmax = 0, vmax = 0, off = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (!(finite(x[i]) && finite(y[i]) && finite(z[i]) && finite(w[i]))) off = 1;
            kmax = fmaxf(kmax, fmaxf(__builtin_fabsf(x[i]), __builtin_fabsf(y[i]))), vmax = fmaxf(vmax, fmaxf(__builtin_fabsf(z[i]), __builtin_fabsf(w[i])));
        }
        auto most = [](float a, float b) { return fmaxf(a, b); };
        const bool fine = over_lanes<LANES>(off, most) == 0;
        const int rest = slot & (a.kv.page_size() - 1), token = rest % KV_BLOCK;
        char *block = stored ? a.kv.block(slot >> a.kv.page_shift, head, rest) : nullptr, *vr = values + r * ROW + 16 * j * ELEM;
        if constexpr (ELEM == 2) {
            if (stored) {
                *reinterpret_cast<uint4 *>(block + kv_key_offset<2>(token, u.c0)) = kept(kh0, fine, 0x7e007e00u);
                *reinterpret_cast<uint4 *>(block + kv_key_offset<2>(token, u.c1)) = kept(kh1, fine, 0x7e007e00u);
            }
            *reinterpret_cast<uint4 *>(vr) = kept(v0, fine, 0);
            *reinterpret_cast<uint4 *>(vr + 16) = kept(v1, fine, 0);
        } else {
            kmax = over_lanes<LANES>(kmax, most), vmax = over_lanes<LANES>(vmax, most);
            const bool some_k = fine && kmax >= KV_NOTHING, some_v = fine && vmax >= KV_NOTHING;
            const float inv_k = 127.0f / kmax, inv_v = 127.0f / vmax;
            if (stored) {
                *reinterpret_cast<uint2 *>(block + kv_key_offset<1>(token, u.c0)) = codes8(x, inv_k, some_k);
                *reinterpret_cast<uint2 *>(block + kv_key_offset<1>(token, u.c1)) = codes8(y, inv_k, some_k);
                if (j < 4) {
                    const float sk = !fine ? __builtin_nanf("") : some_k ? kmax / 127.0f : 0x1p-31f, sv = some_v ? vmax / 127.0f : 0x1p-31f;
                    const float out = j == 0 ? sk : j == 1 ? sv : j == 2 ? log2f(sv) : 1.0f / sv;
                    reinterpret_cast<float *>(block + kv_scale_offset(D))[j * KV_BLOCK + token] = out;
                }
            }
            const uint2 c0 = codes8(z, inv_v, some_v), c1 = codes8(w, inv_v, some_v);
            *reinterpret_cast<uint4 *>(vr) = make_uint4(c0.x, c0.y, c1.x, c1.y);
        }
    }
    __syncthreads();
    const int c = tid % D;                                // values: a channel per thread, every second piece
    for (int i = tid / D; i < p.count; i += 2) {
        const int row = p.row[i], kind = p.kind[i], s = p.slot[row], in_page = s & (a.kv.page_size() - 1);
        char *to = a.kv.block(s >> a.kv.page_shift, head, in_page) + kv_value_offset<ELEM>(in_page % KV_BLOCK, c, D);
        if constexpr (ELEM == 2) {
            auto two = [&](int k) {
                const char *from = values + (row + k) * ROW + 2 * c;
                return (unsigned)*reinterpret_cast<const uint16_t *>(from) | (unsigned)*reinterpret_cast<const uint16_t *>(from + ROW) << 16;
            };
            if (kind == WHOLE) *reinterpret_cast<uint4 *>(to) = make_uint4(two(0), two(2), two(8), two(10));
            else if (kind == FOUR) *reinterpret_cast<uint2 *>(to) = make_uint2(two(0), two(2));
            else *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(values + row * ROW + 2 * c);
        } else {
            auto four = [&](int k) {
                const uint8_t *from = reinterpret_cast<const uint8_t *>(values) + (row + k) * ROW + c;
                return (unsigned)from[0] | (unsigned)from[ROW] << 8 | (unsigned)from[2 * ROW] << 16 | (unsigned)from[3 * ROW] << 24;
            };
            if (kind == WHOLE) *reinterpret_cast<uint4 *>(to) = make_uint4(four(0), four(8), four(16), four(24));
            else if (kind == FOUR) *reinterpret_cast<unsigned *>(to) = four(0);
            else *reinterpret_cast<uint8_t *>(to) = *(reinterpret_cast<const uint8_t *>(values) + row * ROW + c);
        }
    }
}

template <int ELEM, int D, int TILE>
__global__ __launch_bounds__(2 * D) void kv_read_kernel(KvView kv, const int32_t *__restrict__ slots, int T, __half *__restrict__ k, int64_t ldk,
                                                        __half *__restrict__ v, int64_t ldv)
{
    constexpr int LANES = D / 16, ROW = ELEM * D + 16, MOST = TILE + KV_BLOCK - 1;
    __shared__ Pieces p;
    __shared__ __attribute__((aligned(16))) char values[MOST * ROW];
    const int tid = threadIdx.x, head = blockIdx.x % kv.heads, t0 = blockIdx.x / kv.heads * TILE;
    const Rows rows = find_rows<TILE>(slots, t0, T, kv);
    if (tid < 64) find_pieces<ELEM>(p, rows);
    __syncthreads();
    auto scale_of = [&](const char *block, int token, int which) { return reinterpret_cast<const float *>(block + kv_scale_offset(D))[which * KV_BLOCK + token]; };
    float first_scale = 0;                                // of the values of this thread's first row: under way with them
    if (ELEM == 1 && v && tid / LANES < rows.n) {
        const int slot = p.slot[tid / LANES], rest = slot & (kv.page_size() - 1);
        if (slot >= 0) first_scale = scale_of(kv.block(slot >> kv.page_shift, head, rest), rest % KV_BLOCK, 1);
    }
    const int c = tid % D;
    if (v) {
        const int count = p.count;
        for (int i0 = tid / D; i0 < count; i0 += 8) {     // four pieces on their way at a time
            uint4 got[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int i = i0 + 2 * n;
                if (i >= count) continue;
                const int kind = p.kind[i], s = p.slot[p.row[i]], in_page = s & (kv.page_size() - 1);
                const char *from = kv.block(s >> kv.page_shift, head, in_page) + kv_value_offset<ELEM>(in_page % KV_BLOCK, c, D);
                if (kind == WHOLE) got[n] = *reinterpret_cast<const uint4 *>(from);
                else if (kind == FOUR && ELEM == 2) got[n].x = *reinterpret_cast<const unsigned *>(from), got[n].y = *reinterpret_cast<const unsigned *>(from + 4);
                else if (kind == FOUR) got[n].x = *reinterpret_cast<const unsigned *>(from);
                else got[n].x = ELEM == 2 ? *reinterpret_cast<const uint16_t *>(from) : *reinterpret_cast<const uint8_t *>(from);
            }
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const int i = i0 + 2 * n;
                if (i >= count) continue;
                const int kind = p.kind[i];
                char *to = values + p.row[i] * ROW + c * ELEM;
                if constexpr (ELEM == 2) {
                    auto put = [&](int k, unsigned w) { *reinterpret_cast<uint16_t *>(to + k * ROW) = (uint16_t)w, *reinterpret_cast<uint16_t *>(to + (k + 1) * ROW) = (uint16_t)(w >> 16); };
                    if (kind == ONE) *reinterpret_cast<uint16_t *>(to) = (uint16_t)got[n].x;
                    else put(0, got[n].x), put(2, got[n].y);
                    if (kind == WHOLE) put(8, got[n].z), put(10, got[n].w);
                } else {
                    auto put = [&](int k, unsigned w) {
#pragma unroll
                        for (int b = 0; b < 4; ++b) *reinterpret_cast<uint8_t *>(to + (k + b) * ROW) = (uint8_t)(w >> (8 * b));
                    };
                    if (kind == ONE) *reinterpret_cast<uint8_t *>(to) = (uint8_t)got[n].x;
                    else put(0, got[n].x);
                    if (kind == WHOLE) put(8, got[n].y), put(16, got[n].z), put(24, got[n].w);
                }
            }
        }
    }
    // 16 channels of a row
    auto store = [&](__half *to, bool there, const char *from, int second, float scale) {
        uint4 a = make_uint4(0, 0, 0, 0), b = a;
        if (there) {
            const uint4 w = *reinterpret_cast<const uint4 *>(from);
            if constexpr (ELEM == 2) {
                a = w, b = *reinterpret_cast<const uint4 *>(from + second);
            } else {
                const unsigned x[4] = {w.x, w.y, w.z, w.w};
                float lo[8], hi[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    lo[i] = (float)((int)(x[i / 4] >> (8 * (i % 4)) & 255u) - 128) * scale;
                    hi[i] = (float)((int)(x[2 + i / 4] >> (8 * (i % 4)) & 255u) - 128) * scale;
                }
                a = narrow8(lo), b = narrow8(hi);
            }
        }
        *reinterpret_cast<uint4 *>(to) = a, *reinterpret_cast<uint4 *>(to + 8) = b;
    };
    const int j = tid % LANES;
    auto each_row = [&](auto f) {
        for (int r = tid / LANES; r < rows.n; r += 32) {
            const int slot = p.slot[r], rest = slot & (kv.page_size() - 1);
            const char *block = slot < 0 ? kv.base : kv.block(slot >> kv.page_shift, head, rest);
            f(r, slot >= 0, block, rest % KV_BLOCK, t0 + rows.first + r);
        }
    };
    const int64_t column = (int64_t)head * D + 16 * j;
    if (k)
        each_row([&](int, bool there, const char *block, int token, int t) {
            const float scale = ELEM == 1 && there ? scale_of(block, token, 0) : 0.f;
            store(k + t * ldk + column, there, block + kv_key_offset<ELEM>(token, 16 * j), 512, scale);
        });
    if (v) {
        __syncthreads();
        each_row([&](int r, bool there, const char *block, int token, int t) {
            const float scale = ELEM == 1 && there ? (r < 32 ? first_scale : scale_of(block, token, 1)) : 0.f;
            store(v + t * ldv + column, there, values + r * ROW + 16 * j * ELEM, 16, scale);
        });
    }
}

__global__ void kv_no_requests_kernel(const int32_t *pool, int32_t *pool_out, int32_t *cu_new)
{
    const int i = threadIdx.x;
    const int x = i < 2 ? pool[i] : 0;
    if (i < 3) pool_out[i] = x;
    if (i == 3) cu_new[0] = 0;
}

}  // namespace

int launch_kv_resize(const int32_t *old_len, const int32_t *want_len, int requests, int page_shift, int32_t *ring, int pages,
                     const int32_t *pool, int32_t *pool_out, int32_t *table, int64_t ld_table, int columns, int32_t *kv_len,
                     int32_t *cu_new, int32_t *slots, int32_t *positions, int max_tokens, hipStream_t st)
{
    if (requests == 0) {
        kv_no_requests_kernel<<<1, 64, 0, st>>>(pool, pool_out, cu_new);
        return check_hip(hipGetLastError(), "kv_no_requests_kernel");
    }
    const ResizeArgs a = {old_len, want_len, ring, pool, pool_out, table, ld_table, kv_len, cu_new, slots, positions, requests, page_shift, pages, columns, max_tokens};
    const int grid = (int)min((int64_t)512, 1 + ((int64_t)max_tokens + 2 * (int64_t)requests) / RESIZE_THREADS);
    // requests of a thread: as few as hold them (64 requests 4.8 us with 1, 9.9 with 16; 1024 requests 5.9 with 4, 10.9 with 16)
    if (requests <= RESIZE_THREADS) kv_resize_kernel<1><<<grid, RESIZE_THREADS, 0, st>>>(a);
    else if (requests <= 4 * RESIZE_THREADS) kv_resize_kernel<4><<<grid, RESIZE_THREADS, 0, st>>>(a);
    else kv_resize_kernel<RESIZE_MOST / RESIZE_THREADS><<<grid, RESIZE_THREADS, 0, st>>>(a);
    return check_hip(hipGetLastError(), "kv_resize_kernel");
}

#define QL_KV_DISPATCH(kv, CALL)                                                  \
    do {                                                                          \
        if ((kv).bits == 16) {                                                    \
            if ((kv).D == 64) CALL(2, 64);                                        \
            else if ((kv).D == 128) CALL(2, 128);                                 \
            else CALL(2, 256);                                                    \
        } else {                                                                  \
            if ((kv).D == 64) CALL(1, 64);                                        \
            else if ((kv).D == 128) CALL(1, 128);                                 \
            else CALL(1, 256);                                                    \
        }                                                                         \
    } while (0)

// Rows of a workgroup: 8 where 32 would make no more than two workgroups for every CU, whose single tokens are moved one after the other.
// Append and read back, us, 8 / 32 rows, 8 heads, int8: 128 single tokens 10.6 / 19.1; 4 requests with 512 tokens 11.6 / 14.4, 1024 13.7 / 16.9,
// 2048 20.2 / 20.1, 4096 37 / 28; 32 heads, 512 tokens 16.7 / 18.8, 1024 22 / 20; 16000 tokens of one head 61 / 59.
static int tile_rows(int T, int heads) { return T <= 4096 && (int64_t)T * heads <= 512 * 32 ? 8 : 32; }

int launch_kv_append(const __half *q, int64_t ldq, const __half *k, int64_t ldk, const __half *v, int64_t ldv, int T, int q_heads,
                     const float *cos_sin, int rotary, int max_positions, const int32_t *positions, const int32_t *slots,
                     __half *q_out, int64_t ldqo, const KvView &kv, hipStream_t st)
{
    const int tile = tile_rows(T, kv.heads);
    const int64_t pairs = (int64_t)T * q_heads, kv_groups = (int64_t)ceil_div(T, tile) * kv.heads, grid = kv_groups + (pairs + 31) / 32;
    if (grid >= (int64_t)1 << 31 || pairs >= ((int64_t)1 << 32) - 64) return fail(QL_ERR_UNSUPPORTED, "%d tokens of %d and %d heads are more than a launch holds", T, q_heads, kv.heads);
    const AppendArgs a = {q, k, v, ldq, ldk, ldv, ldqo, q_out, cos_sin, positions, slots, T, q_heads, rotary, max_positions, (int)kv_groups, kv};
#define QL_CALL(E, D)                                                                 \
    do {                                                                              \
        if (tile == 8) kv_append_kernel<E, D, 8><<<(unsigned)grid, 2 * D, 0, st>>>(a); \
        else kv_append_kernel<E, D, 32><<<(unsigned)grid, 2 * D, 0, st>>>(a);         \
    } while (0)
    QL_KV_DISPATCH(kv, QL_CALL);
#undef QL_CALL
    return check_hip(hipGetLastError(), "kv_append_kernel");
}

int launch_kv_read(const KvView &kv, const int32_t *slots, int T, __half *k, int64_t ldk, __half *v, int64_t ldv, hipStream_t st)
{
    const int tile = tile_rows(T, kv.heads);
    const int64_t grid = (int64_t)ceil_div(T, tile) * kv.heads;
    if (grid >= (int64_t)1 << 31) return fail(QL_ERR_UNSUPPORTED, "%d tokens of %d heads are more than a launch holds", T, kv.heads);
#define QL_CALL(E, D)                                                                                             \
    do {                                                                                                          \
        if (tile == 8) kv_read_kernel<E, D, 8><<<(unsigned)grid, 2 * D, 0, st>>>(kv, slots, T, k, ldk, v, ldv);   \
        else kv_read_kernel<E, D, 32><<<(unsigned)grid, 2 * D, 0, st>>>(kv, slots, T, k, ldk, v, ldv);            \
    } while (0)
    QL_KV_DISPATCH(kv, QL_CALL);
#undef QL_CALL
    return check_hip(hipGetLastError(), "kv_read_kernel");
}

}  // namespace ql
