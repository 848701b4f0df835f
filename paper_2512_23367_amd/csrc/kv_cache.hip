// Bookkeeping of the paged key/value cache, and what writes and reads it (layout: include/qlinear.h, kv_cache.h).
#include "kv_cache.h"

namespace ql {
namespace {

// ---- lengths -> pages, slots, positions ------------------------------------------------------------------------
// With n_b = new tokens, T_b = take_b pages, R_b = give_b pages of request b, everything follows from three prefix sums over the
// requests: row t belongs to the request whose range of cu holds it, the i-th page taken is ring[head + i], the i-th given
// back goes to ring[head + free + i].  No step waits for another, so one launch does it: every workgroup forms the sums itself (at most
// 4096 requests, from the caches) and takes a share of the tokens and pages.  The places of the ring that a call reads and
// those that it writes are different ones, entries of the table that are looked up for tokens are not those that are written;
// only the pool's state is read by all and written at the end, by the workgroup that finishes last, so that it may be updated in place.
constexpr int RESIZE_THREADS = 256;
constexpr int RESIZE_MOST = 4096;

__device__ inline int64_t wave_prefix(int64_t v, int lane)    // inclusive
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// exclusive prefix sum over the workgroup's threads; total in `sum`
__device__ inline int64_t block_prefix(int64_t v, int64_t *part, int64_t &sum)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t inc = wave_prefix(v, lane);
    __syncthreads();                                          // (of an earlier use of `part`)
    if (lane == 63) part[wave] = inc;
    __syncthreads();
    int64_t before = 0;
    sum = 0;
#pragma unroll
    for (int w = 0; w < RESIZE_THREADS / 64; ++w) {
        if (w < wave) before += part[w];
        sum += part[w];
    }
    return before + inc - v;
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

__global__ __launch_bounds__(RESIZE_THREADS) void kv_resize_kernel(const int32_t *__restrict__ old_len, const int32_t *__restrict__ want_len, int B,
                                                                   int page_shift, int32_t *ring, int pages, const int32_t *pool, int32_t *pool_out,
                                                                   int32_t *table, int64_t ld_table, int columns, int32_t *__restrict__ kv_len,
                                                                   int32_t *__restrict__ cu_new, int32_t *__restrict__ slots,
                                                                   int32_t *__restrict__ positions, int max_tokens)
{
    __shared__ int cu[RESIZE_MOST + 1], takes[RESIZE_MOST + 1], gives[RESIZE_MOST + 1];
    __shared__ int64_t part[RESIZE_THREADS / 64];
    const int tid = threadIdx.x, page = 1 << page_shift, cap = columns << page_shift;
    const int per = (B + RESIZE_THREADS - 1) / RESIZE_THREADS, first = min(B, tid * per), last = min(B, first + per);

    int head = pool[0] % pages, free = pool[1];
    head = head < 0 ? head + pages : head;
    free = min(max(free, 0), pages);

    auto old_of = [&](int b) { return min(max(old_len[b], 0), cap); };
    auto pages_of = [&](int len) { return (int)(((int64_t)len + page - 1) >> page_shift); };

    int64_t mine = 0, sum;
    for (int b = first; b < last; ++b) mine += max(0, max(want_len[b], 0) - old_of(b));
    int64_t at = block_prefix(mine, part, sum);
    for (int b = first; b < last; ++b) {
        cu[b] = (int)min(at, (int64_t)max_tokens);
        at += max(0, max(want_len[b], 0) - old_of(b));
    }
    if (tid == 0) cu[B] = (int)min(sum, (int64_t)max_tokens);
    __syncthreads();

    // the length that request b would have with pages for all of it
    auto target_of = [&](int b) {
        const int o = old_of(b), w = max(want_len[b], 0);
        return w < o ? w : (int)min((int64_t)o + (cu[b + 1] - cu[b]), (int64_t)cap);
    };
    int64_t both = 0;                                         // pages taken, pages given << 32 (each sum below 2^31)
    for (int b = first; b < last; ++b) {
        const int d = pages_of(target_of(b)) - pages_of(old_of(b));
        both += d > 0 ? (int64_t)d : (int64_t)-d << 32;
    }
    int64_t all;
    int64_t before = block_prefix(both, part, all);
    int64_t lost = 0;
    for (int b = first; b < last; ++b) {
        const int o = old_of(b), t = target_of(b), has = pages_of(o), d = pages_of(t) - has, w = max(want_len[b], 0);
        const int taken = (int)(before & 0xffffffff);
        takes[b] = taken, gives[b] = (int)(before >> 32);
        before += d > 0 ? (int64_t)d : (int64_t)-d << 32;
        const int got = d > 0 ? min(max(free - taken, 0), d) : 0;
        const int len = w < o ? w : (int)min((int64_t)t, (int64_t)(has + got) << page_shift);
        if (w >= o) lost += (int64_t)o + (cu[b + 1] - cu[b]) - len;
        if (blockIdx.x == 0) kv_len[b] = len, cu_new[b] = cu[b];
    }
    if (tid == 0) {
        takes[B] = (int)(all & 0xffffffff), gives[B] = (int)(all >> 32);
        if (blockIdx.x == 0) cu_new[B] = cu[B];
    }
    int64_t lost_sum;
    block_prefix(lost, part, lost_sum);                       // (its barriers also make takes and gives visible)

    const int from = blockIdx.x * RESIZE_THREADS + tid, step = gridDim.x * RESIZE_THREADS;
    const int taken = min(takes[B], free), given = min(gives[B], pages - free);   // (a pool that is in order has room for all of them)
    auto ring_at = [&](int64_t i) { return ring + (head + i) % pages; };
    for (int64_t t = from; t < cu[B]; t += step) {
        const int b = request_of(cu, B, (int)t), o = old_of(b), has = pages_of(o);
        const int64_t pos = (int64_t)o + (t - cu[b]);
        const int64_t j = pos >> page_shift;
        int p = -1;
        if (j < has) p = table[b * ld_table + j];
        else if (pos < cap && takes[b] + j - has < free) p = *ring_at(takes[b] + j - has);
        slots[t] = p >= 0 && p < pages ? (p << page_shift) + (int)(pos & (page - 1)) : -1;
        positions[t] = (int)min(pos, (int64_t)INT32_MAX);
    }
    for (int64_t i = from; i < taken; i += step) {
        const int b = request_of(takes, B, (int)i);
        table[b * ld_table + pages_of(old_of(b)) + (i - takes[b])] = *ring_at(i);
    }
    for (int64_t i = from; i < given; i += step) {
        const int b = request_of(gives, B, (int)i);
        *ring_at((int64_t)free + i) = table[b * ld_table + pages_of(max(want_len[b], 0)) + (i - gives[b])];
    }

    if (gridDim.x > 1) {                                      // all have read the pool's state once the last one arrives
        __shared__ int arrived;
        __syncthreads();
        if (tid == 0) arrived = __hip_atomic_fetch_add(pool_out + 3, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (int)gridDim.x - 1) return;
    }
    if (tid == 0) {
        pool_out[0] = (int)(((int64_t)head + taken) % pages);
        pool_out[1] = free - taken + given;
        pool_out[2] = (int)min(lost_sum, (int64_t)INT32_MAX);
        __hip_atomic_store(pool_out + 3, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// ---- new tokens into the cache ---------------------------------------------------------------------------------

__device__ inline bool finite(float x) { return __builtin_fabsf(x) <= 3.402823466e38f; }

__device__ inline float wave_max(float v)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// One wavefront per token and head; lane l holds channels l, l + 64, ...
template <int ELEM, int D>
__global__ __launch_bounds__(256) void kv_append_kernel(const __half *q, int64_t ldq, const __half *__restrict__ k, int64_t ldk,
                                                        const __half *__restrict__ v, int64_t ldv, int T, int q_heads,
                                                        const float *__restrict__ cos_sin, int rotary, int max_positions,
                                                        const int32_t *__restrict__ positions, const int32_t *__restrict__ slots, __half *q_out,
                                                        int64_t ldqo, KvView kv)
{
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (t >= T) return;
    const int half = rotary / 2;
    const float *row = nullptr;
    if (rotary) row = cos_sin + (int64_t)min(max(positions[t], 0), max_positions - 1) * rotary;
    auto rotated = [&](const __half *x, float (&out)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = lane + 64 * i;
            const float a = __half2float(x[c]);
            if (c < rotary) {
                const bool lower = c < half;
                const float b = __half2float(x[lower ? c + half : c - half]);
                const float co = row[lower ? c : c - half], si = row[half + (lower ? c : c - half)];
                const float m = a * co, n = b * si;
                out[i] = lower ? m - n : m + n;
            } else {
                out[i] = a;
            }
        }
    };
    if ((int)blockIdx.y < q_heads) {
        const int64_t at = (int64_t)blockIdx.y * D;
        float x[N];
        rotated(q + t * ldq + at, x);
#pragma unroll
        for (int i = 0; i < N; ++i) q_out[t * ldqo + at + lane + 64 * i] = __float2half(x[i]);
        return;
    }
    const int h = blockIdx.y - q_heads, slot = slots[t];
    if ((unsigned)slot >= (unsigned)kv.pages << kv.page_shift) return;
    float x[N], y[N];
    rotated(k + t * ldk + (int64_t)h * D, x);
    bool fine = true;
    float kmax = 0, vmax = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        y[i] = __half2float(v[t * ldv + (int64_t)h * D + lane + 64 * i]);
        if (ELEM == 2) x[i] = __half2float(__float2half(x[i]));
        fine = fine && finite(x[i]) && finite(y[i]);
        kmax = fmaxf(kmax, __builtin_fabsf(x[i])), vmax = fmaxf(vmax, __builtin_fabsf(y[i]));
    }
    fine = __all(fine);
    const int rest = slot & (kv.page_size() - 1), token = rest % KV_BLOCK;
    char *block = kv.block(slot >> kv.page_shift, h, rest);
    if (ELEM == 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = lane + 64 * i;
            *reinterpret_cast<__half *>(block + kv_key_offset<2>(token, c)) = fine ? __float2half(x[i]) : __ushort_as_half(0x7e00);
            *reinterpret_cast<__half *>(block + kv_value_offset<2>(token, c, D)) = fine ? __float2half(y[i]) : __ushort_as_half(0);
        }
        return;
    }
    kmax = wave_max(kmax), vmax = wave_max(vmax);
    const bool some_k = fine && kmax >= KV_NOTHING, some_v = fine && vmax >= KV_NOTHING;
    const float inv_k = 127.0f / kmax, inv_v = 127.0f / vmax;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int c = lane + 64 * i;
        const float ck = some_k ? fminf(fmaxf(rintf(x[i] * inv_k), -127.f), 127.f) : 0.f;
        const float cv = some_v ? fminf(fmaxf(rintf(y[i] * inv_v), -127.f), 127.f) : 0.f;
        *reinterpret_cast<uint8_t *>(block + kv_key_offset<1>(token, c)) = (uint8_t)((int)ck + 128);
        *reinterpret_cast<uint8_t *>(block + kv_value_offset<1>(token, c, D)) = (uint8_t)((int)cv + 128);
    }
    if (lane < 4) {
        const float sk = !fine ? __builtin_nanf("") : some_k ? kmax / 127.0f : 0x1p-31f, sv = some_v ? vmax / 127.0f : 0x1p-31f;
        const float out = lane == 0 ? sk : lane == 1 ? sv : lane == 2 ? log2f(sv) : 1.0f / sv;
        reinterpret_cast<float *>(block + kv_scale_offset(D))[lane * KV_BLOCK + token] = out;
    }
}

// One wavefront per token and head.
template <int ELEM, int D>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView kv, const int32_t *__restrict__ slots, int T, __half *__restrict__ k, int64_t ldk,
                                                      __half *__restrict__ v, int64_t ldv)
{
    const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6), h = blockIdx.y;
    if (t >= T) return;
    const int slot = slots[t];
    const bool there = (unsigned)slot < (unsigned)kv.pages << kv.page_shift;
    const int rest = there ? slot & (kv.page_size() - 1) : 0, token = rest % KV_BLOCK;
    const char *block = kv.block(there ? slot >> kv.page_shift : 0, h, rest);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const int c = lane + 64 * i;
        float a = 0, b = 0;
        if (there) {
            const char *pk = block + kv_key_offset<ELEM>(token, c), *pv = block + kv_value_offset<ELEM>(token, c, D);
            if (ELEM == 2) {
                a = __half2float(*reinterpret_cast<const __half *>(pk)), b = __half2float(*reinterpret_cast<const __half *>(pv));
            } else {
                const float *s = reinterpret_cast<const float *>(block + kv_scale_offset(D));
                a = (float)(*reinterpret_cast<const uint8_t *>(pk) - 128) * s[token];
                b = (float)(*reinterpret_cast<const uint8_t *>(pv) - 128) * s[KV_BLOCK + token];
            }
        }
        if (k) k[t * ldk + (int64_t)h * D + c] = __float2half(a);
        if (v) v[t * ldv + (int64_t)h * D + c] = __float2half(b);
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
    const int grid = min(256, max(1, max(ceil_div(max_tokens, 4 * RESIZE_THREADS), requests / 64)));
    kv_resize_kernel<<<grid, RESIZE_THREADS, 0, st>>>(old_len, want_len, requests, page_shift, ring, pages, pool, pool_out, table, ld_table, columns,
                                                      kv_len, cu_new, slots, positions, max_tokens);
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

int launch_kv_append(const __half *q, int64_t ldq, const __half *k, int64_t ldk, const __half *v, int64_t ldv, int T, int q_heads,
                     const float *cos_sin, int rotary, int max_positions, const int32_t *positions, const int32_t *slots,
                     __half *q_out, int64_t ldqo, const KvView &kv, hipStream_t st)
{
    const dim3 grid(ceil_div(T, 4), q_heads + kv.heads);
#define QL_CALL(E, D) kv_append_kernel<E, D><<<grid, 256, 0, st>>>(q, ldq, k, ldk, v, ldv, T, q_heads, cos_sin, rotary, max_positions, positions, slots, q_out, ldqo, kv)
    QL_KV_DISPATCH(kv, QL_CALL);
#undef QL_CALL
    return check_hip(hipGetLastError(), "kv_append_kernel");
}

int launch_kv_read(const KvView &kv, const int32_t *slots, int T, __half *k, int64_t ldk, __half *v, int64_t ldv, hipStream_t st)
{
    const dim3 grid(ceil_div(T, 4), kv.heads);
#define QL_CALL(E, D) kv_read_kernel<E, D><<<grid, 256, 0, st>>>(kv, slots, T, k, ldk, v, ldv)
    QL_KV_DISPATCH(kv, QL_CALL);
#undef QL_CALL
    return check_hip(hipGetLastError(), "kv_read_kernel");
}

}  // namespace ql
