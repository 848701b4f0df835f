// Attention of new tokens over the paged key/value cache (include/qlinear.h).
#include "kv_cache.h"

namespace ql {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef unsigned char u8x16 __attribute__((ext_vector_type(16)));

// One wavefront per new token and query head, one pass over the cache in steps of two blocks: lane l scores token l of the
// step (its key is 16-byte pieces, 512 bytes apart), the running maximum and sum are those of the whole wavefront, and for the output lane l
// holds channels l, l + 64, ... (whose values of consecutive tokens are 16-byte pieces as well).
template <int ELEM, int D>
__global__ __launch_bounds__(64) void attention_kernel(AttnArgs a)
{
    constexpr int N = D / 64;
    __shared__ float sq[D], sp[64], sv[64];
    const int lane = threadIdx.x, t = blockIdx.x, head = blockIdx.y, g = head / a.group;
    if (t < a.cu[0] || t >= a.cu[a.requests]) return;
    int b = 0, hi = a.requests;
    while (hi - b > 1) {
        const int mid = (b + hi) / 2;
        if (a.cu[mid] <= t) b = mid; else hi = mid;
    }
    const int len = (int)min((int64_t)max(a.len[b], 0), (int64_t)a.columns << a.kv.page_shift);
    int first = 0, end = len;
    if (a.causal) {
        const int64_t pos = (int64_t)a.ctx[b] + (t - a.cu[b]);
        end = (int)max((int64_t)0, min((int64_t)len, pos + 1));
        if (a.window) first = (int)max((int64_t)0, pos - a.window + 1);
    }
    for (int i = 0; i < N; ++i) sq[lane + 64 * i] = __half2float(a.q[t * a.ldq + (int64_t)head * D + lane + 64 * i]);
    __syncthreads();
    float m = -INFINITY, l = 0, o[N];
    for (int i = 0; i < N; ++i) o[i] = 0;
    for (int j0 = first & ~63; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        auto page_of = [&](int j) { return a.table[b * a.ld_table + (j >> a.kv.page_shift)]; };
        bool seen = j >= first && j < end;
        const int page = seen ? page_of(j) : 0;
        seen = seen && (unsigned)page < (unsigned)a.kv.pages;
        float s = 0, scale_v = 1;
        if (seen) {
            const char *block = a.kv.block(page, g, j & (a.kv.page_size() - 1));
            const float *of = reinterpret_cast<const float *>(block + kv_scale_offset(D));
            for (int c = 0; c < D; c += 8) {
                const char *p = block + kv_key_offset<ELEM>(j % KV_BLOCK, c);
                for (int i = 0; i < 8; ++i)
                    s = fmaf(sq[c + i], ELEM == 2 ? __half2float(reinterpret_cast<const __half *>(p)[i]) : (float)(reinterpret_cast<const uint8_t *>(p)[i] - 128), s);
            }
            if (ELEM == 1) s *= of[j % KV_BLOCK], scale_v = of[KV_BLOCK + j % KV_BLOCK];
            s *= a.scale;
        } else {
            s = -INFINITY;
        }
        float top = s;
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
        const float p = expf(s - base), keep = expf(m - base);
        float sum = p;
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        l = l * keep + sum, m = m_new;
        sp[lane] = p, sv[lane] = seen ? scale_v : 0.f;
        __syncthreads();
        for (int i = 0; i < N; ++i) o[i] *= keep;
        for (int half = 0; half < 64; half += KV_BLOCK) {
            if (j0 + half >= end || j0 + half + KV_BLOCK <= first) continue;
            const int pg = page_of(j0 + half);
            if ((unsigned)pg >= (unsigned)a.kv.pages) continue;
            const char *block = a.kv.block(pg, g, (j0 + half) & (a.kv.page_size() - 1));
            for (int i = 0; i < N; ++i)
                for (int r = 0; r < KV_BLOCK; ++r) {
                    const char *p = block + kv_value_offset<ELEM>(r, lane + 64 * i, D);
                    const float x = ELEM == 2 ? __half2float(*reinterpret_cast<const __half *>(p)) : (float)(*reinterpret_cast<const uint8_t *>(p) - 128);
                    const float w = sv[half + r];
                    if (w != 0.f) o[i] = fmaf(sp[half + r], x * w, o[i]);
                }
        }
        __syncthreads();
    }
    for (int i = 0; i < N; ++i)
        a.y[t * a.ldy + (int64_t)head * D + lane + 64 * i] = __float2half(l == 0 ? 0.f : o[i] / l);
}

}  // namespace

size_t attention_workspace_bytes(const KvView &, int, int, int, int) { return 0; }

int launch_attention(const AttnArgs &a, hipStream_t st)
{
    const dim3 grid(a.T, a.q_heads);
    auto run = [&](auto kernel) { kernel<<<grid, 64, 0, st>>>(a); };
    if (a.kv.bits == 16) {
        if (a.kv.D == 64) run(attention_kernel<2, 64>);
        else if (a.kv.D == 128) run(attention_kernel<2, 128>);
        else run(attention_kernel<2, 256>);
    } else {
        if (a.kv.D == 64) run(attention_kernel<1, 64>);
        else if (a.kv.D == 128) run(attention_kernel<1, 128>);
        else run(attention_kernel<1, 256>);
    }
    return check_hip(hipGetLastError(), "attention_kernel");
}

}  // namespace ql
