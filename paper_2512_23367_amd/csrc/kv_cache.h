// The paged key/value cache: its layout (include/qlinear.h) and the kernels' view of it.
#pragma once

#include "common.h"

namespace ql {

constexpr int KV_BLOCK = 32;                       // tokens of a block
constexpr int KV_SCALES = 512;                     // bytes of a block's scales (int8)
constexpr float KV_NOTHING = 0x1p-100f;            // a vector whose largest magnitude is below is stored as zeros

__host__ __device__ inline int kv_block_bytes(int D, int bits) { return 2 * KV_BLOCK * D * (bits / 8) + (bits == 8 ? KV_SCALES : 0); }

struct KvView {
    char *base;
    int heads, D, pages, bits;
    int page_shift;                                // log2(page_size)
    int block_bytes;

    __host__ __device__ int page_size() const { return 1 << page_shift; }
    // first byte of the block that holds token `rest` (0 .. page_size - 1) of a page, for one head
    __device__ char *block(int page, int head, int rest) const
    {
        return base + (((((int64_t)page * heads + head) << page_shift) + rest) >> 5) * block_bytes;
    }
};

// Byte offsets in a block (ELEM: 2 bytes of fp16, 1 of int8).
template <int ELEM>
__host__ __device__ inline int kv_key_offset(int token, int channel)
{
    if (ELEM == 2) return (channel >> 4) * 1024 + ((channel >> 3) & 1) * 512 + token * 16 + (channel & 7) * 2;
    return (channel >> 5) * 1024 + ((channel >> 4) & 1) * 512 + token * 16 + (channel & 15);
}
template <int ELEM>
__host__ __device__ inline int kv_value_offset(int token, int channel, int D)
{
    const int s = token >> 4, jh = (token >> 3) & 1, h = (token >> 2) & 1, jl = token & 3;
    if (ELEM == 2) return KV_BLOCK * D * 2 + (channel >> 5) * 2048 + s * 1024 + h * 512 + (channel & 31) * 16 + (4 * jh + jl) * 2;
    return KV_BLOCK * D + (channel >> 5) * 1024 + h * 512 + (channel & 31) * 16 + 8 * s + 4 * jh + jl;
}
__host__ __device__ inline int kv_scale_offset(int D) { return 2 * KV_BLOCK * D; }   // then [4][32] fp32

struct AttnArgs {
    const __half *q;
    int64_t ldq;
    __half *y;
    int64_t ldy;
    KvView kv;
    const int32_t *table;
    int64_t ld_table;
    int columns;
    const int32_t *cu, *ctx, *len;
    int T, requests, q_heads, group;
    unsigned group_mul, group_shift;     // r / group = (high word of r * group_mul, + r) >> group_shift for r below 2^31
    float scale;
    int causal, window;
    int max_new;
    void *ws;
    size_t ws_bytes;
};

int launch_kv_resize(const int32_t *old_len, const int32_t *want_len, int requests, int page_shift, int32_t *ring, int pages,
                     const int32_t *pool, int32_t *pool_out, int32_t *table, int64_t ld_table, int columns, int32_t *kv_len,
                     int32_t *cu_new, int32_t *slots, int32_t *positions, int max_tokens, hipStream_t st);
int launch_kv_append(const __half *q, int64_t ldq, const __half *k, int64_t ldk, const __half *v, int64_t ldv, int T, int q_heads,
                     const float *cos_sin, int rotary, int max_positions, const int32_t *positions, const int32_t *slots,
                     __half *q_out, int64_t ldqo, const KvView &kv, hipStream_t st);
int launch_kv_read(const KvView &kv, const int32_t *slots, int T, __half *k, int64_t ldk, __half *v, int64_t ldv, hipStream_t st);
size_t attention_workspace_bytes(const KvView &kv, int T, int requests, int q_heads, int max_new);
int launch_attention(const AttnArgs &a, hipStream_t st);

}  // namespace ql
