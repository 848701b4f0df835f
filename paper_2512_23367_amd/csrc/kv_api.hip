// C ABI of the paged key/value cache and the attention over it: argument validation and dispatch (include/qlinear.h).
#include <cmath>

#include "kv_cache.h"

namespace ql {
namespace {

constexpr int MAX_REQUESTS = 4096;      // of a resize: prefix sums of the requests in LDS

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int check_page_size(int page_size)
{
    if (page_size < KV_BLOCK || page_size > 1024 || (page_size & (page_size - 1)))
        return fail(QL_ERR_SHAPE, "page_size=%d must be a power of two from 32 to 1024", page_size);
    return QL_OK;
}

int check_pages(int pages, int page_size)
{
    if (pages < 1 || (int64_t)pages * page_size >= ((int64_t)1 << 31))
        return fail(QL_ERR_SHAPE, "pages=%d must be positive and pages * page_size below 2^31", pages);
    return QL_OK;
}

int view_of(const ql_kv_format *f, void *cache, KvView *v)
{
    if (!f) return fail(QL_ERR_NULL, "format is NULL");
    if (f->bits != 8 && f->bits != 16) return fail(QL_ERR_UNSUPPORTED, "unsupported bits=%d of a cache: 8 or 16", f->bits);
    if (f->head_dim != 64 && f->head_dim != 128 && f->head_dim != 256)
        return fail(QL_ERR_UNSUPPORTED, "unsupported head_dim=%d: 64, 128 or 256", f->head_dim);
    if (f->heads < 1 || f->heads > 65535) return fail(QL_ERR_SHAPE, "heads=%d must be positive (at most 65535)", f->heads);
    QL_TRY(check_page_size(f->page_size));
    QL_TRY(check_pages(f->pages, f->page_size));
    *v = KvView{static_cast<char *>(cache), f->heads, f->head_dim, f->pages, f->bits, __builtin_ctz(f->page_size),
                kv_block_bytes(f->head_dim, f->bits)};
    return QL_OK;
}

int check_cache(const void *cache)
{
    if (!cache) return fail(QL_ERR_NULL, "cache is NULL");
    if (!aligned(cache, 256)) return fail(QL_ERR_ALIGN, "cache must be 256-byte aligned");
    return QL_OK;
}

int check_rows(const void *p, int64_t ld, int64_t columns, const char *name)
{
    if (!p) return fail(QL_ERR_NULL, "%s is NULL", name);
    if (!aligned(p, 16) || ld % 8) return fail(QL_ERR_ALIGN, "%s needs 16-byte alignment and a leading dimension that is a multiple of 8", name);
    if (ld < columns) return fail(QL_ERR_ALIGN, "the leading dimension %lld of %s is less than its %lld columns", (long long)ld, name, (long long)columns);
    if (ld > MAX_ROW_STRIDE) return fail(QL_ERR_SHAPE, "the leading dimension of %s exceeds 2^27", name);
    return QL_OK;
}

int check_ints(const void *p, const char *name)
{
    if (!p) return fail(QL_ERR_NULL, "%s is NULL", name);
    if (!aligned(p, 4)) return fail(QL_ERR_ALIGN, "%s must be 4-byte aligned", name);
    return QL_OK;
}

// Whether T rows of nx columns at x and of ny columns at y share bytes (two column ranges of one buffer do not).
bool rows_meet(const void *x, int64_t ldx, int64_t nx, const void *y, int64_t ldy, int64_t ny, int T)
{
    if (!bytes_overlap(x, 2 * ((size_t)(T - 1) * ldx + nx), y, 2 * ((size_t)(T - 1) * ldy + ny))) return false;
    if (ldx != ldy) return true;
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(x), y0 = reinterpret_cast<uintptr_t>(y), ld = 2 * (uintptr_t)ldx;
    const uintptr_t shift = y0 >= x0 ? (y0 - x0) % ld : (ld - (x0 - y0) % ld) % ld;
    return shift < 2 * (uintptr_t)nx || shift + 2 * (uintptr_t)ny > ld;
}

int check_q_heads(int q_heads, int heads)
{
    if (q_heads < 1 || q_heads % heads) return fail(QL_ERR_SHAPE, "q_heads=%d must be a positive multiple of the cache's %d heads", q_heads, heads);
    return QL_OK;
}

}  // namespace
}  // namespace ql

using namespace ql;

#pragma GCC visibility push(default)
extern "C" {

int ql_kv_cache_bytes(const ql_kv_format *format, size_t *bytes)
{
    KvView v;
    QL_TRY(view_of(format, nullptr, &v));
    if (!bytes) return fail(QL_ERR_NULL, "bytes is NULL");
    *bytes = (size_t)v.pages * v.heads * (format->page_size / KV_BLOCK) * v.block_bytes;
    return QL_OK;
}

int ql_kv_resize(const int32_t *old_len, const int32_t *want_len, int requests, int page_size, int32_t *ring, int pages,
                 const int32_t *pool, int32_t *pool_out, int32_t *block_table, int64_t ld_table, int columns, int32_t *kv_len,
                 int32_t *cu_new, int32_t *slots, int32_t *positions, int max_tokens, void *stream)
{
    QL_TRY(check_page_size(page_size));
    QL_TRY(check_pages(pages, page_size));
    if (requests < 0 || max_tokens < 0 || columns < 1)
        return fail(QL_ERR_SHAPE, "requests=%d and max_tokens=%d must not be negative, columns=%d positive", requests, max_tokens, columns);
    if (requests > MAX_REQUESTS || (int64_t)requests * columns >= ((int64_t)1 << 31) || (int64_t)columns * page_size >= ((int64_t)1 << 31))
        return fail(QL_ERR_UNSUPPORTED, "at most %d requests (requests=%d), requests * columns and columns * page_size below 2^31", MAX_REQUESTS, requests);
    QL_TRY(check_ints(pool, "pool"));
    QL_TRY(check_ints(pool_out, "pool_out"));
    QL_TRY(check_ints(cu_new, "cu_new"));
    QL_TRY(check_ints(ring, "ring"));
    if (max_tokens) {
        QL_TRY(check_ints(slots, "slots"));
        QL_TRY(check_ints(positions, "positions"));
    }
    if (requests) {
        QL_TRY(check_ints(old_len, "old_len"));
        QL_TRY(check_ints(want_len, "want_len"));
        QL_TRY(check_ints(block_table, "block_table"));
        QL_TRY(check_ints(kv_len, "kv_len"));
        if (ld_table < columns) return fail(QL_ERR_SHAPE, "ld_table=%lld is less than columns=%d", (long long)ld_table, columns);
        const size_t n = 4 * (size_t)requests;
        const size_t most = 4 * (size_t)max_tokens;
        auto meets = [&](const void *p, size_t bytes) { return bytes_overlap(p, bytes, old_len, n) || bytes_overlap(p, bytes, want_len, n); };
        if (meets(kv_len, n) || meets(cu_new, n + 4) || (most && (meets(slots, most) || meets(positions, most))))
            return fail(QL_ERR_UNSUPPORTED, "kv_len, cu_new, slots and positions may not overlap old_len or want_len");
    }
    if (pool_out != pool && bytes_overlap(pool, 16, pool_out, 16)) return fail(QL_ERR_UNSUPPORTED, "pool_out is pool or does not overlap it");
    return launch_kv_resize(old_len, want_len, requests, __builtin_ctz(page_size), ring, pages, pool, pool_out, block_table, ld_table, columns,
                            kv_len, cu_new, slots, positions, max_tokens, static_cast<hipStream_t>(stream));
}

int ql_kv_append(const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, int T, int q_heads,
                 const float *cos_sin, int rotary_dim, int max_positions, const int32_t *positions, const int32_t *slots,
                 void *q_out, int64_t ldqo, void *cache, const ql_kv_format *format, void *stream)
{
    KvView kv;
    QL_TRY(view_of(format, cache, &kv));
    if (T < 0) return fail(QL_ERR_SHAPE, "T must not be negative (T=%d)", T);
    if (cos_sin) {
        if (rotary_dim < 16 || rotary_dim % 16 || rotary_dim > kv.D)
            return fail(QL_ERR_SHAPE, "rotary_dim=%d must be a positive multiple of 16, at most head_dim=%d", rotary_dim, kv.D);
        if (max_positions < 1) return fail(QL_ERR_SHAPE, "max_positions=%d must be positive", max_positions);
        if (!aligned(cos_sin, 16)) return fail(QL_ERR_ALIGN, "cos_sin must be 16-byte aligned");
    } else if (rotary_dim || q) {
        return fail(QL_ERR_UNSUPPORTED, "without cos_sin rotary_dim is 0 and q NULL");
    }
    if (q) {
        QL_TRY(check_q_heads(q_heads, kv.heads));
        if ((int64_t)q_heads + kv.heads > 65535) return fail(QL_ERR_UNSUPPORTED, "q_heads=%d is too large", q_heads);
    } else if (q_heads || q_out) {
        return fail(QL_ERR_SHAPE, "without q q_heads is 0 and q_out NULL");
    }
    if (T == 0) return QL_OK;
    QL_TRY(check_cache(cache));
    QL_TRY(check_ints(slots, "slots"));
    if (cos_sin) QL_TRY(check_ints(positions, "positions"));
    const int64_t nq = (int64_t)q_heads * kv.D, nk = (int64_t)kv.heads * kv.D;
    QL_TRY(check_rows(k, ldk, nk, "k"));
    QL_TRY(check_rows(v, ldv, nk, "v"));
    if (q) {
        QL_TRY(check_rows(q, ldq, nq, "q"));
        QL_TRY(check_rows(q_out, ldqo, nq, "q_out"));
        if ((q_out == q ? ldqo != ldq : rows_meet(q, ldq, nq, q_out, ldqo, nq, T)) || rows_meet(k, ldk, nk, q_out, ldqo, nq, T) ||
            rows_meet(v, ldv, nk, q_out, ldqo, nq, T))
            return fail(QL_ERR_UNSUPPORTED, "q_out is q (with its leading dimension) or does not overlap q, k and v");
    }
    return launch_kv_append(static_cast<const __half *>(q), ldq, static_cast<const __half *>(k), ldk, static_cast<const __half *>(v), ldv, T,
                            q_heads, cos_sin, rotary_dim, max_positions, positions, slots, static_cast<__half *>(q_out), ldqo, kv,
                            static_cast<hipStream_t>(stream));
}

int ql_kv_read(const void *cache, const ql_kv_format *format, const int32_t *slots, int T, void *k, int64_t ldk, void *v,
               int64_t ldv, void *stream)
{
    KvView kv;
    QL_TRY(view_of(format, const_cast<void *>(cache), &kv));
    if (T < 0) return fail(QL_ERR_SHAPE, "T must not be negative (T=%d)", T);
    if (T == 0) return QL_OK;
    QL_TRY(check_cache(cache));
    QL_TRY(check_ints(slots, "slots"));
    if (!k && !v) return fail(QL_ERR_NULL, "k and v are both NULL");
    const int64_t n = (int64_t)kv.heads * kv.D;
    if (k) QL_TRY(check_rows(k, ldk, n, "k"));
    if (v) QL_TRY(check_rows(v, ldv, n, "v"));
    return launch_kv_read(kv, slots, T, static_cast<__half *>(k), ldk, static_cast<__half *>(v), ldv, static_cast<hipStream_t>(stream));
}

static int check_attention_sizes(const KvView &kv, int T, int requests, int q_heads, int max_new)
{
    if (T < 0 || requests < 0 || max_new < 0)
        return fail(QL_ERR_SHAPE, "T=%d, requests=%d and max_new=%d must not be negative", T, requests, max_new);
    QL_TRY(check_q_heads(q_heads, kv.heads));
    if (requests > 65536 || (int64_t)T * (q_heads / kv.heads) >= ((int64_t)1 << 28))
        return fail(QL_ERR_UNSUPPORTED, "at most 65536 requests (requests=%d) and T * q_heads / heads below 2^28", requests);
    return QL_OK;
}

int ql_paged_attention_bytes(const ql_kv_format *format, int T, int requests, int q_heads, int max_new, size_t *bytes)
{
    KvView kv;
    QL_TRY(view_of(format, nullptr, &kv));
    if (!bytes) return fail(QL_ERR_NULL, "bytes is NULL");
    QL_TRY(check_attention_sizes(kv, T, requests, q_heads, max_new));
    *bytes = attention_workspace_bytes(kv, T, requests, q_heads, max_new);
    return QL_OK;
}

int ql_paged_attention(const void *q, int64_t ldq, int T, int q_heads, const void *cache, const ql_kv_format *format,
                       const int32_t *block_table, int64_t ld_table, int columns, const int32_t *cu_new, const int32_t *ctx_len,
                       const int32_t *kv_len, int requests, float scale, int causal, int window, int max_new, void *y, int64_t ldy,
                       void *ws, size_t ws_bytes, void *stream)
{
    KvView kv;
    QL_TRY(view_of(format, const_cast<void *>(cache), &kv));
    QL_TRY(check_attention_sizes(kv, T, requests, q_heads, max_new));
    if (!std::isfinite(scale)) return fail(QL_ERR_SHAPE, "scale must be finite");
    if (causal != 0 && causal != 1) return fail(QL_ERR_SHAPE, "causal=%d must be 0 or 1", causal);
    if (window < 0 || (window && !causal)) return fail(QL_ERR_SHAPE, "window=%d must not be negative, and 0 without causal", window);
    if (T == 0 || requests == 0) return QL_OK;
    QL_TRY(check_cache(cache));
    if (columns < 1 || (int64_t)columns * format->page_size > ((int64_t)1 << 30))
        return fail(QL_ERR_SHAPE, "columns=%d must be positive and columns * page_size at most 2^30", columns);
    if (ld_table < columns) return fail(QL_ERR_SHAPE, "ld_table=%lld is less than columns=%d", (long long)ld_table, columns);
    QL_TRY(check_ints(block_table, "block_table"));
    QL_TRY(check_ints(cu_new, "cu_new"));
    QL_TRY(check_ints(kv_len, "kv_len"));
    if (causal) QL_TRY(check_ints(ctx_len, "ctx_len"));
    const int64_t n = (int64_t)q_heads * kv.D;
    QL_TRY(check_rows(q, ldq, n, "q"));
    QL_TRY(check_rows(y, ldy, n, "y"));
    if (q == y ? ldq != ldy : rows_meet(q, ldq, n, y, ldy, n, T))
        return fail(QL_ERR_UNSUPPORTED, "y is q (with its leading dimension) or does not overlap it");
    if (!aligned(ws, 256)) return fail(QL_ERR_ALIGN, "ws must be 256-byte aligned");
    AttnArgs a = {};
    a.q = static_cast<const __half *>(q);
    a.ldq = ldq;
    a.y = static_cast<__half *>(y);
    a.ldy = ldy;
    a.kv = kv;
    a.table = block_table;
    a.ld_table = ld_table;
    a.columns = columns;
    a.cu = cu_new;
    a.ctx = causal ? ctx_len : nullptr;
    a.len = kv_len;
    a.T = T;
    a.requests = requests;
    a.q_heads = q_heads;
    a.group = q_heads / kv.heads;
    while ((1u << a.group_shift) < (unsigned)a.group) ++a.group_shift;
    a.group_mul = (unsigned)((((uint64_t)1 << 32) * ((1u << a.group_shift) - (unsigned)a.group)) / (unsigned)a.group + 1);
    a.scale = scale;
    a.causal = causal;
    a.window = window;
    a.max_new = max_new;
    a.ws = ws;
    a.ws_bytes = ws_bytes;
    return launch_attention(a, static_cast<hipStream_t>(stream));
}

}  // extern "C"
#pragma GCC visibility pop
