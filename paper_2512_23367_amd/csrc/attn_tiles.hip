// Attention of many new tokens over the paged cache: workgroups of several wavefronts, 32 rows each, that share tiles of keys and values
// in LDS.
#include "attention.h"
#include "gemm_tiles.h"

namespace ql {
namespace {

__device__ inline unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, h2{(_Float16)a, (_Float16)b}); }
__device__ inline h8 as_h8(u4 v) { return __builtin_bit_cast(h8, v); }

// Four codes (stored plus 128) -> four fp16, exactly: a byte under the exponent of 1024 is 1024 + byte.
__device__ inline void widen_codes(unsigned w, unsigned &lo, unsigned &hi)
{
    const h2 off = {(_Float16)1152, (_Float16)1152};
    lo = __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - off);
    hi = __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - off);
}

// Tiles that are fetched ahead, and taken between two barriers.  (us, one / two of them: eight wavefronts, fp16, 16384 tokens 2131 / 2093, int8,
// 2 x 1000 on 9000 and 17000, 638 / 641; four wavefronts, of which two workgroups share a CU otherwise: 16 x 5 new tokens, 64 + 8 heads, 72 / 81.)
constexpr int tile_distance(int ELEM, int NW) { return ELEM == 2 && NW == 8 ? 2 : 1; }

template <int ELEM, int D, int NW>
__global__ __launch_bounds__(NW * 64, D == 256 ? 1 : 2) void attn_tile_kernel(AttnArgs a, AttnPlan plan, float c, unsigned flip)
{
    constexpr int BM = 32 * NW, TB = D == 256 ? 1 : 2;               // rows; blocks of 32 tokens in a tile of keys
    constexpr int TOK = 32 * TB, KS = D / 16, ET = D / 32;
    constexpr int BLOCK = 32 * D * 4;                                // bytes of a block's keys and values in LDS (fp16)
    constexpr int VALU_ONLY = 0x6;                                   // sched_barrier: vector and scalar arithmetic may pass
    constexpr int DIST = tile_distance(ELEM, NW);
    constexpr int SC = ELEM == 1 ? 3 * TOK : 1;
    extern __shared__ __attribute__((aligned(1024))) char stage[];
    auto tile = [&](int i) { return stage + i * TB * BLOCK; };
    __shared__ __attribute__((aligned(16))) float scales[2 * DIST][SC];
    __shared__ AttnScratch scratch;

    const int kvh = blockIdx.x % a.kv.heads, index = blockIdx.x / a.kv.heads;
    AttnItem it;
    if (!attn_take<NW * 64, BM>(a, plan, index, kvh, scratch, it)) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, h = lane >> 5;
    const int row0 = it.tile * BM, wrow0 = row0 + wave * 32, row = wrow0 + col;
    const bool live = row < it.r.rows;
    const int token = live ? attn_token(a, row) : 0, head = kvh * a.group + (live ? row - token * a.group : 0);
    // positions: of this lane's row, of the wavefront's first and last (scalar, so that the loop branches on scalars: 16384 tokens 2085 us, so 2028)
    auto position = [&](int r) { return (int)min(max((int64_t)it.r.ctx + attn_token(a, r), (int64_t)-1), (int64_t)INT32_MAX); };
    const int pos = position(live ? row : 0);
    const int pos0 = __builtin_amdgcn_readfirstlane(position(wrow0)), pos1 = __builtin_amdgcn_readfirstlane(position(min(wrow0 + 32, it.r.rows) - 1));
    const int rows = __builtin_amdgcn_readfirstlane(it.r.rows - wrow0);   // from this wavefront's first

    int low, high;
    attn_range(a, it.r, row0, min(row0 + BM, it.r.rows), low, high);
    attn_part_range(low, high, it.part, it.parts);
    low = __builtin_amdgcn_readfirstlane(low), high = __builtin_amdgcn_readfirstlane(high);

    // queries: column operand, 8 channels of a step per lane, in the order of the keys' channels
    h8 q[KS];
    {
        const __half *src = a.q + (int64_t)(it.r.cu + token) * a.ldq + (int64_t)head * D;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const int d = ELEM == 2 ? 16 * s + 8 * h : 32 * (s / 2) + 16 * h + 8 * (s % 2);
            u4 v = {0, 0, 0, 0};
            if (live) v = *reinterpret_cast<const u4 *>(src + d);
            q[s] = attn_query(as_h8(v ^ flip));
        }
    }

    f16v o[ET];
#pragma unroll
    for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[e][i] = 0;
    float m = -INFINITY, l = 0;
    bool far = false;                                                // of the wavefront: see ATTN_FAR

    // the table's entries of 64 tiles at a time, one per lane (a load for every tile: 8192 tokens, D = 64, 339 us, so 336)
    const int32_t *row_of_table = a.table + (int64_t)it.b * a.ld_table;
    int entries[TB], shift = a.kv.page_shift;
    asm("" : "+v"(shift));                                           // (a copy for the lanes, or the scalar one moves there, too)
    auto look_up = [&](int first) {
#pragma unroll
        for (int i = 0; i < TB; ++i) {
            const int64_t t = low + (int64_t)(first + lane) * TOK + 32 * i;
            entries[i] = t < high ? row_of_table[t >> shift] : -1;
        }
    };
    auto page_of = [&](int turn, int i) {                            // of block i of a tile, -1: none
        const int p = __builtin_amdgcn_readlane(entries[i], turn & 63);
        return (unsigned)p < (unsigned)a.kv.pages ? p : -1;
    };
    auto block_at = [&](int page, int t) { return a.kv.block(max(page, 0), kvh, t & (a.kv.page_size() - 1)); };

    // of the tile at hand, of the next ones (int8: in private memory, 32 bytes that every turn stores, as clear() picks them by lane)
    int pages[DIST + 1][TB];

    // ---- a tile into LDS ----
    constexpr int PIECES = ELEM == 2 ? TB * BLOCK / 1024 / NW : TB * BLOCK / 2 / 1024 / NW;   // KB per wavefront, as stored
    u4 staged[ELEM == 1 ? PIECES : 1];
    float staged_scale[3];
    auto fetch = [&](int t, char *to, const int (&pg)[TB]) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            constexpr int PER = BLOCK / (ELEM == 2 ? 1024 : 2048);   // pieces of a block
            static_assert(PER % NW == 0, "a piece's block does not depend on the wavefront");   // (one address for a block's pieces)
            const int p = i * NW + wave, blk = i * NW / PER, off = (i * NW % PER + wave) * 1024;
            // (a block without a page: a buffer of no bytes, whose loads return zeros)
            const int page = TB == 1 ? pg[0] : blk ? pg[TB - 1] : pg[0];
            const __amdgpu_buffer_rsrc_t rs = make_rsrc(block_at(page, t + 32 * blk), page >= 0 ? (unsigned)a.kv.block_bytes : 0u);
            if constexpr (ELEM == 2)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, LDS_PTR(to + p * 1024), 16, off + lane * 16, 0, 0, 0);
            else
                staged[i] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rs, off + lane * 16, 0, 0));
        }
        if constexpr (ELEM == 1) {
            if (tid < TOK) {
                const int blk = tid / 32, page = TB == 1 ? pg[0] : blk ? pg[TB - 1] : pg[0];
                const float *s = reinterpret_cast<const float *>(block_at(page, t + 32 * blk) + kv_scale_offset(D)) + tid % 32;
                staged_scale[0] = s[0], staged_scale[1] = s[64], staged_scale[2] = s[96];
            }
        }
    };
    auto settle = [&](char *to, float *sc) {                         // int8: widen what was fetched into LDS
        if constexpr (ELEM == 1) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const int p = i * NW + wave;
                u4 lo, hi;
                unsigned x, y;
                widen_codes(staged[i][0], x, y), lo[0] = x, lo[1] = y;
                widen_codes(staged[i][1], x, y), lo[2] = x, lo[3] = y;
                widen_codes(staged[i][2], x, y), hi[0] = x, hi[1] = y;
                widen_codes(staged[i][3], x, y), hi[2] = x, hi[3] = y;
                *reinterpret_cast<u4 *>(to + p * 2048 + lane * 16) = lo;
                *reinterpret_cast<u4 *>(to + p * 2048 + 1024 + lane * 16) = hi;
            }
            if (tid < TOK) sc[tid] = staged_scale[0] * c, sc[TOK + tid] = staged_scale[1], sc[2 * TOK + tid] = staged_scale[2];
        } else {
            wait_vmcnt<0>();
        }
    };

    // What lies behind the last token, or on no page, is whatever memory held: its weights are 0, but 0 times NaN is not.  fp16: values of
    // such tokens are cleared (one tile of a workgroup); int8: the reciprocal scales, codes are finite.
    auto whole = [&](int t, const int (&pg)[TB]) {
        bool w = t <= high - TOK;
#pragma unroll
        for (int i = 0; i < TB; ++i) w = w && pg[i] >= 0;
        return w;
    };
    auto clear = [&](int t, char *to, float *sc, const int (&pg)[TB]) {
        if constexpr (ELEM == 1) {
            if (tid < TOK && !(t + tid < high && (TB == 1 || tid < 32 ? pg[0] : pg[TB - 1]) >= 0)) sc[tid] = 0, sc[TOK + tid] = 0, sc[2 * TOK + tid] = 0;
        } else {
            for (int i = tid; i < TB * 2 * ET * 64; i += NW * 64) {  // 8 tokens of a channel each
                const int blk = i / (2 * ET * 64), at = i % (2 * ET * 64), k = at / 64 % 2, hh = at / 32 % 2;
                u4 *p = reinterpret_cast<u4 *>(to + blk * BLOCK + 32 * D * 2 + at * 16);
                u4 v = *p;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int tk = t + 32 * blk + 16 * k + 8 * (e / 4) + 4 * hh + e % 4;
                    if (!(tk < high && (blk ? pg[TB - 1] : pg[0]) >= 0)) v[e / 2] &= e % 2 ? 0x0000ffffu : 0xffff0000u;
                }
                *p = v;
            }
        }
        __syncthreads();
    };

    // ---- one tile: S^T = K Q^T, softmax down the columns, O^T += V^T P^T ----
    auto take = [&](bool masked, int t, const char *from, const float *sc, const int (&pg)[TB]) {
        // The operands from LDS are asked for a block ahead: a read takes as long as four matrix instructions, and left to itself the
        // compiler keeps two of them under way.
        f16v s[TB];
        h8 x[KS];
        auto key = [&](int b, int k) { return *reinterpret_cast<const h8 *>(from + b * BLOCK + k * 1024 + lane * 16); };
        auto value = [&](int b, int i) { return *reinterpret_cast<const h8 *>(from + b * BLOCK + 32 * D * 2 + (i % ET) * 2048 + (i / ET) * 1024 + lane * 16); };
#pragma unroll
        for (int i = 0; i < KS; ++i) x[i] = key(i % TB, i / TB);
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0;
        __builtin_amdgcn_s_setprio(1);                               // ahead of the other wavefront's softmax (int8 chunks 630 -> 621 us)
#pragma unroll
        for (int i = 0; i < TB * KS; ++i) {                          // the blocks in turn: no product waits for the one before
            s[i % TB] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i % KS], q[i / TB], s[i % TB], 0, 0, 0);
            x[i % KS] = i + KS < TB * KS ? key((i + KS) % TB, (i + KS) / TB) : value(0, i % KS);
            __builtin_amdgcn_sched_barrier(VALU_ONLY);
        }
        if constexpr (ELEM == 1) {
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4) {
                    const int j = 32 * b + 8 * i4 + 4 * h;           // token of the tile of element 4 i4
                    const f4 sk = *reinterpret_cast<const f4 *>(sc + j), lv = *reinterpret_cast<const f4 *>(sc + TOK + j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[b][4 * i4 + i] = fmaf(s[b][4 * i4 + i], sk[i], lv[i]);
                }
        }
        if (masked) {
            asm volatile("");                                        // or the compiler compares and selects for every tile
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                const int t0 = t + 32 * b;
                const int last = (pg[b] < 0 ? -1 : a.causal ? min(high - 1, pos) : high - 1) - t0;
                const int first = a.window ? max(pos - a.window, t0 - 1) - (t0 - 1) : 0;
                // bit k: token k of the block is seen; two operations an element (comparing and selecting, four: 16384 tokens
                // 2119 us, so 2106; D = 256, 4096 tokens, 252, 234)
                const unsigned seen = (last < 0 ? 0u : ~0u >> (31 - min(last, 31))) & (first > 31 ? 0u : ~0u << first);
                const unsigned mine = seen >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const unsigned all = __builtin_amdgcn_sbfe((int)mine, 8 * (i / 4) + i % 4, 1);
                    s[b][i] = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, (float)s[b][i]) & all) | (0xff800000u & ~all));
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        {
            unsigned x, y;
            lane_pair<32>(__builtin_bit_cast(unsigned, top), x, y);
            top = fmaxf(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
        }
        constexpr bool RAW = ELEM == 2;                              // scores still without the factor c
        const float factor = RAW ? c : 1.0f;
        // The maximum follows only when a score exceeds it by 2^8: with ATTN_LEAD weights up to 2^15, and the sums are rarely rescaled.
        if (__any((top - m) * factor > 8.0f)) {
            const float to = fmaxf(m, top), keep = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - to) * factor);
            m = to;
            far = __any(attn_far(m, factor));
            l *= keep;
#pragma unroll
            for (int e = 0; e < ET; ++e)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[e][i] *= keep;
        }
        float base = m == -INFINITY ? 0.f : fmaf(-m, factor, ATTN_LEAD);
        if (far) {
            asm volatile("");                                        // (a branch: hardly any call takes it)
            const float off = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] -= off;
            base = ATTN_LEAD;
        }
        h8 p[TB][2];
        // of the tile: a small weight is not lost beside all before it.  (One chain of additions, two: 16384 tokens of D = 128 2011 us, 1999; D = 64, six prompts,
        // 42.3, 43.2; D = 256, 4096 tokens, 212, 213.)
        constexpr int CHAINS = D == 128 ? 2 : 1;
        float sums[CHAINS] = {};
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            unsigned w[8];
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) {
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = __builtin_amdgcn_exp2f(RAW ? fmaf(s[b][4 * i4 + i], c, base) : s[b][4 * i4 + i] + base);
                if constexpr (ELEM == 1) {
                    const f4 iv = *reinterpret_cast<const f4 *>(sc + 2 * TOK + 32 * b + 8 * i4 + 4 * h);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sums[i % CHAINS] = fmaf(x[i], iv[i], sums[i % CHAINS]);
                }
                w[2 * i4] = pack2(x[0], x[1]), w[2 * i4 + 1] = pack2(x[2], x[3]);
                if constexpr (ELEM == 2) {                           // two weights (as rounded for the products) a step; plain sums: D = 64 53.4 us for 50.7
                    const h2 one = {(_Float16)1, (_Float16)1};
                    sums[0] = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w[2 * i4]), one, sums[0], false);
                    sums[CHAINS - 1] = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w[2 * i4 + 1]), one, sums[CHAINS - 1], false);
                }
            }
            p[b][0] = as_h8(u4{w[0], w[1], w[2], w[3]}), p[b][1] = as_h8(u4{w[4], w[5], w[6], w[7]});
        }
        l += CHAINS == 2 ? sums[0] + sums[CHAINS - 1] : sums[0];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int b = 0; b < TB; ++b)
#pragma unroll
            for (int i = 0; i < KS; ++i) {                           // (KS = 2 ET operands of values, too)
                o[i % ET] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[i], p[b][i / ET], o[i % ET], 0, 0, 0);
                if (b + 1 < TB) x[i] = value(b + 1, i);
                __builtin_amdgcn_sched_barrier(VALU_ONLY);
            }
        __builtin_amdgcn_s_setprio(0);
    };

    // ---- over the tiles ----
    if (low < high) {
        const int turns = (high - low - 1) / TOK + 1;
        look_up(0);
#pragma unroll
        for (int d = 0; d < DIST; ++d) {
#pragma unroll
            for (int i = 0; i < TB; ++i) pages[d + 1][i] = page_of(d, i);
            if (d < turns) {
                fetch(low + d * TOK, tile(d), pages[d + 1]);
                settle(tile(d), scales[d]);
            }
        }
        for (int turn = 0; turn < turns; ++turn) {
            const int t = low + turn * TOK, cur = turn % (2 * DIST), to = (turn + DIST) % (2 * DIST);
            if (turn % DIST == 0) __syncthreads();                   // tiles turn .. turn + DIST - 1 are there, the other buffers free
            const bool more = turn + DIST < turns;
            if (more && ((turn + DIST) & 63) == 0) look_up(turn + DIST);
#pragma unroll
            for (int i = 0; i < TB; ++i) {
#pragma unroll
                for (int d = 0; d < DIST; ++d) pages[d][i] = pages[d + 1][i];
                pages[DIST][i] = page_of(turn + DIST, i);
            }
            if (more) fetch(t + DIST * TOK, tile(to), pages[DIST]);
            if (!whole(t, pages[0])) clear(t, tile(cur), scales[cur], pages[0]);
            const bool some = rows > 0 && (!a.causal || (t <= pos1 && (!a.window || t + TOK - 1 > pos0 - a.window)));
            if (some) {
                bool plain = whole(t, pages[0]);
                if (a.causal) plain = plain && t + TOK - 1 <= pos0 && (!a.window || t > pos1 - a.window);
                take(!plain, t, tile(cur), scales[cur], pages[0]);
            }
            if (ELEM == 1 ? more : turn % DIST == DIST - 1) settle(tile(to), scales[to]);
        }
    }

    // ---- out ----
    {
        unsigned x, y;
        lane_pair<32>(__builtin_bit_cast(unsigned, l), x, y);
        l = __builtin_bit_cast(float, x) + __builtin_bit_cast(float, y);
    }
    if (it.parts > 1) {
        if (!live) return;
        float *out = attn_partial(a, plan, it.item, kvh);
        const int r = wave * 32 + col;
#pragma unroll
        for (int e = 0; e < ET; ++e)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4)
                *reinterpret_cast<f4 *>(out + (size_t)r * D + 32 * e + 8 * i4 + 4 * h) = f4{o[e][4 * i4], o[e][4 * i4 + 1], o[e][4 * i4 + 2], o[e][4 * i4 + 3]};
        if (h == 0) out[(size_t)BM * D + r] = m, out[(size_t)BM * (D + 1) + r] = l;
        return;
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    __half *dst = a.y + (int64_t)(it.r.cu + token) * a.ldy + (int64_t)head * D;
#pragma unroll
    for (int e = 0; e < ET; ++e)
#pragma unroll
        for (int i8 = 0; i8 < 2; ++i8) {
            // quads 4 h .. of 8 channels each: halves of the wavefront trade, so that every lane stores 8 channels
            const unsigned a0 = pack2(o[e][8 * i8] * inv, o[e][8 * i8 + 1] * inv), a1 = pack2(o[e][8 * i8 + 2] * inv, o[e][8 * i8 + 3] * inv);
            const unsigned b0 = pack2(o[e][8 * i8 + 4] * inv, o[e][8 * i8 + 5] * inv), b1 = pack2(o[e][8 * i8 + 6] * inv, o[e][8 * i8 + 7] * inv);
            const auto x = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), y = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            if (live) *reinterpret_cast<u4 *>(dst + 32 * e + 16 * i8 + 8 * h) = u4{x[0], y[0], x[1], y[1]};
        }
}

template <int ELEM, int D, int NW>
int launch(const AttnArgs &a, const AttnPlan &p, float c, unsigned flip, hipStream_t st)
{
    constexpr int LDS = 2 * tile_distance(ELEM, NW) * (D == 256 ? 1 : 2) * 32 * D * 4;
    auto kern = attn_tile_kernel<ELEM, D, NW>;
    // once per kernel and process; the initialisation of a function-local static is thread-safe
    static const hipError_t attr_status = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    QL_TRY(check_hip(attr_status, "hipFuncSetAttribute(max dynamic LDS)"));
    kern<<<(unsigned)(p.items * a.kv.heads), NW * 64, LDS, st>>>(a, p, c, flip);
    return check_hip(hipGetLastError(), "attn_tile_kernel");
}

}  // namespace

int launch_attention_tiles(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st)
{
    const unsigned flip = a.scale < 0 ? 0x80008000u : 0u;
    if (a.kv.bits == 16) {
        if (a.kv.D == 64) return launch<2, 64, 4>(a, p, c, flip, st);
        if (a.kv.D == 256) return launch<2, 256, 4>(a, p, c, flip, st);
        return p.bm == 256 ? launch<2, 128, 8>(a, p, c, flip, st) : launch<2, 128, 4>(a, p, c, flip, st);
    }
    if (a.kv.D == 64) return launch<1, 64, 4>(a, p, c, flip, st);
    if (a.kv.D == 256) return launch<1, 256, 4>(a, p, c, flip, st);
    return p.bm == 256 ? launch<1, 128, 8>(a, p, c, flip, st) : launch<1, 128, 4>(a, p, c, flip, st);
}

}  // namespace ql
