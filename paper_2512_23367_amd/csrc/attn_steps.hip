// Attention of few new tokens over the paged cache (decode steps, drafts): the four wavefronts of a workgroup share out the tokens and
// stream keys and values from memory straight to registers.
#include "attention.h"

namespace ql {
namespace {

__device__ inline unsigned pack2(float a, float b) { return __builtin_bit_cast(unsigned, h2{(_Float16)a, (_Float16)b}); }
__device__ inline h8 as_h8(u4 v) { return __builtin_bit_cast(h8, v); }

// Eight codes (stored plus 128) -> eight fp16, exactly: a byte under the exponent of 1024 is 1024 + byte.
__device__ inline h8 widen_codes(unsigned a, unsigned b)
{
    const h2 off = {(_Float16)1152, (_Float16)1152};
    auto pair = [&](unsigned w, unsigned select) { return __builtin_bit_cast(unsigned, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, w, select)) - off); };
    return as_h8(u4{pair(a, 0x04010400u), pair(a, 0x04030402u), pair(b, 0x04010400u), pair(b, 0x04030402u)});
}

template <typename OP>
__device__ inline float over_quarters(float v, OP op)                // of the lanes that hold one row: l, l ^ 16, l ^ 32, l ^ 48
{
    unsigned x, y;
    lane_pair<16>(__builtin_bit_cast(unsigned, v), x, y);
    v = op(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
    lane_pair<32>(__builtin_bit_cast(unsigned, v), x, y);
    return op(__builtin_bit_cast(float, x), __builtin_bit_cast(float, y));
}

// OCC: workgroups of a CU at least
template <int ELEM, int D, int NQ, int OCC>
__global__ __launch_bounds__(256, OCC) void attn_step_kernel(AttnArgs a, AttnPlan plan, float c, unsigned flip)
{
    constexpr int BM = 16 * NQ, NW = 4;
    constexpr int TOK = ELEM == 2 ? 32 : 64;                         // tokens of a wavefront's turn: 64 bytes of every lane's keys and values at D = 128
    constexpr int ST = TOK / 16, KT = D / 32, ET = D / 16;           // score tiles of 16 tokens, steps of 32 channels, output tiles of 16
    constexpr int KL = ST * KT / (ELEM == 2 ? 1 : 2), VL = ET;       // 16-byte loads of a lane
    constexpr int EP = ET < 8 / NQ ? ET : 8 / NQ;                    // output tiles that the wavefronts add up at a time
    static_assert(ET % EP == 0, "whole passes");
    __shared__ __attribute__((aligned(16))) float sums[NW][NQ * EP * 256];
    __shared__ __attribute__((aligned(16))) float scales[ELEM == 1 ? NW : 1][ELEM == 1 ? 3 * TOK : 1];
    __shared__ float sm[NW][BM], sl[NW][BM];
    __shared__ AttnScratch scratch;

    const int kvh = blockIdx.x % a.kv.heads, index = blockIdx.x / a.kv.heads;
    AttnItem it;
    if (!attn_take<NW * 64, BM>(a, plan, index, kvh, scratch, it)) return;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, qd = lane >> 4;
    const int row0 = it.tile * BM;
    auto position = [&](int r) { return (int)min(max((int64_t)it.r.ctx + attn_token(a, r), (int64_t)-1), (int64_t)INT32_MAX); };
    const int pos0 = position(row0), pos1 = position(min(row0 + BM, it.r.rows) - 1);

    int low, high;
    attn_range(a, it.r, row0, min(row0 + BM, it.r.rows), low, high);
    attn_part_range(low, high, it.part, it.parts);
    low = __builtin_amdgcn_readfirstlane(low), high = __builtin_amdgcn_readfirstlane(high);

    int pos[NQ];
    h8 q[NQ][KT];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int row = row0 + 16 * n + col;
        const bool live = row < it.r.rows;
        const int token = live ? attn_token(a, row) : 0, head = kvh * a.group + (live ? row - token * a.group : 0);
        pos[n] = position(live ? row : 0);
        const __half *src = a.q + (int64_t)(it.r.cu + token) * a.ldq + (int64_t)head * D;
#pragma unroll
        for (int k = 0; k < KT; ++k) {
            const int d = ELEM == 2 ? 32 * k + 8 * qd : 64 * (k / 2) + 16 * qd + 8 * (k % 2);
            u4 v = {0, 0, 0, 0};
            if (live) v = *reinterpret_cast<const u4 *>(src + d);
            q[n][k] = as_h8(v ^ flip);
        }
    }

    // Turn i of this wavefront: tokens low + (i NW + wave) TOK ... The table's entries of 64 turns at a time, one per lane.
    const int32_t *row_of_table = a.table + (int64_t)it.b * a.ld_table;
    const int start = low + wave * TOK, turns = start < high ? (high - start - 1) / (NW * TOK) + 1 : 0;
    constexpr int PG = TOK / 32;
    int entries[PG];
    auto look_up = [&](int first) {
#pragma unroll
        for (int i = 0; i < PG; ++i) {
            const int64_t t = start + (int64_t)(first + lane) * NW * TOK + 32 * i;
            entries[i] = t < high ? row_of_table[t >> a.kv.page_shift] : -1;
        }
    };
    auto page_of = [&](int turn, int i) {
        const int p = __builtin_amdgcn_readlane(entries[i], turn & 63);
        return (unsigned)p < (unsigned)a.kv.pages ? p : -1;
    };
    auto token_of = [&](int turn) { return start + turn * NW * TOK; };

    // Which token a score tile's row is, and which channels a lane holds of it, is chosen so that the weights come out of the score tiles
    // as the values' product takes them, without a move between lanes:
    //   fp16  one block; tile t, row r: token 16 (r / 8) + 8 t + r % 8;                channels 32 k + 8 qd ...
    //   int8  two blocks; tile 2 s + t, row r: block r / 8, token 16 s + 8 t + r % 8;  channels 64 (k / 2) + 16 qd + 8 (k % 2) ...
    u4 kx[KL], vx[VL];
    float sx[3];
    const int key_at = (qd / 2) * 1024 + (qd % 2) * 512 + (col % 8) * 16 + (ELEM == 2 ? (col / 8) * 256 : 0);
    const int value_at = 32 * D * ELEM + (ELEM == 2 ? (qd / 2) * 1024 : 0) + (qd % 2) * 512 + col * 16;
    auto block_at = [&](int page, int t) { return a.kv.block(max(page, 0), kvh, t & (a.kv.page_size() - 1)); };
    auto load_keys = [&](int turn) {
        const int t = token_of(turn);
        const char *p0 = block_at(page_of(turn, 0), t) + key_at;
        if constexpr (ELEM == 2) {
#pragma unroll
            for (int i = 0; i < KL; ++i) kx[i] = *reinterpret_cast<const u4 *>(p0 + (i / ST) * 2048 + (i % ST) * 128);
        } else {
            const char *p1 = block_at(page_of(turn, PG - 1), t + 32) + key_at, *p = col / 8 ? p1 : p0;
#pragma unroll
            for (int i = 0; i < KL; ++i) kx[i] = *reinterpret_cast<const u4 *>(p + (i / ST) * 2048 + (i % ST) * 128);
            const float *s = reinterpret_cast<const float *>((lane / 32 ? p1 : p0) - key_at + kv_scale_offset(D)) + lane % 32;
            sx[0] = s[0], sx[1] = s[64], sx[2] = s[96];
        }
    };
    auto load_values = [&](int turn) {
        const int t = token_of(turn);
        const char *p = block_at(page_of(turn, 0), t) + value_at;
        if constexpr (ELEM == 1) {
            const char *p1 = block_at(page_of(turn, PG - 1), t + 32) + value_at;
            p = qd / 2 ? p1 : p;
        }
#pragma unroll
        for (int e = 0; e < VL; ++e) vx[e] = *reinterpret_cast<const u4 *>(p + (e / 2) * 1024 * ELEM + (e % 2) * 256);
    };

    f4 o[NQ][ET];
    constexpr bool RAW = ELEM == 2;                                  // scores and maxima still without the factor c
    const float factor = RAW ? c : 1.0f;
    float m[NQ], l[NQ];
    bool far[NQ];                                                    // of the wavefront: see ATTN_FAR
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = -INFINITY, l[n] = 0, far[n] = false;
#pragma unroll
        for (int e = 0; e < ET; ++e) o[n][e] = f4{0, 0, 0, 0};
    }
    float *sc = scales[ELEM == 1 ? wave : 0];

    if (turns) {
        look_up(0);
        load_keys(0);
        load_values(0);
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int k = 0; k < KT; ++k) q[n][k] = attn_query(q[n][k]);   // (behind the loads, which need not wait for them)
    }
    for (int i = 0; i < turns; ++i) {
        const int t = token_of(i);
        bool plain = t <= high - TOK && (!a.causal || (t + TOK - 1 <= pos0 && (!a.window || t > pos1 - a.window)));
        int page[PG];
#pragma unroll
        for (int b = 0; b < PG; ++b) page[b] = page_of(i, b), plain = plain && page[b] >= 0;
        const bool more = i + 1 < turns;

        f4 s[NQ][ST];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int x = 0; x < ST; ++x) s[n][x] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < KL; ++j) {
            if constexpr (ELEM == 2) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) s[n][j % ST] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(kx[j]), q[n][j / ST], s[n][j % ST], 0, 0, 0);
            } else {
                const h8 x0 = widen_codes(kx[j][0], kx[j][1]), x1 = widen_codes(kx[j][2], kx[j][3]);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    s[n][j % ST] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, q[n][2 * (j / ST)], s[n][j % ST], 0, 0, 0);
                    s[n][j % ST] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, q[n][2 * (j / ST) + 1], s[n][j % ST], 0, 0, 0);
                }
            }
        }
        // the token of element 0 of this lane in score tile x, from the turn's first
        auto token4 = [&](int x) { return ELEM == 2 ? 16 * (qd / 2) + 8 * x + 4 * (qd % 2) : 32 * (qd / 2) + 8 * x + 4 * (qd % 2); };
        if constexpr (ELEM == 1) {
            const bool there = t + lane < high && (lane / 32 ? page[PG - 1] : page[0]) >= 0;   // (behind: whatever memory held, NaN among it)
            sc[lane] = there ? sx[0] * c : 0.f, sc[TOK + lane] = there ? sx[1] : 0.f, sc[2 * TOK + lane] = there ? sx[2] : 0.f;
            asm volatile("" ::: "memory");   // (same wavefront, LDS operations complete in order: only the compiler must keep them so)
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int x = 0; x < ST; ++x) {
                const f4 sk = *reinterpret_cast<const f4 *>(sc + token4(x)), lv = *reinterpret_cast<const f4 *>(sc + TOK + token4(x));
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][x][j] = fmaf(s[n][x][j], sk[j], lv[j]);
            }
        }
        if (more) {
            if (((i + 1) & 63) == 0) look_up(i + 1);
            load_keys(i + 1);
        }
        if (!plain) {
            asm volatile("");                                        // or the compiler compares and selects in every turn
            const bool there = ELEM == 1 ? (qd / 2 ? page[PG - 1] : page[0]) >= 0 : page[0] >= 0;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int last = !there ? -1 : a.causal ? min(high - 1, pos[n]) : high - 1, first = a.window ? pos[n] - a.window : -1;
#pragma unroll
                for (int x = 0; x < ST; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int tk = t + token4(x) + j;
                        if (tk > last || tk <= first) s[n][x][j] = -INFINITY;
                    }
            }
            if constexpr (ELEM == 2) {                               // values behind the last token: 0 times NaN is not 0
                u4 clean = {~0u, ~0u, ~0u, ~0u};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(t + token4(j / 4) + j % 4 < high && there)) clean[j / 2] &= j % 2 ? 0x0000ffffu : 0xffff0000u;
#pragma unroll
                for (int e = 0; e < VL; ++e) vx[e] &= clean;
            }
        }
        h8 p[NQ][ELEM == 2 ? 1 : 2];
        float iv[ELEM == 1 ? ST * 4 : 1];
        if constexpr (ELEM == 1) {
#pragma unroll
            for (int x = 0; x < ST; ++x) {
                const f4 v = *reinterpret_cast<const f4 *>(sc + 2 * TOK + token4(x));
#pragma unroll
                for (int j = 0; j < 4; ++j) iv[4 * x + j] = v[j];
            }
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float top = s[n][0][0];
#pragma unroll
            for (int x = 0; x < ST; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, s[n][x][j]);
            top = over_quarters(top, [](float x, float y) { return fmaxf(x, y); });
            // The maximum follows only when a score exceeds it by 2^8: with ATTN_LEAD weights up to 2^15, and the sums are rarely rescaled.
            if (__any((top - m[n]) * factor > 8.0f)) {
                const float to = fmaxf(m[n], top), keep = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[n] - to) * factor);
                m[n] = to;
                far[n] = __any(attn_far(to, factor));
                l[n] *= keep;
#pragma unroll
                for (int e = 0; e < ET; ++e) o[n][e] *= keep;
            }
            float base = m[n] == -INFINITY ? 0.f : fmaf(-m[n], factor, ATTN_LEAD);
            if (far[n]) {
                asm volatile("");                                    // (a branch: hardly any call takes it)
                const float off = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
                for (int x = 0; x < ST; ++x)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[n][x][j] -= off;
                base = ATTN_LEAD;
            }
            unsigned w[ST * 2];
            float sum = 0;                                           // of the turn: a small weight is not lost beside all before it
#pragma unroll
            for (int x = 0; x < ST; ++x) {
                float e[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    e[j] = __builtin_amdgcn_exp2f(RAW ? fmaf(s[n][x][j], c, base) : s[n][x][j] + base);
                    sum = ELEM == 1 ? fmaf(e[j], iv[ELEM == 1 ? 4 * x + j : 0], sum) : sum + e[j];
                }
                w[2 * x] = pack2(e[0], e[1]), w[2 * x + 1] = pack2(e[2], e[3]);
            }
            l[n] += sum;
            p[n][0] = as_h8(u4{w[0], w[1], w[2], w[3]});
            if constexpr (ELEM == 1) p[n][1] = as_h8(u4{w[4], w[5], w[6], w[7]});
        }
#pragma unroll
        for (int e = 0; e < ET; ++e) {
            if constexpr (ELEM == 2) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(as_h8(vx[e]), p[n][0], o[n][e], 0, 0, 0);
            } else {
                const h8 x0 = widen_codes(vx[e][0], vx[e][1]), x1 = widen_codes(vx[e][2], vx[e][3]);
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    o[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x0, p[n][0], o[n][e], 0, 0, 0);
                    o[n][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x1, p[n][ELEM == 1 ? 1 : 0], o[n][e], 0, 0, 0);
                }
            }
        }
        if (more) load_values(i + 1);
        if constexpr (ELEM == 1) __builtin_amdgcn_wave_barrier();
    }

    // ---- the wavefronts' results together ----
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        l[n] = over_quarters(l[n], [](float x, float y) { return x + y; });
        if (qd == 0) sm[wave][16 * n + col] = m[n];
    }
    __syncthreads();
    float top[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        top[n] = fmaxf(fmaxf(sm[0][16 * n + col], sm[1][16 * n + col]), fmaxf(sm[2][16 * n + col], sm[3][16 * n + col]));
        const float w = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[n] - top[n]) * factor);
        l[n] *= w;
        if (qd == 0) sl[wave][16 * n + col] = l[n];
#pragma unroll
        for (int e = 0; e < ET; ++e) o[n][e] *= w;
    }
    const bool partial = it.parts > 1;
    float *out = partial ? attn_partial(a, plan, it.item, kvh) : nullptr;
#pragma unroll
    for (int e0 = 0; e0 < ET; e0 += EP) {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < EP; ++e) *reinterpret_cast<f4 *>(&sums[wave][((n * EP + e) * 64 + lane) * 4]) = o[n][e0 + e];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NQ * EP / NW; ++k) {                     // tile k NW + wave: rows col, channels 4 qd ...
            const int at = k * NW + wave, n = at / EP, e = e0 + at % EP, r = 16 * n + col, row = row0 + r;
            f4 v = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < NW; ++w) v += *reinterpret_cast<const f4 *>(&sums[w][(at * 64 + lane) * 4]);
            const float sum = (sl[0][r] + sl[1][r]) + (sl[2][r] + sl[3][r]);
            if (row < it.r.rows) {
                if (partial) {
                    *reinterpret_cast<f4 *>(out + (size_t)r * D + 16 * e + 4 * qd) = v;
                } else {
                    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
                    const int token = attn_token(a, row);
                    __half *dst = a.y + (int64_t)(it.r.cu + token) * a.ldy + (int64_t)(kvh * a.group + row - token * a.group) * D + 16 * e + 4 * qd;
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv));
                }
            }
        }
        __syncthreads();
    }
    if (partial && tid < BM) {
        float t = fmaxf(fmaxf(sm[0][tid], sm[1][tid]), fmaxf(sm[2][tid], sm[3][tid]));
        out[(size_t)BM * D + tid] = t, out[(size_t)BM * (D + 1) + tid] = (sl[0][tid] + sl[1][tid]) + (sl[2][tid] + sl[3][tid]);
    }
}

template <int ELEM, int D>
int launch(const AttnArgs &a, const AttnPlan &p, float c, unsigned flip, hipStream_t st)
{
    const unsigned grid = (unsigned)(p.items * a.kv.heads);
    if constexpr (D < 256) {
        if (p.bm == 32) {
            // (int8, D = 128, spills 15 registers; its reloads in the loop wait for the next turn's keys)
            attn_step_kernel<ELEM, D, 2, 2><<<grid, 256, 0, st>>>(a, p, c, flip);
            return check_hip(hipGetLastError(), "attn_step_kernel");
        }
    }
    // D = 256: one workgroup a CU with registers for all, but two where requests are short and their workgroups wait more than they load (fp16 spills
    // three registers there, int8 many; us, one / two; 8 heads, 126 requests of 40, 250 and 900 tokens: fp16 38.5 / 23.6, 68.5 / 59.0, 170 / 171, 32 of 200..4096 114 / 124; int8
    // 40 / 27, 54 / 54, 109 / 145).
    if (D < 256 || (ELEM == 2 && p.step == 2)) attn_step_kernel<ELEM, D, 1, ELEM == 1 && D == 256 ? 1 : 2><<<grid, 256, 0, st>>>(a, p, c, flip);
    else attn_step_kernel<ELEM, D, 1, D == 256 ? 1 : 2><<<grid, 256, 0, st>>>(a, p, c, flip);
    return check_hip(hipGetLastError(), "attn_step_kernel");
}

}  // namespace

int launch_attention_steps(const AttnArgs &a, const AttnPlan &p, float c, hipStream_t st)
{
    const unsigned flip = a.scale < 0 ? 0x80008000u : 0u;
    if (a.kv.bits == 16) {
        if (a.kv.D == 64) return launch<2, 64>(a, p, c, flip, st);
        if (a.kv.D == 128) return launch<2, 128>(a, p, c, flip, st);
        return launch<2, 256>(a, p, c, flip, st);
    }
    if (a.kv.D == 64) return launch<1, 64>(a, p, c, flip, st);
    if (a.kv.D == 128) return launch<1, 128>(a, p, c, flip, st);
    return launch<1, 256>(a, p, c, flip, st);
}

}  // namespace ql
