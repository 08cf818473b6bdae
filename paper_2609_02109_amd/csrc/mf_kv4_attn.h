// Attention over the paged 4-bit cache (the kernel; mf_kv4_attn.hip plans and
// launches it).  One pass over the tokens with a running maximum and sum.
//
// A wave holds RT tiles of 16 rows (row = query token x head of the group that
// shares a key head).  The codes are matrix operands as they are: a 16-bit float
// whose bits are the whole number c is the subnormal c 2^-24 (binary16, up to c =
// 2047) or c 2^-133 (bfloat16, up to 255), which the matrix instructions take
// exactly and at full rate.  So one and makes two operands of a dword, the codes
// at bits 0.. of each half, and one more those at bits 4.., 16 times as large: 5
// operations for 8 codes where a conversion to 16 + c took 8 and a sum to take the
// 16 out again.  Per 16 tokens S^T = K Q^T, and per group of G dims
//   s = sum_g scale_g sum_d c q + off_g sum_d q,
// the queries taken 2^e times first (their largest at the top of the type's range;
// 2^-4 of that where they meet the larger codes), and the last sum over g a matrix
// product itself (sum q in two binary16 pieces, 22 bits).  S^T comes out with the
// tokens 4 (l / 16) + r of row l % 16 in lane l, which is how the next product
// O^T = V^T P^T takes its right operand: softmax weights stay in their lane.
//   o = sum_t w c + sum_t p off_g,   w = p scale_g,
// p and w rounded to binary16 (11 bits; everything else is fp32).  Weights are
// kept relative to 2^base.  The largest score is looked for only where a weight
// shows that it is needed: a step's weights are computed with the base at hand,
// and when one reaches 2^14, so that w could leave binary16's range, the base goes
// to the largest score so far (in powers of two) less 10 and the step's weights
// are computed again.  Binary16 then holds weights down to 2^-34 of the largest,
// and the small weights of long contexts are not lost; a step's w are brought to
// the same range by a power of two where scales are not of ordinary size.
#pragma once

#include "mf_serve_dev.h"

namespace mfs {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uniform(long long x)
{
    return (long long)((unsigned long long)(unsigned)uniform((int)(x >> 32)) << 32 | (unsigned)uniform((int)x));
}
// What a row sees: tokens lo .. hi.
struct Sight {
    int lo, hi;
};
__device__ __forceinline__ Sight sight_of(long long p, int window, int limit)
{
    Sight v;
    v.hi = p < limit ? (int)(p < -1 ? -1 : p) : limit - 1;
    const long long lo = window > 0 ? p - window + 1 : 0;
    v.lo = lo <= 0 ? 0 : lo < limit ? (int)lo : limit;
    return v;
}

// What a wave keeps for its rows: lane l's is row l % 16 of each tile.
constexpr float kNoBase = -1e30f;   // before the first token; finite, so that differences of bases are
template <int D, int G, int RT>
struct AttnState {
    static constexpr int DT = D / 16, NG = D / G;
    f32x4 o[RT][DT];      // sum w c, 2^-24 (even t) or 2^-20 times: dims 16 t + 4 (l / 16) + r
    f32x4 om[RT];         // sum p off: element r is group (4 (l / 16) + r) % NG
    float base[RT], l[RT];   // weights are relative to 2^base; sum of p over the lane's tokens
};

// A step's 32 tokens as a lane holds them (mf_serve.h; u: the block of 16).
template <int D, int G>
struct AttnTokens {
    static constexpr int NS = D / 32, NG = D / G;
    Words<NS> kc[2], vc[2];      // codes
    Words<2 * NG> ks[2], vs[2];  // scales of tokens 4 (l / 16) .. + 3, two words a group
    u32x2 ko[2];                 // key offsets of token l % 16: a left operand's pairs of groups
    u32x2 vo[2];                 // value offsets of group l % NG, tokens 4 (l / 16) .. + 3
};

template <int D, int G>
__device__ __forceinline__ void load_keys(AttnTokens<D, G> &x, int u, const uint8_t *rec, int lane)
{
    constexpr int NS = D / 32, NG = D / G;
    const int col = lane & 15, qt = lane >> 4;
    const uint8_t *t = rec + 16 * D;
    x.kc[u] = load_words<NS>(rec + lane * (D / 8));
    x.ks[u] = load_words<2 * NG>(t + qt * 16 * NG);
    const uint8_t *ko = t + 64 * NG + col * 2 * NG;
    if constexpr (NG == 1) x.ko[u] = (u32x2){*(const uint16_t *)ko, 0};
    if constexpr (NG == 2) x.ko[u] = (u32x2){*(const uint32_t *)ko, 0};
    if constexpr (NG == 4) x.ko[u] = *(const u32x2 *)ko;
    if constexpr (NG == 8) x.ko[u] = *(const u32x2 *)(ko + (qt & 1) * 8);
}
template <int D, int G>
__device__ __forceinline__ void load_values(AttnTokens<D, G> &x, int u, const uint8_t *rec, int lane)
{
    constexpr int NS = D / 32, NG = D / G;
    const int col = lane & 15, qt = lane >> 4;
    const uint8_t *t = rec + 16 * D;
    x.vc[u] = load_words<NS>(rec + 8 * D + lane * (D / 8));
    x.vs[u] = load_words<2 * NG>(t + qt * 16 * NG + 8 * NG);
    x.vo[u] = *(const u32x2 *)(t + 96 * NG + (col & (NG - 1)) * 32 + qt * 8);
}

// A dword's codes as an operand: pairs 0 and 2 as they are, pairs 1 and 3 16 times.
__device__ __forceinline__ u32x4 code_operand(uint32_t w)
{
    const uint32_t v = w >> 8;
    return (u32x4){w & 0x000f000fu, w & 0x00f000f0u, v & 0x000f000fu, v & 0x00f000f0u};
}
// A score in the units of the products, over its true value, is 2^-L times this; 2^L <= the row's largest query < 2^(L + 1).
template <bool F16>
constexpr float kQueryUnit = F16 ? 0x1p-9f : 0x1p-7f;   // 2^(15 - 24), 2^(126 - 133)

__device__ __forceinline__ float half_of(uint32_t w, int hi) { return (float)bits<f16x2>(w)[hi]; }

// Whether a row sees the lane's token e (0..7) of a step; ok: bit u says that block u lies in a page of the cache.
__device__ __forceinline__ bool sees(const Sight &v, int ok, int t0, int qt, int e)
{
    const int tok = t0 + 16 * (e >> 2) + 4 * qt + (e & 3);
    return (ok >> (e >> 2) & 1) && tok >= v.lo && tok <= v.hi;
}

// Of tokens 2 e, 2 e + 1 of the lane's, the halves that a row sees.
__device__ __forceinline__ uint32_t seen_pair(const Sight &v, int ok, int t0, int qt, int e)
{
    return (sees(v, ok, t0, qt, 2 * e) ? 0xffffu : 0u) | (sees(v, ok, t0, qt, 2 * e + 1) ? 0xffff0000u : 0u);
}

// The largest of a row's eight numbers a lane, as whole numbers of 16 bits.
__device__ __forceinline__ uint32_t largest(u32x4 v)
{
    const u16x2 m = __builtin_elementwise_max(__builtin_elementwise_max(bits<u16x2>(v[0]), bits<u16x2>(v[1])),
                                              __builtin_elementwise_max(bits<u16x2>(v[2]), bits<u16x2>(v[3])));
    return (uint32_t)quarters_max((float)max(m[0], m[1]));
}

// Scales of 2^-7 (bit 13) up to 2 (bit 14), and 0, leave the products with the weights well inside binary16's range.
// Of eight scales a lane, turned by kPlain: above kPlain where one is of another size.
constexpr uint32_t kPlain = 0x2000;
__device__ __forceinline__ u16x2 plainness(uint32_t scales) { return bits<u16x2>(scales ^ (kPlain | kPlain << 16)); }

// The power of two that a row's scales of a group (scales: of the tokens that it sees, others 0) are taken times: their
// products with the weights w, and they, come to the top of binary16's range, below 2^15.  0 where all are plain.
__device__ __forceinline__ int unit_of(u32x4 scales, u32x4 w)
{
    u32x4 products, turned;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        products[e] = bits<uint32_t>(bits<f16x2>(w[e]) * bits<f16x2>(scales[e]));
        turned[e] = bits<uint32_t>(plainness(scales[e]));
    }
    const bool plain = largest(turned) <= kPlain;
    const int scale = (int)(largest(scales) >> 10) - 15, weight = (int)(largest(w) >> 10) - 15, product = (int)(largest(products) >> 10) - 15;
    // past binary16's range a product is at most its largest factors'; 2^15 is the largest that the scales are taken times
    return plain ? 0 : min(min(14 - scale, 15), 14 - (product < 16 ? product : scale + weight + 1));
}

// keys_done, values_done: called where the step has no more use for its keys and its values, to
// fetch the next step's into their place.  full: every row sees every token; all: what any row sees, for the memory
// of the others may hold anything; c: softmax scale times log2 e (and the row's power of two).
template <bool F16, int D, int G, int RT, class FK, class FV>
__device__ __forceinline__ void attn_step(AttnState<D, G, RT> &st, const u32x4 (&q)[RT][D / 32], const u32x2 (&qsum)[RT],
                                          const AttnTokens<D, G> &x, const Sight (&see)[RT],
                                          bool full, int ok, const Sight &all, int t0, const float (&c)[RT],
                                          const FK &keys_done, const FV &values_done)
{
    constexpr int NG = D / G, IPG = G / 32;
    const int qt = (threadIdx.x & 63) >> 4;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    float p[RT][2][4];
#pragma unroll
    for (int u = 0; u < 2; u++) {
        f32x4 sc[RT];
#pragma unroll
        for (int t = 0; t < RT; t++) {
            sc[t] = __builtin_amdgcn_mfma_f32_16x16x16f16(bits<f16x4>(x.ko[u]), bits<f16x4>(qsum[t]), zero, 0, 0, 0);
            if (F16) sc[t] *= kQueryUnit<true>;
        }
#pragma unroll
        for (int g = 0; g < NG; g++) {
            f32x4 P[RT];
#pragma unroll
            for (int i = 0; i < IPG; i++) {
                const u32x4 A = code_operand(x.kc[u].w[g * IPG + i]);
#pragma unroll
                for (int t = 0; t < RT; t++) P[t] = mfma<F16>(A, q[t][g * IPG + i], i ? P[t] : zero);
            }
#pragma unroll
            for (int t = 0; t < RT; t++)
#pragma unroll
                for (int r = 0; r < 4; r++) sc[t][r] = fmaf(half_of(x.ks[u].w[2 * g + (r >> 1)], r & 1), P[t][r], sc[t][r]);
        }
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int r = 0; r < 4; r++) p[t][u][r] = sc[t][r];
    }
    keys_done();
    if (!full) {
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (!sees(see[t], ok, t0, qt, e)) p[t][e >> 2][e & 3] = -INFINITY;
    }
    u32x4 w[RT];
    float e[RT][8];
    for (bool raised = false;; raised = true) {   // twice at most
        int highest[RT], over = 0;
        constexpr int most = (15 + 14) << 10;   // 2^14 in binary16
#pragma unroll
        for (int t = 0; t < RT; t++) {
#pragma unroll
            for (int i = 0; i < 8; i++) e[t][i] = __builtin_amdgcn_exp2f(fmaf(p[t][i >> 2][i & 3], c[t], -st.base[t]));
#pragma unroll
            for (int i = 0; i < 4; i++) w[t][i] = pack2<true>(e[t][2 * i], e[t][2 * i + 1]);
            // none is negative: as whole numbers they are in the same order
            const u16x2 high = __builtin_elementwise_max(__builtin_elementwise_max(bits<u16x2>(w[t][0]), bits<u16x2>(w[t][1])),
                                                         __builtin_elementwise_max(bits<u16x2>(w[t][2]), bits<u16x2>(w[t][3])));
            highest[t] = max(high[0], high[1]);
            over = max(over, highest[t]);
        }
        if (raised || !__any(over >= most)) break;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            // only the rows that need it, so that no row's result depends on another's
            const bool hit = quarters_max((float)highest[t]) >= (float)most;
            float mx = p[t][0][0];
#pragma unroll
            for (int i = 1; i < 8; i++) mx = fmaxf(mx, p[t][i >> 2][i & 3]);
            mx = fmaf(quarters_max(mx), c[t], -10.f);
            const float base = hit ? fmaxf(mx, st.base[t]) : st.base[t], a = __builtin_amdgcn_exp2f(st.base[t] - base);
            st.base[t] = base;
            st.l[t] *= a;
            st.om[t] *= a;
#pragma unroll
            for (int d = 0; d < D / 16; d++) st.o[t][d] *= a;
        }
    }
#pragma unroll
    for (int t = 0; t < RT; t++)
#pragma unroll
        for (int i = 0; i < 8; i++) st.l[t] += e[t][i];
    u32x4 vo = {x.vo[0][0], x.vo[0][1], x.vo[1][0], x.vo[1][1]};
    u16x2 turned = {0, 0};   // above kPlain where some row sees a scale that is not plain
#pragma unroll
    for (int g = 0; g < NG; g++)
#pragma unroll
        for (int e = 0; e < 4; e++) turned = __builtin_elementwise_max(turned, plainness(x.vs[e >> 1].w[2 * g + (e & 1)]));
    if (!full) {
        // what no row sees may be anything, not a number too; a zero weight does not make it zero
        turned = (u16x2){0, 0};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const uint32_t seen = seen_pair(all, ok, t0, qt, e);
            vo[e] &= seen;
#pragma unroll
            for (int g = 0; g < NG; g++) turned = __builtin_elementwise_max(turned, plainness(x.vs[e >> 1].w[2 * g + (e & 1)] & seen));
        }
    }
#pragma unroll
    for (int t = 0; t < RT; t++) st.om[t] = mfma<true>(vo, w[t], st.om[t]);
    // Scales of 2 and above may take w out of binary16's range, scales below 2^-7 to its end, where it has few bits or
    // none; both are rare.  Where a row sees one, the group's scales of this step and the sums that the products go
    // into are taken 2^up times, and the sums back: per row, and of the scales that the row sees, so that no row's
    // result depends on anything else.
    const bool odd = __any(max(turned[0], turned[1]) > kPlain);
    int up[RT][NG];
#pragma unroll
    for (int g = 0; g < NG; g++) {
        u32x4 wg[RT];
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int e = 0; e < 4; e++) wg[t][e] = bits<uint32_t>(bits<f16x2>(w[t][e]) * bits<f16x2>(x.vs[e >> 1].w[2 * g + (e & 1)]));
        if (odd || !full) {   // nor do scales of tokens that the row does not see
#pragma unroll
            for (int t = 0; t < RT; t++) {
                u32x4 scales;
#pragma unroll
                for (int e = 0; e < 4; e++) scales[e] = x.vs[e >> 1].w[2 * g + (e & 1)] & (full ? ~0u : seen_pair(see[t], ok, t0, qt, e));
                if (odd) {
                    up[t][g] = unit_of(scales, w[t]);
                    const _Float16 f = (_Float16)__builtin_amdgcn_ldexpf(1.f, up[t][g]);
#pragma unroll
                    for (int e = 0; e < 4; e++) scales[e] = bits<uint32_t>(bits<f16x2>(scales[e]) * (f16x2){f, f});
#pragma unroll
                    for (int d = g * (G / 16); d < (g + 1) * (G / 16); d++)
#pragma unroll
                        for (int r = 0; r < 4; r++) st.o[t][d][r] = __builtin_amdgcn_ldexpf(st.o[t][d][r], up[t][g]);
                }
#pragma unroll
                for (int e = 0; e < 4; e++) wg[t][e] = bits<uint32_t>(bits<f16x2>(w[t][e]) * bits<f16x2>(scales[e]));
            }
        }
#pragma unroll
        for (int i = g * IPG; i < (g + 1) * IPG; i++) {
            const u32x4 a = code_operand(x.vc[0].w[i]), b = code_operand(x.vc[1].w[i]);
            const u32x4 lo = {a[0], a[2], b[0], b[2]}, hi = {a[1], a[3], b[1], b[3]};
#pragma unroll
            for (int t = 0; t < RT; t++) {
                st.o[t][2 * i] = mfma<true>(lo, wg[t], st.o[t][2 * i]);
                st.o[t][2 * i + 1] = mfma<true>(hi, wg[t], st.o[t][2 * i + 1]);
            }
        }
    }
    if (odd) {
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int d = 0; d < D / 16; d++)
#pragma unroll
                for (int r = 0; r < 4; r++) st.o[t][d][r] = __builtin_amdgcn_ldexpf(st.o[t][d][r], -up[t][d * 16 / G]);
    }
    values_done();
}

// A sequence of the batch as far as it lies in the step's rows and the cache,
// whatever the device arrays hold.
struct SeqRows {
    int q0, n;            // first row, rows
    int limit;            // tokens of the cache that may be read
    long long first_p;    // position of the first row
};
// The batch's numbers of a sequence, and what they come to.
struct SeqRaw {
    int q0, q1, kv;
};
__device__ __forceinline__ SeqRaw seq_raw(const KvBatch &b, int s) { return {b.q_start[s], b.q_start[s + 1], b.kv_len[s]}; }
__device__ __forceinline__ SeqRows seq_rows(const KvBatch &b, const SeqRaw &w)
{
    SeqRows r;
    r.q0 = w.q0;
    r.limit = max(0, min(w.kv, b.max_kv));
    r.first_p = (long long)w.kv - ((long long)w.q1 - w.q0);
    // max_new: a workgroup's rows and the parts' room are made for it
    r.n = w.q0 < 0 || w.q0 >= b.rows || w.q1 <= w.q0 ? 0 : min(min(w.q1, b.rows) - w.q0, b.max_new);
    return r;
}

// Tokens [from, to) that rows i0 .. i1 of a sequence see, from on a step's bound.
struct Range {
    int from, to;
};
__device__ __forceinline__ Range range_of(const SeqRows &r, int i0, int i1, int window)
{
    return {sight_of(r.first_p + i0, window, r.limit).lo & ~(kAttnStep - 1), sight_of(r.first_p + i1, window, r.limit).hi + 1};
}

// Units of kAttnUnit tokens that one head of a sequence takes: one at least
// where there are rows, for someone has to write them.
__device__ __forceinline__ int units_of(const KvAttnArgs &a, const SeqRaw &w)
{
    const SeqRows r = seq_rows(a.b, w);
    if (r.n == 0) return 0;
    const Range t = range_of(r, 0, r.n - 1, a.window);
    return t.to > t.from ? (t.to - t.from + kAttnUnit - 1) / kAttnUnit : 1;
}

__device__ __forceinline__ int wave_scan(int x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// 64 sequences as the lanes hold them: units of one head, and those up to and with the lane's.
struct Lanes {
    SeqRaw raw;
    int units, upto, all;
};
__device__ __forceinline__ Lanes lanes_at(const KvAttnArgs &a, int s0, int lane)
{
    Lanes l = {{0, 0, 0}, 0, 0, 0};
    if (s0 + lane < a.b.n_seq) {
        l.raw = seq_raw(a.b, s0 + lane);
        l.units = units_of(a, l.raw);
    }
    l.upto = wave_scan(l.units, lane);
    l.all = __builtin_amdgcn_readlane(l.upto, 63);
    return l;
}

// Rows row0 .. of one sequence and key head over its tokens [begin, end):
// into the output (slot < 0) or a slot of the parts.
// NW: waves that share the rows and take different tokens; 0: the wave has rows of its own.
// AHEAD: a step's keys and values are fetched where the step before has no more use for its
// own, which takes some 20 registers.
template <bool F16, int D, int G, int RT, int NW, bool AHEAD>
__device__ __forceinline__ void attn_item(const KvAttnArgs &a, int s, int h, const SeqRows &sr, int row0, int row_end, int begin, int end,
                                          long long slot)
{
    constexpr int NS = D / 32, NG = D / G, IPG = G / 32, DT = D / 16;
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int last = min(row_end, row0 + RT * 16) - 1, limit = sr.limit;

    // rows past the last are computed as the last and not stored
    u32x4 q[RT][NS];
    Sight see[RT];
    int qrow[RT], qhead[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int r = min(row0 + 16 * t + col, last);
        const int i = r / a.per_kv;
        qrow[t] = sr.q0 + i;
        qhead[t] = h * a.per_kv + (r - i * a.per_kv);
        see[t] = sight_of(sr.first_p + i, a.window, limit);
        const uint16_t *x = (const uint16_t *)a.q + (long long)qrow[t] * a.q_stride + (long long)qhead[t] * a.q_head + qt * 8;
#pragma unroll
        for (int d = 0; d < NS; d++) q[t][d] = load16(x + 32 * d);
    }
    const Sight see0 = sight_of(sr.first_p + row0 / a.per_kv, a.window, limit), see1 = sight_of(sr.first_p + last / a.per_kv, a.window, limit);
    const Sight all = {see0.lo, see1.hi};

    const int *table = a.b.table + (long long)s * a.b.table_stride;
    constexpr bool ROWS = NW == 0;
    constexpr int STRIDE = kAttnStep * (ROWS ? 1 : NW);
    // Where the records of the next 32 steps start, in bytes: lane 2 i + u has block u
    // of step i, -1 where there is none.  One gather for 32 steps: a page number
    // that is fetched for the step at hand costs it a trip to memory.
    long long starts;
    const auto find = [&](int t0) {
        const int at = t0 + (lane >> 1) * STRIDE, blk = (at >> 4) + (lane & 1);
        starts = -1;
        if (at < end && blk * kKvBlock < limit) {
            const int pc = page_of_block(a.g, blk), page = table[pc];
            if ((unsigned)page < (unsigned)a.g.n_pages)
                starts = (((long long)page * a.g.n_kv_heads + h) * a.g.blocks_per_page + (blk - pc * a.g.blocks_per_page)) * a.g.rec;
        }
    };
    const auto start_of = [&](int l) {
        return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(starts >> 32), l) << 32 |
                           (unsigned)__builtin_amdgcn_readlane((int)starts, l));
    };
    // a step's records, and which of them there are; where there is none the first one is read, and masked
    struct Step {
        const uint8_t *rec[2];
        int ok;
    };
    const auto step_at = [&](int i) {
        Step r;
        r.ok = 0;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const long long at = start_of(2 * i + u);
            r.ok |= (at >= 0) << u;
            r.rec[u] = a.g.pages + (at < 0 ? 0 : at);
        }
        return r;
    };
    // the first step's records are on their way while the queries are made ready
    int t0 = begin + (ROWS ? 0 : wave * kAttnStep), i = 0;
    AttnTokens<D, G> x;
    Step now = {{a.g.pages, a.g.pages}, 0};
    if (t0 < end) {
        find(t0);
        now = step_at(0);
#pragma unroll
        for (int u = 0; u < 2; u++) load_keys(x, u, now.rec[u], lane);
#pragma unroll
        for (int u = 0; u < 2; u++) load_values(x, u, now.rec[u], lane);
    }

    u32x2 qsum[RT];        // sum q as the right operand of the offsets' product: its pieces
    float c[RT];
    AttnState<D, G, RT> st;
#pragma unroll
    for (int t = 0; t < RT; t++) {
        float qs[NG], big = 0.f;
#pragma unroll
        for (int g = 0; g < NG; g++) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < IPG; i++) x = mfma<F16>(ones8<F16>(), q[t][g * IPG + i], x);
            qs[g] = x[0];
        }
#pragma unroll
        for (int d = 0; d < NS; d++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                big = fmaxf(big, fmaxf(fabsf(to_float<F16>((uint16_t)q[t][d][j])), fabsf(to_float<F16>((uint16_t)(q[t][d][j] >> 16)))));
        const int L = max((int)(__float_as_uint(quarters_max(big)) >> 23), 1) - 127, up = (F16 ? 15 : 126) - L;
#pragma unroll
        for (int d = 0; d < NS; d++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                q[t][d][j] = pack2<F16>(__builtin_amdgcn_ldexpf(to_float<F16>((uint16_t)q[t][d][j]), up - 4 * (j & 1)),
                                        __builtin_amdgcn_ldexpf(to_float<F16>((uint16_t)(q[t][d][j] >> 16)), up - 4 * (j & 1)));
        // never 0: times the score of a token that is not seen, minus infinity, that would be a NaN
        c[t] = fmaxf(__builtin_amdgcn_ldexpf(a.scale_log2 / kQueryUnit<F16>, L), 0x1p-126f);
        f16x4 piece = {(_Float16)0.f, (_Float16)0.f, (_Float16)0.f, (_Float16)0.f};
#pragma unroll
        for (int g = 0; g < NG; g++) {
            // binary16's sums in units of 2^L (a piece of 2^-9 of them would be subnormal; attn_step makes up for it)
            const float x = __builtin_amdgcn_ldexpf(F16 ? qs[g] : qs[g] * kQueryUnit<false>, -L);
            const _Float16 hi = (_Float16)x, lo = (_Float16)(x - (float)hi);
            if (NG <= 4) {
                if (qt == 0) piece[g & 3] = hi;
                if (qt == 1) piece[g & 3] = lo;
            } else {
                if (qt == g / 4) piece[g & 3] = hi;
                if (qt == 2 + g / 4) piece[g & 3] = lo;
            }
        }
        qsum[t] = bits<u32x2>(piece);
        st.om[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        st.base[t] = kNoBase;
        st.l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; d++) st.o[t][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    const auto keys_of = [&](const Step &r) {
#pragma unroll
        for (int u = 0; u < 2; u++) load_keys(x, u, r.rec[u], lane);
    };
    const auto values_of = [&](const Step &r) {
#pragma unroll
        for (int u = 0; u < 2; u++) load_values(x, u, r.rec[u], lane);
    };
    while (t0 < end) {
        const bool full = now.ok == 3 && t0 >= see1.lo && t0 + kAttnStep - 1 <= see0.hi;
        if (++i == 32 && AHEAD) {
            find(t0 + STRIDE);
            i = 0;
        }
        if constexpr (AHEAD) {
            const Step next = step_at(i);   // past the end: records that are none
            attn_step<F16, D, G, RT>(st, q, qsum, x, see, full, now.ok, all, t0, c, [&] { keys_of(next); }, [&] { values_of(next); });
            now = next;
        } else {
            attn_step<F16, D, G, RT>(st, q, qsum, x, see, full, now.ok, all, t0, c, [] {}, [] {});
            if (t0 + STRIDE < end) {
                if (i == 32) {
                    find(t0 + STRIDE);
                    i = 0;
                }
                now = step_at(i);
                keys_of(now);
                values_of(now);
            }
        }
        t0 += STRIDE;
    }

    // the lanes' own sums together; o: the values' weighted sum
#pragma unroll
    for (int t = 0; t < RT; t++) {
        st.l[t] = quarters_sum(st.l[t]);
#pragma unroll
        for (int g = 0; g < NG; g++) {
            float om = st.om[t][g & 3];
            if (NG == 8) {
                const float far = __shfl_xor(om, 16);
                if ((qt & 1) != g / 4) om = far;
            }
#pragma unroll
            for (int d = g * (G / 16); d < (g + 1) * (G / 16); d++)
#pragma unroll
                for (int r = 0; r < 4; r++) st.o[t][d][r] = fmaf(st.o[t][d][r], d & 1 ? 0x1p20f : 0x1p24f, om);
        }
    }
    if constexpr (!ROWS) {
        // the upper half of the waves hands over to the lower, and so on
        __shared__ f32x4 so[NW / 2][RT * DT][64];
        __shared__ f32x2 sm[NW / 2][RT][64];
#pragma unroll
        for (int half = NW / 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int t = 0; t < RT; t++) {
                    sm[wave - half][t][lane] = (f32x2){st.base[t], st.l[t]};
#pragma unroll
                    for (int d = 0; d < DT; d++) so[wave - half][t * DT + d][lane] = st.o[t][d];
                }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int t = 0; t < RT; t++) {
                    const f32x2 other = sm[wave][t][lane];
                    const float base = fmaxf(st.base[t], other[0]);
                    const float x = __builtin_amdgcn_exp2f(st.base[t] - base), y = __builtin_amdgcn_exp2f(other[0] - base);
                    st.base[t] = base;
                    st.l[t] = st.l[t] * x + other[1] * y;
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        const f32x4 v = so[wave][t * DT + d][lane];
#pragma unroll
                        for (int r = 0; r < 4; r++) st.o[t][d][r] = st.o[t][d][r] * x + v[r] * y;
                    }
                }
            }
            __syncthreads();
        }
        if (wave != 0) return;
    }
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int r = row0 + 16 * t + col;
        if (r > last) continue;
        if (slot < 0) {
            const bool none = st.l[t] == 0.f;   // no token; a NaN stays one
            const float inv = none ? 0.f : 1.f / st.l[t];
            uint16_t *y = (uint16_t *)a.out + (long long)qrow[t] * a.out_stride + (long long)qhead[t] * a.out_head + qt * 4;
#pragma unroll
            for (int d = 0; d < DT; d++) {
                const f32x4 v = st.o[t][d] * inv;
                const u32x2 o = {pack2<F16>(v[0], v[1]), pack2<F16>(v[2], v[3])};
                __builtin_memcpy(__builtin_assume_aligned(y + 16 * d, 2), &o, 8);
            }
            if (a.lse && qt == 0)
                a.lse[(long long)qrow[t] * a.n_heads + qhead[t]] =
                    none ? -INFINITY : (st.base[t] + __builtin_amdgcn_logf(st.l[t])) * 0.69314718055994531f;
        } else {
            const long long at = slot * a.slot_rows + (ROWS ? r % a.slot_rows : r);
            float *y = a.part + at * D + qt * 4;
#pragma unroll
            for (int d = 0; d < DT; d++) *(f32x4 *)(y + 16 * d) = st.o[t][d];
            if (qt == 0) ((f32x2 *)(a.part + (long long)a.slots * a.slot_rows * D))[at] = (f32x2){st.base[t], st.l[t]};
        }
    }
}

// By rows (many query tokens; bound by vector instructions, 68 % of the SIMDs' cycles
// beside 34 % of matrix ones: 2 x 1024 query tokens of 32 heads over 12345 tokens take 545 us,
// 721 TFLOP/s; a third tile of rows a wave would share the codes' work further and has no
// registers): a workgroup takes a tile of attn_rows rows, its
// waves 16 RT of them each, over a part of their tokens.
template <bool F16, int D, int G, int RT>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn_rows_kernel(KvAttnArgs a)
{
    constexpr int WG_ROWS = attn_rows(RT, true);
    const int wg = a.first + (int)blockIdx.x, split = wg % a.splits, item = wg / a.splits;
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
    const int row_end = (int)min((long long)sr.n * a.per_kv, (long long)(tile + 1) * WG_ROWS);
    const int row0 = tile * WG_ROWS + wave_id() * RT * 16;
    if (row0 >= row_end) return;
    const Range t = range_of(sr, row0 / a.per_kv, (min(row_end, row0 + RT * 16) - 1) / a.per_kv, a.window);
    const long long part = t.from + (long long)split * a.chunk;
    const int begin = (int)min(part, (long long)t.to), end = split + 1 == a.splits ? t.to : (int)min(part + a.chunk, (long long)t.to);
    attn_item<F16, D, G, RT, 0, true>(a, s, h, sr, row0, row_end, begin, end, a.splits == 1 ? -1 : (long long)item * a.splits + split);
}

// By tokens (few rows: 16 RT at most of a sequence and key head; long contexts are bound by
// the cache's bytes, 2 x 131072 tokens of 8 heads of 128 in 51 us of kernel, 5.4 TB/s; ragged
// batches by the items' beginnings and ends too, 32 requests of up to 16384 in 85 us beside a join
// of 6, 3.8 TB/s; one short request by the chain of one wave's steps, 1000 tokens in 11 us: a second
// step on its way ahead and 16 waves were both slower): the waves of a
// workgroup take every fourth step each.  Whole: a workgroup per sequence and
// head.  Otherwise a.workgroups of them, as many as the card holds, take equal
// shares of all sequences' tokens: a share may end inside a head, whose parts
// the join adds up; slot 2 w is for a head that workgroup w found begun, 2 w + 1
// for one that it leaves unfinished.
template <bool F16, int D, int G, int RT, int NW, bool WHOLE>
__global__ __launch_bounds__(NW * 64, 2) void attn_tokens_kernel(KvAttnArgs a)
{
    if constexpr (WHOLE) {
        const int wg = a.first + (int)blockIdx.x, h = wg % a.g.n_kv_heads, s = wg / a.g.n_kv_heads;
        const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
        if (sr.n == 0) return;
        const Range t = range_of(sr, 0, sr.n - 1, a.window);
        attn_item<F16, D, G, RT, NW, RT == 1>(a, s, h, sr, 0, sr.n * a.per_kv, t.from, t.to, -1);
        return;
    }
    const int lane = threadIdx.x & 63, heads = a.g.n_kv_heads;
    Lanes l = lanes_at(a, 0, lane);
    long long total = l.all;
    for (int s0 = 64; s0 < a.b.n_seq; s0 += 64) total += lanes_at(a, s0, lane).all;
    // units of all sequences (the outer order) and heads (the inner) in a row, `share` of them to a workgroup
    const long long all = total * heads, share = (all + a.workgroups - 1) / a.workgroups, p = blockIdx.x * share;
    if (p >= all) return;
    long long todo = min(share, all - p), before = 0;
    int s0 = 0;
    while (p >= (before + l.all) * heads) {   // there is such a sequence: p < all
        before += l.all;
        s0 += 64;
        l = lanes_at(a, s0, lane);
    }
    int i = __popcll(__ballot((before + l.upto) * heads <= p));   // a prefix of the lanes
    int units = __builtin_amdgcn_readlane(l.units, i);
    const long long in = p - (before + __builtin_amdgcn_readlane(l.upto, i) - units) * heads;
    int h = (int)(in / units), off = (int)(in - (long long)h * units);
    while (todo > 0) {
        const SeqRaw raw = {__builtin_amdgcn_readlane(l.raw.q0, i), __builtin_amdgcn_readlane(l.raw.q1, i), __builtin_amdgcn_readlane(l.raw.kv, i)};
        const SeqRows sr = seq_rows(a.b, raw);
        const Range t = range_of(sr, 0, sr.n - 1, a.window);
        const int take = (int)min((long long)(units - off), todo);
        const bool begun = off > 0, ends = off + take == units;
        const int begin = t.from + off * kAttnUnit, end = min(t.to, begin + take * kAttnUnit);
        attn_item<F16, D, G, RT, NW, false>(a, s0 + i, h, sr, 0, sr.n * a.per_kv, begin, end, !begun && ends ? -1ll : 2ll * blockIdx.x + (begun ? 0 : 1));
        todo -= take;
        off = 0;
        if (todo > 0 && ++h == heads) {
            h = 0;
            do {   // the next sequence with rows: there is one, units are left
                if (++i == 64) {
                    i = 0;
                    s0 += 64;
                    l = lanes_at(a, s0, lane);
                }
                units = __builtin_amdgcn_readlane(l.units, i);
            } while (units == 0);
        }
    }
}

// A kernel over `workgroups` of them, in as many launches as they take.
inline hipError_t each_launch(void (*kernel)(KvAttnArgs), KvAttnArgs a, long long workgroups, int threads, hipStream_t s)
{
    const long long most = most_workgroups(threads);
    for (long long first = 0; first < workgroups; first += most) {
        a.first = (int)first;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(workgroups - first < most ? workgroups - first : most)), dim3(threads), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// One head size's kernels (mf_kv4_attn_d*.hip).
template <bool F16, int D, int G>
hipError_t pick_attn(const KvAttnArgs &a, const KvPlan &p, hipStream_t s)
{
    const auto go = [&](void (*kernel)(KvAttnArgs), int waves) { return each_launch(kernel, a, p.workgroups, waves * 64, s); };
    if (p.rows_by_wave) return go(attn_rows_kernel<F16, D, G, D < 256 ? 2 : 1>, kAttnWaves);
    if (D < 256 && p.rt == 2) {
        constexpr int RT = D < 256 ? 2 : 1;
        if (!p.whole) return go(attn_tokens_kernel<F16, D, G, RT, 4, false>, 4);
        return p.waves == 8 ? go(attn_tokens_kernel<F16, D, G, RT, 8, true>, 8) : go(attn_tokens_kernel<F16, D, G, RT, 4, true>, 4);
    }
    if (!p.whole) return go(attn_tokens_kernel<F16, D, G, 1, 4, false>, 4);
    return p.waves == 8 ? go(attn_tokens_kernel<F16, D, G, 1, 8, true>, 8) : go(attn_tokens_kernel<F16, D, G, 1, 4, true>, 4);
}

}  // namespace mfs
