// Attention over the paged 4-bit cache (the kernel; mf_kv4_attn.hip plans and
// launches it).  One pass over the tokens with a running maximum and sum.
//
// A wave holds RT tiles of 16 rows (row = query token x head of the group that
// shares a key head).  Per 16 tokens it computes S^T = K Q^T with the key codes
// as they are, 16 + c, and per group of G dims
//   s = sum_g scale_g (sum_d (16 + c) q - 16 sum_d q) + off_g sum_d q:
// -16 sum q is the product's starting value, and the last sum over g is a matrix
// product itself (sum q in two binary16 pieces, 22 bits).  S^T comes out with the
// tokens 4 (l / 16) + r of row l % 16 in lane l, which is how the next product
// O^T = V^T P^T takes its right operand: softmax weights stay in their lane.
//   o = sum_t w (16 + c) - 16 sum_t w + sum_t p off_g,   w = p scale_g,
// p and w rounded to binary16 (11 bits; everything else is fp32), the second sum
// from the same instruction with ones for codes, so that the 16 cancels exactly.
// Weights are kept relative to 2^base, base = the largest s so far (in powers of
// two) less 14, more where a step has scales of 2 and above, so that p, w <
// 2^15: binary16 then holds weights down to 2^-38 of the largest, and the small
// weights of long contexts are not lost.
#pragma once

#include "mf_serve_dev.h"

namespace mfs {

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

template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const uint8_t *p)
{
    Words<N> r;
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; i++) {
            const u32x4 v = ((const u32x4 *)p)[i];
#pragma unroll
            for (int j = 0; j < 4; j++) r.w[4 * i + j] = v[j];
        }
    } else {
        static_assert(N == 2, "8 bytes");
        const u32x2 v = *(const u32x2 *)p;
        r.w[0] = v[0];
        r.w[1] = v[1];
    }
    return r;
}

// What a wave keeps for its rows: lane l's is row l % 16 of each tile.
template <int D, int G, int RT>
struct AttnState {
    static constexpr int DT = D / 16, NG = D / G;
    f32x4 o[RT][DT];      // sum w (16 + c): dims 16 t + 4 (l / 16) + r
    f32x4 ow[RT][NG];     // sum w, in every element
    f32x4 om[RT];         // sum p off: element r is group (4 (l / 16) + r) % NG
    float base[RT], l[RT];   // weights are relative to 2^base; sum of p over the lane's tokens
};

// A step's 32 tokens as a lane holds them (mf_serve.h; u: the block of 16).
template <int D, int G>
struct AttnTokens {
    static constexpr int NS = D / 32, NG = D / G;
    Words<NS> kc[2], vc[2];      // codes
    u32x2 ks[2][NG], vs[2][NG];  // scales of tokens 4 (l / 16) .. + 3
    u32x2 ko[2];                 // key offsets of token l % 16: a right operand's pairs of groups
    u32x2 vo[2];                 // value offsets of group l % NG, tokens 4 (l / 16) .. + 3
};

template <int D, int G>
__device__ __forceinline__ void load_tokens(AttnTokens<D, G> &x, int u, const uint8_t *rec, int lane)
{
    constexpr int NS = D / 32, NG = D / G;
    const int col = lane & 15, qt = lane >> 4;
    x.kc[u] = load_words<NS>(rec + lane * (D / 8));
    x.vc[u] = load_words<NS>(rec + 8 * D + lane * (D / 8));
    const uint8_t *t = rec + 16 * D;
#pragma unroll
    for (int g = 0; g < NG; g++) {
        x.ks[u][g] = *(const u32x2 *)(t + g * 32 + qt * 8);
        x.vs[u][g] = *(const u32x2 *)(t + 64 * NG + g * 32 + qt * 8);
    }
    const uint8_t *ko = t + 32 * NG + col * 2 * NG;
    if constexpr (NG == 1) x.ko[u] = (u32x2){*(const uint16_t *)ko, 0};
    if constexpr (NG == 2) x.ko[u] = (u32x2){*(const uint32_t *)ko, 0};
    if constexpr (NG == 4) x.ko[u] = *(const u32x2 *)ko;
    if constexpr (NG == 8) x.ko[u] = *(const u32x2 *)(ko + (qt & 1) * 8);
    x.vo[u] = *(const u32x2 *)(t + 96 * NG + (col & (NG - 1)) * 32 + qt * 8);
}

__device__ __forceinline__ float half_of(uint32_t w, int hi) { return (float)bits<f16x2>(w)[hi]; }

// limit: tokens from it on were never written; c: softmax scale times log2 e (and the row's power of two).
template <bool F16, int D, int G, int RT, bool MASK>
__device__ __forceinline__ void attn_step(AttnState<D, G, RT> &st, const u32x4 (&q)[RT][D / 32], const f32x4 (&start)[RT][D / G],
                                          const u32x2 (&qsum)[RT], const AttnTokens<D, G> &x, const Sight (&see)[RT],
                                          const bool (&ok)[2], int limit, int t0, const float (&c)[RT])
{
    constexpr int NG = D / G, IPG = G / 32;
    const int qt = (threadIdx.x & 63) >> 4;
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    float p[RT][2][4];
    uint32_t keep[RT][2][2];   // halves of the weights that the row sees
#pragma unroll
    for (int u = 0; u < 2; u++) {
        f32x4 sc[RT];
#pragma unroll
        for (int t = 0; t < RT; t++)
            sc[t] = __builtin_amdgcn_mfma_f32_16x16x16f16(bits<f16x4>(x.ko[u]), bits<f16x4>(qsum[t]), zero, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < NG; g++) {
            f32x4 P[RT];
#pragma unroll
            for (int i = 0; i < IPG; i++) {
                const u32x4 A = codes8<F16>(x.kc[u].w[g * IPG + i]);
#pragma unroll
                for (int t = 0; t < RT; t++) P[t] = mfma<F16>(A, q[t][g * IPG + i], i ? P[t] : start[t][g]);
            }
#pragma unroll
            for (int t = 0; t < RT; t++)
#pragma unroll
                for (int r = 0; r < 4; r++) sc[t][r] = fmaf(half_of(x.ks[u][g][r >> 1], r & 1), P[t][r], sc[t][r]);
        }
#pragma unroll
        for (int t = 0; t < RT; t++) {
            keep[t][u][0] = keep[t][u][1] = 0;
#pragma unroll
            for (int r = 0; r < 4; r++) {
                p[t][u][r] = sc[t][r];
                if (MASK) {
                    const int tok = t0 + 16 * u + 4 * qt + r;
                    if (ok[u] && tok >= see[t].lo && tok <= see[t].hi) keep[t][u][r >> 1] |= r & 1 ? 0xffff0000u : 0xffffu;
                    else p[t][u][r] = -INFINITY;
                }
            }
        }
    }
    // scales of 2 and above (bit 14) are rare, and cost a lower start of the weights
    uint32_t any = 0;
#pragma unroll
    for (int g = 0; g < NG; g++) any |= x.vs[0][g][0] | x.vs[0][g][1] | x.vs[1][g][0] | x.vs[1][g][1];
    float room = 14.f;
    if (__any(any & 0x40004000u)) {
        float v = 1.f;
#pragma unroll
        for (int g = 0; g < NG; g++)
#pragma unroll
            for (int e = 0; e < 8; e++) v = fmaxf(v, half_of(x.vs[e >> 2][g][(e >> 1) & 1], e & 1));
        v = fminf(quarters_max(v), 65504.f);
        room = 14.f - (float)((__float_as_uint(v) >> 23) - 127u);
    }
    u32x4 w[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        float mx = p[t][0][0];
#pragma unroll
        for (int e = 1; e < 8; e++) mx = fmaxf(mx, p[t][e >> 2][e & 3]);
        mx = fmaf(quarters_max(mx), c[t], -room);
        if (__any(mx > st.base[t])) {
            const float base = fmaxf(mx, st.base[t]), a = base == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.base[t] - base);
            st.base[t] = base;
            st.l[t] *= a;
            st.om[t] *= a;
#pragma unroll
            for (int g = 0; g < NG; g++) st.ow[t][g] *= a;
#pragma unroll
            for (int d = 0; d < D / 16; d++) st.o[t][d] *= a;
        }
        const float base = st.base[t] == -INFINITY ? 0.f : st.base[t];
#pragma unroll
        for (int u = 0; u < 2; u++) {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                p[t][u][r] = __builtin_amdgcn_exp2f(fmaf(p[t][u][r], c[t], -base));
                st.l[t] += p[t][u][r];
            }
            w[t][2 * u] = pack2<true>(p[t][u][0], p[t][u][1]);
            w[t][2 * u + 1] = pack2<true>(p[t][u][2], p[t][u][3]);
        }
    }
    u32x4 vo = {x.vo[0][0], x.vo[0][1], x.vo[1][0], x.vo[1][1]};
    if (MASK) {
        // what was never written may be anything; a zero weight does not make it zero
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int tok = t0 + 16 * (e >> 1) + 4 * qt + 2 * (e & 1);
            vo[e] &= (ok[e >> 1] && tok < limit ? 0xffffu : 0u) | (ok[e >> 1] && tok + 1 < limit ? 0xffff0000u : 0u);
        }
    }
#pragma unroll
    for (int t = 0; t < RT; t++) st.om[t] = mfma<true>(vo, w[t], st.om[t]);
#pragma unroll
    for (int g = 0; g < NG; g++) {
        u32x4 wg[RT];
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                wg[t][e] = bits<uint32_t>(bits<f16x2>(w[t][e]) * bits<f16x2>(x.vs[e >> 1][g][e & 1]));
                if (MASK) wg[t][e] &= keep[t][e >> 1][e & 1];
            }
#pragma unroll
        for (int i = g * IPG; i < (g + 1) * IPG; i++) {
            const uint32_t a = x.vc[0].w[i], b = x.vc[1].w[i];
            const u32x4 lo = {codes2<true, 0>(a), codes2<true, 1>(a), codes2<true, 0>(b), codes2<true, 1>(b)};
            const u32x4 hi = {codes2<true, 2>(a), codes2<true, 3>(a), codes2<true, 2>(b), codes2<true, 3>(b)};
#pragma unroll
            for (int t = 0; t < RT; t++) {
                st.o[t][2 * i] = mfma<true>(lo, wg[t], st.o[t][2 * i]);
                st.o[t][2 * i + 1] = mfma<true>(hi, wg[t], st.o[t][2 * i + 1]);
            }
        }
#pragma unroll
        for (int t = 0; t < RT; t++) st.ow[t][g] = mfma<true>(ones8<true>(), wg[t], st.ow[t][g]);
    }
}

// Work item: (sequence, key head, tile of attn_rows rows); splits workgroups take
// parts of its tokens.  ROWS: the waves take different rows, all tokens each;
// otherwise the same rows, every fourth step of tokens each, joined in LDS.
template <bool F16, int D, int G, int RT, bool ROWS>
__global__ __launch_bounds__(kAttnWaves * 64) void attn_kernel(KvAttnArgs a)
{
    constexpr int NS = D / 32, NG = D / G, IPG = G / 32, DT = D / 16, WG_ROWS = attn_rows(RT, ROWS);
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int split = (int)(blockIdx.x % a.splits), item = (int)(blockIdx.x / a.splits);
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const int q0 = a.b.q_start[s];
    const long long q1 = a.b.q_start[s + 1], kv = a.b.kv_len[s];
    const int limit = kv < 0 ? 0 : kv < a.b.max_kv ? (int)kv : a.b.max_kv;
    const long long first_p = kv - (q1 - q0);   // position of the sequence's first row
    const int n = q0 < 0 || q0 >= a.b.rows || q1 <= q0 ? 0 : (int)((q1 < a.b.rows ? q1 : a.b.rows) - q0);
    const int row_end = (int)min((long long)n * a.per_kv, (long long)(tile + 1) * WG_ROWS);
    const int row0 = tile * WG_ROWS + (ROWS ? wave * RT * 16 : 0);
    if (tile * WG_ROWS >= row_end) return;          // the whole workgroup
    if (ROWS && row0 >= row_end) return;            // waves that take rows of their own never meet again
    const int last = min(row_end, row0 + RT * 16) - 1;

    // rows past the last are computed as the last and not stored
    u32x4 q[RT][NS];
    Sight see[RT];
    int qrow[RT], qhead[RT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int r = min(row0 + 16 * t + col, last);
        const int i = r / a.per_kv;
        qrow[t] = q0 + i;
        qhead[t] = h * a.per_kv + (r - i * a.per_kv);
        see[t] = sight_of(first_p + i, a.window, limit);
        const uint16_t *x = (const uint16_t *)a.q + (long long)qrow[t] * a.q_stride + (long long)qhead[t] * a.q_head + qt * 8;
#pragma unroll
        for (int d = 0; d < NS; d++) q[t][d] = load16(x + 32 * d);
    }
    const Sight see0 = sight_of(first_p + row0 / a.per_kv, a.window, limit), see1 = sight_of(first_p + last / a.per_kv, a.window, limit);
    const int from = see0.lo & ~(kAttnStep - 1), to = see1.hi + 1;   // tokens that some row sees, and none after
    const long long part = from + (long long)split * a.chunk;
    const int begin = (int)min(part, (long long)to), end = split + 1 == a.splits ? to : (int)min(part + a.chunk, (long long)to);

    f32x4 start[RT][NG];   // -16 sum q of a group
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
            big = fmaxf(big, fabsf(qs[g]));
        }
        // queries whose sums binary16 may not hold are taken 2^-e times, and their products' scale 2^e
        float down = 1.f;
        c[t] = a.scale_log2;
        if (big >= 16384.f) {
            const int e = (int)(__float_as_uint(big) >> 23) - 127 - 13;
            down = __uint_as_float((uint32_t)(127 - e) << 23);
            c[t] *= __uint_as_float((uint32_t)(127 + e) << 23);
        }
        if (__any(down != 1.f)) {
#pragma unroll
            for (int d = 0; d < NS; d++)
#pragma unroll
                for (int j = 0; j < 4; j++)
                    q[t][d][j] = pack2<F16>(to_float<F16>((uint16_t)q[t][d][j]) * down, to_float<F16>((uint16_t)(q[t][d][j] >> 16)) * down);
        }
        f16x4 piece = {(_Float16)0.f, (_Float16)0.f, (_Float16)0.f, (_Float16)0.f};
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const float x = qs[g] * down;
            start[t][g] = (f32x4){-16.f * x, -16.f * x, -16.f * x, -16.f * x};
            const _Float16 hi = (_Float16)x, lo = (_Float16)(x - (float)hi);
            if (NG <= 4) {
                if (qt == 0) piece[g & 3] = hi;
                if (qt == 1) piece[g & 3] = lo;
            } else {
                if (qt == g / 4) piece[g & 3] = hi;
                if (qt == 2 + g / 4) piece[g & 3] = lo;
            }
            st.ow[t][g] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
        qsum[t] = bits<u32x2>(piece);
        st.om[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        st.base[t] = -INFINITY;
        st.l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; d++) st.o[t][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    const int *table = a.b.table + (long long)s * a.b.table_stride;
    for (int t0 = begin + (ROWS ? 0 : wave * kAttnStep); t0 < end; t0 += kAttnStep * (ROWS ? 1 : kAttnWaves)) {
        AttnTokens<D, G> x;
        bool ok[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int blk = (t0 >> 4) + u;
            int page = -1, in = 0;
            if (blk * kKvBlock < limit) {
                const int pc = page_of_block(a.g, blk);
                page = table[pc];
                in = blk - pc * a.g.blocks_per_page;
            }
            ok[u] = (unsigned)page < (unsigned)a.g.n_pages;
            // a page that is none of the cache's: the first record is read and masked
            const long long at = ok[u] ? ((long long)page * a.g.n_kv_heads + h) * a.g.blocks_per_page + in : 0;
            load_tokens(x, u, a.g.pages + at * a.g.rec, lane);
        }
        const bool full = ok[0] && ok[1] && t0 >= see1.lo && t0 + kAttnStep - 1 <= see0.hi;
        if (full) attn_step<F16, D, G, RT, false>(st, q, start, qsum, x, see, ok, limit, t0, c);
        else attn_step<F16, D, G, RT, true>(st, q, start, qsum, x, see, ok, limit, t0, c);
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
            const float add = om - 16.f * st.ow[t][g][0];
#pragma unroll
            for (int d = g * (G / 16); d < (g + 1) * (G / 16); d++) st.o[t][d] += add;
        }
    }
    if constexpr (!ROWS) {
        // waves 2 and 3 hand over to 0 and 1, then 1 to 0
        __shared__ f32x4 so[2][RT * DT][64];
        __shared__ f32x2 sm[2][RT][64];
#pragma unroll
        for (int half = 2; half >= 1; half >>= 1) {
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
                    const float x = base == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.base[t] - base);
                    const float y = base == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(other[0] - base);
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
        if (a.splits == 1) {
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
            const long long at = ((long long)item * a.splits + split) * WG_ROWS + (r - tile * WG_ROWS);
            float *y = a.part + at * D + qt * 4;
#pragma unroll
            for (int d = 0; d < DT; d++) *(f32x4 *)(y + 16 * d) = st.o[t][d];
            if (qt == 0) ((f32x2 *)(a.part + (long long)a.items * a.splits * WG_ROWS * D))[at] = (f32x2){st.base[t], st.l[t]};
        }
    }
}

template <bool F16, int D, int G, int RT, bool ROWS>
hipError_t go_attn(const KvAttnArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((attn_kernel<F16, D, G, RT, ROWS>), dim3((unsigned)((long long)a.items * a.splits)), dim3(kAttnWaves * 64), 0, s, a);
    return hipGetLastError();
}

// One head size's kernels (mf_kv4_attn_d*.hip).
template <bool F16, int D, int G>
hipError_t pick_attn(const KvAttnArgs &a, const KvPlan &p, hipStream_t s)
{
    if (p.rows_by_wave) return go_attn<F16, D, G, 2, true>(a, s);
    if constexpr (D < 256)
        if (p.rt == 2) return go_attn<F16, D, G, 2, false>(a, s);
    return go_attn<F16, D, G, 1, false>(a, s);
}

}  // namespace mfs
