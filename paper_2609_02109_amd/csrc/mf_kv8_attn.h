// Attention over the paged 8-bit cache (the kernel; mf_kv8_attn.hip plans and
// launches it).  One pass over the tokens with a running base and sum.
//
// A wave holds RT tiles of 16 rows (row = query token x head of the group that
// shares a key head).  A code's byte u = code + 128 is a matrix operand as it is: a
// binary16 number whose bits are u is the subnormal u 2^-24, which the matrix
// instructions take exactly and at full rate; one permutation of bytes makes two.  The
// queries are binary16 operands too, taken 2^e times first so that a row's largest is
// in [2^14, 2^15): bfloat16's 8 bits, and binary16's 11, are all there down to 2^-28 of it.
// Per 16 tokens S^T = K Q^T, begun at -128 sum_d q 2^-24 where it would begin at 0,
// which takes the 128 out again.  S^T comes out with the tokens 4 (l / 16) + r of row
// l % 16 in lane l, which is how the next product O^T = V^T P^T takes its right
// operand: weights stay in their lane.
//
// The keys' scale of a block is a factor of its scores; the values' scale is one of its
// weights, and goes into the exponent: w = 2^(s + log2 scale - base) = p scale 2^-base, rounded to
// binary16 (11 bits; everything else is fp32).  So the base goes by what a
// token can add to the result, not by its weight alone: w below 2^14, and what is 2^-34 of a row's
// largest has bits left, whatever sizes the blocks' values are of.  The sum of p adds w / scale.
// The largest is looked for only where a weight shows that it is needed: when one
// reaches 2^14 the base goes to the largest so far (in powers of two) less 10, and the step's
// weights are computed again.
// Values' operands are whole numbers: 1024 + u, a number of binary16's with the bits 0x6400 | u, less 1152.
#pragma once

#include "mf_kv_attn.h"

namespace mfs {

// A step's 32 tokens as a lane holds them (mf_serve.h; u: the block of 16), and their blocks' scales.
template <int D>
struct Attn8Tokens {
    static constexpr int NC = D / 64;
    u32x4 kc[2][NC], vc[2][NC];
};

// Bytes 2 i, 2 i + 1 of a dword in two halves, below `top` (a byte four times).
template <int I>
__device__ __forceinline__ uint32_t halves(uint32_t w, uint32_t top)
{
    // selector bytes 0..3 are w's, 4..7 top's
    return __builtin_amdgcn_perm(top, w, I ? 0x04030402u : 0x04010400u);
}
__device__ __forceinline__ u32x4 key_operand(uint32_t a, uint32_t b)
{
    return (u32x4){halves<0>(a, 0), halves<1>(a, 0), halves<0>(b, 0), halves<1>(b, 0)};
}
__device__ __forceinline__ u32x4 value_operand(uint32_t a, uint32_t b)
{
    u32x4 o = {halves<0>(a, 0x64646464u), halves<1>(a, 0x64646464u), halves<0>(b, 0x64646464u), halves<1>(b, 0x64646464u)};
    const f16x2 less = {(_Float16)1152.f, (_Float16)1152.f};
#pragma unroll
    for (int i = 0; i < 4; i++) o[i] = bits<uint32_t>(bits<f16x2>(o[i]) - less);
    return o;
}

// Blocks of a step: where their records are, which there are, and what their scales come to.
struct Step8 {
    const uint8_t *rec[2];
    int ok;
    float ks[2], lv[2], iv[2];   // the keys' scale; log2 of the values' scale, and 1 / it
};

__device__ __forceinline__ bool sees8(const Sight &v, int ok, int t0, int qt, int e)
{
    const int tok = t0 + 16 * (e >> 2) + 4 * qt + (e & 3);
    return (ok >> (e >> 2) & 1) && tok >= v.lo && tok <= v.hi;
}

// keys_done, values_done: called where the step has no more use for its keys and its values, to
// fetch the next step's into their place.  full: every row sees every token.  c: softmax scale times log2 e, and the
// row's power of two; first: what its scores begin at.
template <int D, int RT, class FK, class FV>
__device__ __forceinline__ void attn8_step(f32x4 (&o)[RT][D / 16], float (&base)[RT], float (&l)[RT], const u32x4 (&q)[RT][D / 32],
                                           const float (&first)[RT], const Attn8Tokens<D> &x, const Sight (&see)[RT], bool full,
                                           const Step8 &now, int t0, const float (&c)[RT], const FK &keys_done, const FV &values_done)
{
    constexpr int NC = D / 64;
    const int qt = (threadIdx.x & 63) >> 4;
    f32x4 sc[RT][2];
#pragma unroll
    for (int u = 0; u < 2; u++) {
#pragma unroll
        for (int t = 0; t < RT; t++) sc[t][u] = (f32x4){first[t], first[t], first[t], first[t]};
#pragma unroll
        for (int j = 0; j < NC; j++)
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const u32x4 A = key_operand(x.kc[u][j][2 * i], x.kc[u][j][2 * i + 1]);
#pragma unroll
                for (int t = 0; t < RT; t++) sc[t][u] = mfma<true>(A, q[t][2 * j + i], sc[t][u]);
            }
    }
    keys_done();
    u32x4 w[RT];
    float e[RT][8];
    for (bool raised = false;; raised = true) {   // twice at most
        int highest[RT], over = 0;
        constexpr int most = (15 + 14) << 10;   // 2^14 in binary16
#pragma unroll
        for (int t = 0; t < RT; t++) {
#pragma unroll
            for (int i = 0; i < 8; i++) e[t][i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i >> 2][i & 3], now.ks[i >> 2] * c[t], now.lv[i >> 2] - base[t]));
            if (!full) {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (!sees8(see[t], now.ok, t0, qt, i)) e[t][i] = 0.f;
            }
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
            float mx = kNoBase;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float s = fmaf(sc[t][i >> 2][i & 3], now.ks[i >> 2] * c[t], now.lv[i >> 2]);
                if (full || sees8(see[t], now.ok, t0, qt, i)) mx = fmaxf(mx, s);
            }
            mx = quarters_max(mx) - 10.f;
            const float to = hit ? fmaxf(mx, base[t]) : base[t], a = __builtin_amdgcn_exp2f(base[t] - to);
            base[t] = to;
            l[t] *= a;
#pragma unroll
            for (int d = 0; d < D / 16; d++) o[t][d] *= a;
        }
    }
#pragma unroll
    for (int t = 0; t < RT; t++)
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const float sum = (e[t][4 * u] + e[t][4 * u + 1]) + (e[t][4 * u + 2] + e[t][4 * u + 3]), more = fmaf(sum, now.iv[u], l[t]);
            // scales of blocks that the row does not see may be anything, not a number too
            l[t] = full || sum != 0.f ? more : l[t];
        }
#pragma unroll
    for (int j = 0; j < NC; j++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const u32x4 A = value_operand(x.vc[0][j][i], x.vc[1][j][i]);
#pragma unroll
            for (int t = 0; t < RT; t++) o[t][4 * j + i] = mfma<true>(A, w[t], o[t][4 * j + i]);
        }
    values_done();
}

// Rows row0 .. of one sequence and key head over its tokens [begin, end):
// into the output (slot < 0) or a slot of the parts.
// NW: waves that share the rows and take different tokens; 0: the wave has rows of its own.
template <bool F16, int D, int RT, int NW>
__device__ __forceinline__ void attn8_item(const KvAttnArgs &a, int s, int h, const SeqRows &sr, int row0, int row_end, int begin, int end,
                                           long long slot)
{
    constexpr int NS = D / 32, NC = D / 64, DT = D / 16;
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
        const uint16_t *x = (const uint16_t *)a.q + (long long)qrow[t] * a.q_stride + (long long)qhead[t] * a.q_head + qt * 16;
#pragma unroll
        for (int d = 0; d < NS; d++) q[t][d] = load16(x + 64 * (d >> 1) + 8 * (d & 1));
    }
    const Sight see0 = sight_of(sr.first_p + row0 / a.per_kv, a.window, limit), see1 = sight_of(sr.first_p + last / a.per_kv, a.window, limit);

    const int *table = a.b.table + (long long)s * a.b.table_stride;
    const KvScales *scales = kv8_scales(a.g);
    constexpr int STRIDE = kAttnStep * (NW == 0 ? 1 : NW);
    // The records of the next 32 steps, and what their scales come to: lane 2 i + u has block u
    // of step i, -1 where there is none.  One gather for 32 steps: a page number
    // that is fetched for the step at hand costs it a trip to memory.
    long long starts;
    float ks, lv, iv;
    const auto find = [&](int t0) {
        const int at = t0 + (lane >> 1) * STRIDE, blk = (at >> 4) + (lane & 1);
        starts = -1;
        KvScales sc = {1.f, 1.f};
        if (at < end && blk * kKvBlock < limit) {
            const int pc = page_of_block(a.g, blk), page = table[pc];
            if ((unsigned)page < (unsigned)a.g.n_pages) {
                const long long record = ((long long)page * a.g.n_kv_heads + h) * a.g.blocks_per_page + (blk - pc * a.g.blocks_per_page);
                starts = record * a.g.rec;
                sc = scales[record];
            }
        }
        ks = sc.k;
        if (sc.v < kKv8LeastScale) sc.v = kKv8LeastScale;   // memory of zeros
        lv = __builtin_amdgcn_logf(sc.v);   // of base 2
        iv = 1.f / sc.v;
    };
    const auto lane_of = [](float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
    // where there is no record the first one is read, and masked
    const auto step_at = [&](int i) {
        Step8 r;
        r.ok = 0;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int l = 2 * i + u;
            const long long at = (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(starts >> 32), l) << 32 |
                                             (unsigned)__builtin_amdgcn_readlane((int)starts, l));
            r.ok |= (at >= 0) << u;
            r.rec[u] = a.g.pages + (at < 0 ? 0 : at);
            r.ks[u] = lane_of(ks, l);
            r.lv[u] = lane_of(lv, l);
            r.iv[u] = lane_of(iv, l);
        }
        return r;
    };
    Attn8Tokens<D> x;
    const auto keys_of = [&](const Step8 &r) {
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int j = 0; j < NC; j++) x.kc[u][j] = ((const u32x4 *)r.rec[u])[64 * j + lane];
    };
    const auto values_of = [&](const Step8 &r) {
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int j = 0; j < NC; j++) x.vc[u][j] = ((const u32x4 *)(r.rec[u] + 16 * D))[64 * j + lane];
    };
    // the first step's records are on their way while the queries are made ready
    int t0 = begin + (NW == 0 ? 0 : wave * kAttnStep), i = 0;
    Step8 now = {{a.g.pages, a.g.pages}, 0, {1.f, 1.f}, {0.f, 0.f}, {1.f, 1.f}};
    if (t0 < end) {
        find(t0);
        now = step_at(0);
        keys_of(now);
        values_of(now);
    }

    float c[RT], first[RT], base[RT], l[RT];
    f32x4 o[RT][DT];
#pragma unroll
    for (int t = 0; t < RT; t++) {
        float big = 0.f;
#pragma unroll
        for (int d = 0; d < NS; d++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                big = fmaxf(big, fmaxf(fabsf(to_float<F16>((uint16_t)q[t][d][j])), fabsf(to_float<F16>((uint16_t)(q[t][d][j] >> 16)))));
        const int L = max((int)(__float_as_uint(quarters_max(big)) >> 23), 1) - 127;
#pragma unroll
        for (int d = 0; d < NS; d++)
#pragma unroll
            for (int j = 0; j < 4; j++)
                q[t][d][j] = pack2<true>(__builtin_amdgcn_ldexpf(to_float<F16>((uint16_t)q[t][d][j]), 14 - L),
                                         __builtin_amdgcn_ldexpf(to_float<F16>((uint16_t)(q[t][d][j] >> 16)), 14 - L));
        // at most 2^110, so that its product with a scale stays a number
        c[t] = fminf(__builtin_amdgcn_ldexpf(a.scale_log2, L + 10), 0x1p110f);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        const u32x4 less = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};   // -128 2^-24 in each half
#pragma unroll
        for (int d = 0; d < NS; d++) sum = mfma<true>(less, q[t][d], sum);
        first[t] = sum[0];
        base[t] = kNoBase;
        l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < DT; d++) o[t][d] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }

    while (t0 < end) {
        const bool full = now.ok == 3 && t0 >= see1.lo && t0 + kAttnStep - 1 <= see0.hi;
        if (++i == 32) {
            find(t0 + STRIDE);
            i = 0;
        }
        const Step8 next = step_at(i);   // past the end: records that are none
        attn8_step<D, RT>(o, base, l, q, first, x, see, full, now, t0, c, [&] { keys_of(next); }, [&] { values_of(next); });
        now = next;
        t0 += STRIDE;
    }

    // the lanes' own sums together
#pragma unroll
    for (int t = 0; t < RT; t++) l[t] = quarters_sum(l[t]);
    end_item<F16, D, RT, NW>(a, row0, last, qrow, qhead, base, l, o, slot);
}

template <bool F16, int D, int RT>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn8_rows_kernel(KvAttnArgs a)
{
    rows_work<RT>(a, [&](auto... item) { attn8_item<F16, D, RT, 0>(a, item...); });
}

template <bool F16, int D, int RT, int NW, bool WHOLE>
__global__ __launch_bounds__(NW * 64, 2) void attn8_tokens_kernel(KvAttnArgs a)
{
    const auto item_of = [&](auto... item) { attn8_item<F16, D, RT, NW>(a, item...); };
    tokens_work<WHOLE>(a, item_of, item_of);
}

// One head size's kernels (mf_kv8_attn_d*.hip).
template <bool F16, int D>
hipError_t pick_attn8(const KvAttnArgs &a, const KvPlan &p, hipStream_t s)
{
    const auto go = [&](void (*kernel)(KvAttnArgs), int waves) { return each_launch(kernel, a, p.workgroups, waves * 64, s); };
    constexpr int TWO = D < 256 ? 2 : 1;
    if (p.rows_by_wave) return go(attn8_rows_kernel<F16, D, TWO>, kAttnWaves);
    if (p.rt == 2) {
        if (!p.whole) return go(attn8_tokens_kernel<F16, D, TWO, 4, false>, 4);
        return p.waves == 8 ? go(attn8_tokens_kernel<F16, D, TWO, 8, true>, 8) : go(attn8_tokens_kernel<F16, D, TWO, 4, true>, 4);
    }
    if (!p.whole) return go(attn8_tokens_kernel<F16, D, 1, 4, false>, 4);
    return p.waves == 8 ? go(attn8_tokens_kernel<F16, D, 1, 8, true>, 8) : go(attn8_tokens_kernel<F16, D, 1, 4, true>, 4);
}

}  // namespace mfs
