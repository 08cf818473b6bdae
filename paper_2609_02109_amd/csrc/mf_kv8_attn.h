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
// The largest is looked for only where the weights show that it is needed: when four
// together reach 2^14 the base goes to the largest so far less 10 (both as powers of two), and the step's
// weights are computed again.  Rows whose base is 2^20 or more, of either sign, take the largest so far as the
// base at every step and have weights up to 1, of scores that are rounded before the base is taken off: the sum in
// one step, s + (log2 scale - base), is off by some of fp32's places at the base, which from 2^26 on
// is more than binary16 has above the base.
// Values' operands are whole numbers: 1024 + u, a number of binary16's with the bits 0x6400 | u, less 1152.
#pragma once

#include <type_traits>

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

// Blocks of a step: which there are, and what their scales come to.
struct Step8 {
    int ok;
    float ks[2], lv[2], iv[2];   // the keys' scale; log2 of the values' scale, and 1 / it
};

__device__ __forceinline__ bool sees8(const Sight &v, int ok, int t0, int qt, int e)
{
    const int tok = t0 + 16 * (e >> 2) + 4 * qt + (e & 3);
    return (ok >> (e >> 2) & 1) && tok >= v.lo && tok <= v.hi;
}

// What a wave keeps for its rows (lane l's is row l % 16 of each tile): queries q, what they see, c (softmax scale times log2 e,
// and the row's power of two), first (what its scores begin at), base, l, and o (dims 16 d + 4 (l / 16) ..). As arrays
// by themselves: in a struct they take 30 registers more.
//
// key_at(u, n), value_at(n): operands (dims 64 (n / 2) + 16 (l / 16) + 8 (n % 2) .. of block u's keys, dims 16 n + l % 16 of the
// values).
template <int D, int RT, class AK>
__device__ __forceinline__ void attn8_scores(const u32x4 (&q)[RT][D / 32], const float (&first)[RT], f32x4 (&sc)[RT][2], const AK &key_at)
{
#pragma unroll
    for (int u = 0; u < 2; u++) {
#pragma unroll
        for (int t = 0; t < RT; t++) sc[t][u] = (f32x4){first[t], first[t], first[t], first[t]};
#pragma unroll
        for (int n = 0; n < D / 32; n++) {
            const u32x4 A = key_at(u, n);
#pragma unroll
            for (int t = 0; t < RT; t++) sc[t][u] = mfma<true>(A, q[t][n], sc[t][u]);
        }
    }
}

// x anew: what is computed from it is computed here, not before a loop or a branch and kept in registers.
__device__ __forceinline__ int again(int x)
{
    asm volatile("" : "+s"(x));
    return x;
}

// What S times 32 tokens from t0 on add to the rows, by their scores.  full: every row sees every token.
// far: some row of the wave has a base of 2^20 or more.
template <int D, int RT, int S, class AV>
__device__ __forceinline__ void attn8_step(const f32x4 (&sc)[S][RT][2], const Sight (&see)[RT], const float (&c)[RT], float (&base)[RT], float (&l)[RT],
                                           f32x4 (&o)[RT][D / 16], bool full, const Step8 (&now)[S], int t0, bool &far, const AV &value_at)
{
    const int qt = (threadIdx.x & 63) >> 4;
    u32x4 w[S][RT];
    float sum[S][RT][2];   // of a block's weights
    float highest[RT];
    constexpr float most = 16384.f;
    const auto weigh = [&](auto any_base) {
        float over = 0.f;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            highest[t] = 0.f;
#pragma unroll
            for (int k = 0; k < S; k++) {
                float e[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    float x = fmaf(sc[k][t][i >> 2][i & 3], now[k].ks[i >> 2] * c[t], now[k].lv[i >> 2] - base[t]);
                    if (decltype(any_base)::value && is_far(base[t])) x = fmaf(sc[k][t][i >> 2][i & 3], now[k].ks[i >> 2] * c[t], now[k].lv[i >> 2]) - base[t];
                    e[i] = __builtin_amdgcn_exp2f(x);
                }
                if (!full) {
                    const int at = again(t0 + 32 * k);   // else the comparisons are made for every step
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        if (!sees8(see[t], now[k].ok, at, qt, i)) e[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 4; i++) w[k][t][i] = pack2<true>(e[2 * i], e[2 * i + 1]);
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    sum[k][t][u] = (e[4 * u] + e[4 * u + 1]) + (e[4 * u + 2] + e[4 * u + 3]);   // before they are rounded
                    highest[t] = fmaxf(highest[t], sum[k][t][u]);
                }
            }
            over = fmaxf(over, highest[t]);
        }
        return __any(over >= most);
    };
    if (weigh(std::false_type()) || far) {
        bool any = false;
#pragma unroll
        for (int t = 0; t < RT; t++) {
            // only the rows that need it, so that no row's result depends on another's
            const bool over = quarters_max(highest[t]) >= most, hit = over || is_far(base[t]);
            float mx = kNoBase;
#pragma unroll
            for (int k = 0; k < S; k++)
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float s = fmaf(sc[k][t][i >> 2][i & 3], now[k].ks[i >> 2] * c[t], now[k].lv[i >> 2]);
                    if (full || sees8(see[t], now[k].ok, t0 + 32 * k, qt, i)) mx = fmaxf(mx, s);
                }
            mx = quarters_max(mx);
            if (!is_far(mx)) mx -= 10.f;
            const float to = hit ? fmaxf(mx, base[t]) : base[t], a = __builtin_amdgcn_exp2f(base[t] - to);
            base[t] = to;
            any |= is_far(to) && to != kNoBase;
            l[t] *= a;
#pragma unroll
            for (int d = 0; d < D / 16; d++) o[t][d] *= a;
        }
        far = __any(any);
        if (far) weigh(std::true_type());
        else weigh(std::false_type());
    }
#pragma unroll
    for (int k = 0; k < S; k++)
#pragma unroll
        for (int t = 0; t < RT; t++)
#pragma unroll
            for (int u = 0; u < 2; u++) l[t] = fmaf(sum[k][t][u], now[k].iv[u], l[t]);
#pragma unroll
    for (int k = 0; k < S; k++)
#pragma unroll
        for (int n = 0; n < D / 16; n++) {
            const u32x4 A = value_at(k, n);
#pragma unroll
            for (int t = 0; t < RT; t++) o[t][n] = mfma<true>(A, w[k][t], o[t][n]);
        }
}

// The rows of a wave's tiles in the step's tensors; rows past the last are computed as the last and not stored.
template <int RT>
__device__ __forceinline__ void rows_of(const KvAttnArgs &a, int h, const SeqRows &sr, int row0, int last, int (&qrow)[RT], int (&qhead)[RT])
{
#pragma unroll
    for (int t = 0; t < RT; t++) {
        const int r = min(row0 + 16 * t + (int)(threadIdx.x & 15), last), i = r / a.per_kv;
        qrow[t] = sr.q0 + i;
        qhead[t] = h * a.per_kv + (r - i * a.per_kv);
    }
}
// The rows' queries and what they see, on their way while the first step's tokens are.
template <bool F16, int D, int RT>
__device__ __forceinline__ void load_queries(const KvAttnArgs &a, int h, const SeqRows &sr, int row0, int last, u32x4 (&q)[RT][D / 32], Sight (&see)[RT])
{
    int qrow[RT], qhead[RT];
    rows_of<RT>(a, h, sr, row0, last, qrow, qhead);
#pragma unroll
    for (int t = 0; t < RT; t++) {
        see[t] = sight_of(sr.first_p + (qrow[t] - sr.q0), a.window, sr.limit);
        const uint16_t *x = (const uint16_t *)a.q + (long long)qrow[t] * a.q_stride + (long long)qhead[t] * a.q_head + ((threadIdx.x & 63) >> 4) * 16;
#pragma unroll
        for (int d = 0; d < D / 32; d++) q[t][d] = load16(x + 64 * (d >> 1) + 8 * (d & 1));
    }
}
// Queries to operands, nothing seen yet.
template <bool F16, int D, int RT>
__device__ __forceinline__ void make_ready(const KvAttnArgs &a, u32x4 (&q)[RT][D / 32], float (&c)[RT], float (&first)[RT], float (&base)[RT],
                                           float (&l)[RT], f32x4 (&o)[RT][D / 16])
{
    constexpr int NS = D / 32, DT = D / 16;
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
}

// The records of some steps of a sequence's and head's tokens, and what their scales come to: lane 2 i + u has block u of step
// i of 32, STRIDE tokens apart.  One gather for 32 steps: a page number that is fetched for the step at hand costs it
// a trip to memory.
struct Records8 {
    long long start;           // where there is no record that of the first one, which is read, and masked
    unsigned long long there;   // bit l: there is one
    float ks, lv, iv;
    __device__ __forceinline__ void find(const KvAttnArgs &a, const int *table, int h, int t0, int stride, int end, int limit)
    {
        const int lane = threadIdx.x & 63, at = t0 + (lane >> 1) * stride, blk = (at >> 4) + (lane & 1);
        start = 0;
        bool is = false;
        KvScales sc = {1.f, 1.f};
        if (at < end && blk * kKvBlock < limit) {
            const int pc = page_of_block(a.g, blk), page = table[pc];
            is = (unsigned)page < (unsigned)a.g.n_pages;
            if (is) {
                const long long record = ((long long)page * a.g.n_kv_heads + h) * a.g.blocks_per_page + (blk - pc * a.g.blocks_per_page);
                start = record * a.g.rec;
                sc = kv8_scales(a.g)[record];
            }
        }
        there = __ballot(is);
        ks = sc.k;
        if (sc.v < kKv8LeastScale) sc.v = kKv8LeastScale;   // memory of zeros
        lv = __builtin_amdgcn_logf(sc.v);   // of base 2
        iv = sc.v == sc.v ? 1.f / sc.v : 1.f;   // a number, so that it adds nothing to rows that do not see the block; the others have lv
    }
    static __device__ __forceinline__ float lane_of(float x, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); }
    __device__ __forceinline__ long long start_of(int l) const
    {
        return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(start >> 32), l) << 32 |
                           (unsigned)__builtin_amdgcn_readlane((int)start, l));
    }
    __device__ __forceinline__ const uint8_t *record(const KvAttnArgs &a, int l) const { return a.g.pages + start_of(l); }
    __device__ __forceinline__ Step8 step(int i) const
    {
        Step8 r;
        r.ok = (int)(there >> (2 * i)) & 3;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const int l = 2 * i + u;
            r.ks[u] = lane_of(ks, l);
            r.lv[u] = lane_of(lv, l);
            r.iv[u] = lane_of(iv, l);
        }
        return r;
    }
};

// Rows row0 .. of one sequence and key head over its tokens [begin, end):
// into the output (slot < 0) or a slot of the parts.
// NW waves share the rows and take different tokens, which each makes operands of in registers.  Bound by the bytes where
// tokens are many (24 requests over 9100 tokens at the mean, 48 heads over 8 of 128: 85 us for 449 MB, 5.3 TB/s, vector
// instructions 22 % beside it, and 7 us for the join), by one trip to memory after another where they are few (one request
// over 1500: 11 us, six steps a wave after a trip for the lengths and two for the page numbers and scales, and the sum of
// eight waves).
template <bool F16, int D, int RT, int NW>
__device__ __forceinline__ void attn8_item(const KvAttnArgs &a, int s, int h, const SeqRows &sr, int row0, int row_end, int begin, int end,
                                           long long slot)
{
    constexpr int NC = D / 64;
    const int lane = threadIdx.x & 63, wave = wave_id();
    const int last = min(row_end, row0 + RT * 16) - 1, limit = sr.limit;

    u32x4 q[RT][D / 32];
    Sight see[RT];
    float c[RT], first[RT], base[RT], l[RT];
    f32x4 o[RT][D / 16];
    bool far = false;
    load_queries<F16, D, RT>(a, h, sr, row0, last, q, see);
    const Sight see0 = sight_of(sr.first_p + row0 / a.per_kv, a.window, limit), see1 = sight_of(sr.first_p + last / a.per_kv, a.window, limit);

    const int *table = a.b.table + (long long)s * a.b.table_stride;
    constexpr int STRIDE = kAttnStep * NW;
    Records8 records;
    Attn8Tokens<D> x;
    const auto keys = [&](int i) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const uint8_t *rec = records.record(a, 2 * i + u);
#pragma unroll
            for (int j = 0; j < NC; j++) x.kc[u][j] = ((const u32x4 *)rec)[64 * j + lane];
        }
    };
    const auto values = [&](int i) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            const uint8_t *rec = records.record(a, 2 * i + u) + 16 * D;
#pragma unroll
            for (int j = 0; j < NC; j++) x.vc[u][j] = ((const u32x4 *)rec)[64 * j + lane];
        }
    };
    // the first step's records are on their way while the queries are made ready
    int t0 = begin + wave * kAttnStep, i = 0;
    Step8 now[1] = {{0, {1.f, 1.f}, {0.f, 0.f}, {1.f, 1.f}}};
    if (t0 < end) {
        records.find(a, table, h, t0, STRIDE, end, limit);
        now[0] = records.step(0);
        keys(0);
        values(0);
    }

    make_ready<F16, D, RT>(a, q, c, first, base, l, o);

    while (t0 < end) {
        const bool full = now[0].ok == 3 && t0 >= see1.lo && t0 + kAttnStep - 1 <= see0.hi;
        if (++i == 32) {
            records.find(a, table, h, t0 + STRIDE, STRIDE, end, limit);
            i = 0;
        }
        const Step8 next = records.step(i);   // past the end: records that are none
        const auto value_at = [&](int, int n) { return value_operand(x.vc[0][n >> 2][n & 3], x.vc[1][n >> 2][n & 3]); };
        f32x4 sc[1][RT][2];
        attn8_scores<D, RT>(q, first, sc[0], [&](int u, int n) { return key_operand(x.kc[u][n >> 1][2 * (n & 1)], x.kc[u][n >> 1][2 * (n & 1) + 1]); });
        // the next step's keys and values are fetched where this one has no more use for its own
        keys(i);
        attn8_step<D, RT, 1>(sc, see, c, base, l, o, full, now, t0, far, value_at);
        values(i);
        now[0] = next;
        t0 += STRIDE;
    }

    // the lanes' own sums together
#pragma unroll
    for (int t = 0; t < RT; t++) l[t] = quarters_sum(l[t]);
    int qrow[RT], qhead[RT];
    const int r0 = again(row0);
    rows_of<RT>(a, h, sr, r0, last, qrow, qhead);
    end_item<F16, D, RT, NW>(a, r0, last, qrow, qhead, base, l, o, slot);
}

// By rows (many query tokens): a workgroup takes a tile of attn_rows rows, its waves 16 RT of them each, over a part of
// their tokens.  The waves go over the same tokens: each makes a quarter of a step's operands and leaves
// them in LDS for all, for the step after the one that is computed.  Bound by issue: of the SIMDs' cycles vector
// instructions take 46 % (a weight's factor, power of two, sum, rounding and check) and matrix instructions 32 %, with two
// waves a SIMD by registers to put one over the other (2 x 1000 to 1024 query tokens over 8000 to 12000, 32 heads over 8 of
// 128: 430 us, 814 TFLOP/s).
template <bool F16, int D, int RT>
__global__ __launch_bounds__(kAttnWaves * 64, 2) void attn8_rows_kernel(KvAttnArgs a)
{
    static_assert(kAttnWaves == 4, "quarters");
    constexpr int WG_ROWS = attn_rows(RT, true), NC = D / 64, KEYS = 4 * NC, ALL = 8 * NC;   // operands of 32 tokens
    // 64 tokens a step for heads of 64 (2 x 1024 query tokens, 16 heads over 12000: 194 us, 32 a step 200, 128 a step 248) and two tiles
    // a wave (32 over 8 heads of 128 over 11000: 395 and 403), 32 else (one tile: 1 x 1000 over 1000: 33.1, 64 a step 34.7)
    constexpr int S = D == 64 || RT == 2 ? 2 : 1;
    __shared__ u32x4 lds[2][S][ALL][64];
    const int wg = a.first + (int)blockIdx.x, split = wg % a.splits, item = wg / a.splits;
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
    const int row_end = (int)min((long long)sr.n * a.per_kv, (long long)(tile + 1) * WG_ROWS), wg0 = tile * WG_ROWS;
    if (wg0 >= row_end) return;
    const int lane = threadIdx.x & 63, wave = wave_id(), limit = sr.limit;
    // a wave without rows makes operands and computes the tile's last row, which it does not store
    const int row0 = min(wg0 + wave * RT * 16, row_end - 1), last = min(row_end, row0 + RT * 16) - 1;
    const bool own = wg0 + wave * RT * 16 < row_end;
    u32x4 q[RT][D / 32];
    Sight see[RT];
    float c[RT], first[RT], base[RT], l[RT];
    f32x4 o[RT][D / 16];
    bool far = false;
    load_queries<F16, D, RT>(a, h, sr, row0, last, q, see);
    const Sight see0 = sight_of(sr.first_p + row0 / a.per_kv, a.window, limit), see1 = sight_of(sr.first_p + last / a.per_kv, a.window, limit);
    const Range t = range_of(sr, wg0 / a.per_kv, (row_end - 1) / a.per_kv, a.window);
    const long long part = t.from + (long long)split * a.chunk;
    const int begin = (int)min(part, (long long)t.to), end = split + 1 == a.splits ? t.to : (int)min(part + a.chunk, (long long)t.to);

    const int *table = a.b.table + (long long)s * a.b.table_stride;
    Records8 records;
    // this wave's quarter of 32 tokens: keys of block wave / 2, 2 NC dwords a lane; NC dwords of both blocks' values
    uint32_t kc[S][2 * NC], vc[S][2][NC];
    const auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < S; k++) {
            const uint8_t *key = records.record(a, 2 * (i + k) + (wave >> 1)) + lane * 16;
#pragma unroll
            for (int n = 0; n < NC; n++)
                __builtin_memcpy(kc[k] + 2 * n, __builtin_assume_aligned(key + (((wave & 1) * NC + n) >> 1) * 1024 + (((wave & 1) * NC + n) & 1) * 8, 8), 8);
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const uint8_t *value = records.record(a, 2 * (i + k) + u) + 16 * D + lane * 16;
                __builtin_memcpy(vc[k][u], __builtin_assume_aligned(value + (wave * NC >> 2) * 1024 + (wave * NC & 3) * 4, 4 * NC), 4 * NC);
            }
        }
    };
    const auto put = [&](int buf) {
#pragma unroll
        for (int k = 0; k < S; k++) {
#pragma unroll
            for (int n = 0; n < NC; n++) lds[buf][k][wave * NC + n][lane] = key_operand(kc[k][2 * n], kc[k][2 * n + 1]);
#pragma unroll
            for (int n = 0; n < NC; n++) lds[buf][k][KEYS + wave * NC + n][lane] = value_operand(vc[k][0][n], vc[k][1][n]);
        }
    };
    constexpr int STEP = S * kAttnStep;
    int i = 0;   // of the tokens fetched last, in the gather
    Step8 now[S], next[S];
#pragma unroll
    for (int k = 0; k < S; k++) now[k] = next[k] = {0, {1.f, 1.f}, {0.f, 0.f}, {1.f, 1.f}};
    if (begin < end) {
        records.find(a, table, h, begin, kAttnStep, end, limit);
#pragma unroll
        for (int k = 0; k < S; k++) {
            now[k] = records.step(k);
            next[k] = records.step(S + k);
        }
        fetch(0);
    }
    make_ready<F16, D, RT>(a, q, c, first, base, l, o);
    if (begin < end) {
        put(0);
        fetch(i = S);
        lds_barrier();
    }
    int buf = 0;
    for (int t0 = begin; t0 < end; t0 += STEP) {
        put(buf ^ 1);   // past the end: of records that are none, not used
        if ((i += S) == 32) {
            records.find(a, table, h, t0 + 2 * STEP, kAttnStep, end, limit);
            i = 0;
        }
        Step8 then[S];
#pragma unroll
        for (int k = 0; k < S; k++) then[k] = records.step(i + k);
        fetch(i);
        if (t0 <= see1.hi && t0 + STEP > see0.lo) {
            f32x4 sc[S][RT][2];
            int ok = 3;
#pragma unroll
            for (int k = 0; k < S; k++) {
                attn8_scores<D, RT>(q, first, sc[k], [&](int u, int n) { return lds[buf][k][u * 2 * NC + n][lane]; });
                ok &= now[k].ok;
            }
            attn8_step<D, RT, S>(sc, see, c, base, l, o, ok == 3 && t0 >= see1.lo && t0 + STEP - 1 <= see0.hi, now, t0, far,
                                 [&](int k, int n) { return lds[buf][k][KEYS + n][lane]; });
        }
#pragma unroll
        for (int k = 0; k < S; k++) {
            now[k] = next[k];
            next[k] = then[k];
        }
        buf ^= 1;
        lds_barrier();
    }
#pragma unroll
    for (int r = 0; r < RT; r++) l[r] = quarters_sum(l[r]);
    int qrow[RT], qhead[RT];
    const int r0 = again(row0);
    rows_of<RT>(a, h, sr, r0, last, qrow, qhead);
    if (own) end_item<F16, D, RT, 0>(a, r0, last, qrow, qhead, base, l, o, a.splits == 1 ? -1 : (long long)item * a.splits + split);
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
    if (p.rows_by_wave) {
        if constexpr (D == 128)
            if (p.rt == 2) return go(attn8_rows_kernel<F16, D, 2>, kAttnWaves);
        return go(attn8_rows_kernel<F16, D, 1>, kAttnWaves);
    }
    if (p.rt == 2) {
        if (!p.whole) return go(attn8_tokens_kernel<F16, D, TWO, 4, false>, 4);
        return p.waves == 8 ? go(attn8_tokens_kernel<F16, D, TWO, 8, true>, 8) : go(attn8_tokens_kernel<F16, D, TWO, 4, true>, 4);
    }
    if (!p.whole) return go(attn8_tokens_kernel<F16, D, 1, 4, false>, 4);
    return p.waves == 8 ? go(attn8_tokens_kernel<F16, D, 1, 8, true>, 8) : go(attn8_tokens_kernel<F16, D, 1, 4, true>, 4);
}

}  // namespace mfs
