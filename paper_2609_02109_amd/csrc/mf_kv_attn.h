// What attention over the caches shares (mf_kv4_attn.h, mf_kv8_attn.h): what a
// row sees, the shares of the work that workgroups take, and the end of a share.
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

constexpr float kNoBase = -1e38f;   // before the first token: below all scores; finite, so that differences of bases are
// From this base on a score's place in fp32 is 2^-3 and more.  What a step adds to the base and to a score in another
// order no longer meets: weights go by scores that are rounded as the base was, from the largest down, which
// then is the base itself.
constexpr float kFarBase = 0x1p20f;
__device__ __forceinline__ bool is_far(float base) { return fabsf(base) >= kFarBase; }

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

// The end of an item: rows row0 .. last, of which a wave holds RT tiles of 16 (lane l: row l % 16, dims 16 d + 4 (l / 16) ..
// + 3 of the weighted sum o, the sum of weights l, both over 2^base).  Adds up what the NW waves of a workgroup have of the
// same rows (0: each has rows of its own), and puts it into the output (slot < 0) or into a slot of the parts.
template <bool F16, int D, int RT, int NW>
__device__ __forceinline__ void end_item(const KvAttnArgs &a, int row0, int last, const int (&qrow)[RT], const int (&qhead)[RT], float (&base)[RT],
                                         float (&l)[RT], f32x4 (&o)[RT][D / 16], long long slot)
{
    constexpr int DT = D / 16;
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    if constexpr (NW > 0) {
        // the upper half of the waves hands over to the lower, and so on
        __shared__ f32x4 so[NW / 2][RT * DT][64];
        __shared__ f32x2 sm[NW / 2][RT][64];
#pragma unroll
        for (int half = NW / 2; half >= 1; half >>= 1) {
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int t = 0; t < RT; t++) {
                    sm[wave - half][t][lane] = (f32x2){base[t], l[t]};
#pragma unroll
                    for (int d = 0; d < DT; d++) so[wave - half][t * DT + d][lane] = o[t][d];
                }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int t = 0; t < RT; t++) {
                    const f32x2 other = sm[wave][t][lane];
                    const float to = fmaxf(base[t], other[0]);
                    const float x = __builtin_amdgcn_exp2f(base[t] - to), y = __builtin_amdgcn_exp2f(other[0] - to);
                    base[t] = to;
                    l[t] = l[t] * x + other[1] * y;
#pragma unroll
                    for (int d = 0; d < DT; d++) {
                        const f32x4 v = so[wave][t * DT + d][lane];
#pragma unroll
                        for (int r = 0; r < 4; r++) o[t][d][r] = o[t][d][r] * x + v[r] * y;
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
            const bool none = l[t] == 0.f;   // no token; a NaN stays one
            const float inv = none ? 0.f : 1.f / l[t];
            uint16_t *y = (uint16_t *)a.out + (long long)qrow[t] * a.out_stride + (long long)qhead[t] * a.out_head + qt * 4;
#pragma unroll
            for (int d = 0; d < DT; d++) {
                const f32x4 v = o[t][d] * inv;
                const u32x2 out = {pack2<F16>(v[0], v[1]), pack2<F16>(v[2], v[3])};
                __builtin_memcpy(__builtin_assume_aligned(y + 16 * d, 2), &out, 8);
            }
            if (a.lse && qt == 0)
                a.lse[(long long)qrow[t] * a.n_heads + qhead[t]] =
                    none ? -INFINITY : (base[t] + __builtin_amdgcn_logf(l[t])) * 0.69314718055994531f;
        } else {
            const long long at = slot * a.slot_rows + (NW == 0 ? r % a.slot_rows : r);
            float *y = a.part + at * D + qt * 4;
#pragma unroll
            for (int d = 0; d < DT; d++) *(f32x4 *)(y + 16 * d) = o[t][d];
            if (qt == 0) ((f32x2 *)(a.part + (long long)a.slots * a.slot_rows * D))[at] = (f32x2){base[t], l[t]};
        }
    }
}

// By rows: a workgroup takes a tile of attn_rows rows, its waves 16 RT of them each, over a part of their tokens.
template <int RT, class F>
__device__ __forceinline__ void rows_work(const KvAttnArgs &a, const F &item_of)
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
    item_of(s, h, sr, row0, row_end, begin, end, a.splits == 1 ? -1 : (long long)item * a.splits + split);
}

// By tokens (few rows): the waves of a workgroup take every fourth step each.  Whole: a workgroup per sequence and
// head.  Otherwise a.workgroups of them, as many as the card holds, take equal
// shares of all sequences' tokens: a share may end inside a head, whose parts
// the join adds up; slot 2 w is for a head that workgroup w found begun, 2 w + 1
// for one that it leaves unfinished.
template <bool WHOLE, class W, class S>
__device__ __forceinline__ void tokens_work(const KvAttnArgs &a, const W &whole, const S &shared)
{
    if constexpr (WHOLE) {
        const int wg = a.first + (int)blockIdx.x, h = wg % a.g.n_kv_heads, s = wg / a.g.n_kv_heads;
        const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
        if (sr.n == 0) return;
        const Range t = range_of(sr, 0, sr.n - 1, a.window);
        whole(s, h, sr, 0, sr.n * a.per_kv, t.from, t.to, -1);
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
        shared(s0 + i, h, sr, 0, sr.n * a.per_kv, begin, end, !begun && ends ? -1ll : 2ll * blockIdx.x + (begun ? 0 : 1));
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

}  // namespace mfs
