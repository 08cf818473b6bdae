// What the caches' append and read share (mf_kv4.hip, mf_kv8.hip): a step's new
// tokens, the turn of keys and queries by their positions, launches over blocks.
#pragma once

#include "mf_serve_dev.h"

namespace mfs {

// A sequence's new tokens as far as they lie in the step's rows and in the
// cache, whatever the device arrays hold: positions [lo, hi), row = pos + shift.
struct Span {
    int lo, hi;
    long long shift;
    long long row0, row1;   // its rows in [0, rows)
};

__device__ __forceinline__ Span span_of(const KvBatch &b, int s)
{
    Span p;
    const long long r0 = b.q_start[s], r1 = b.q_start[s + 1], kv = b.kv_len[s];
    p.shift = r1 - kv;
    p.row0 = r0 > 0 ? r0 : 0;
    p.row1 = r1 < b.rows ? r1 : b.rows;
    const long long lo = p.row0 - p.shift, hi = p.row1 - p.shift;
    p.lo = lo <= 0 ? 0 : lo < b.max_kv ? (int)lo : b.max_kv;
    p.hi = hi <= 0 ? 0 : hi < b.max_kv ? (int)hi : b.max_kv;
    return p;
}

template <bool F16>
__device__ __forceinline__ void widen8(u32x4 raw, float *v)
{
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = to_float<F16>((uint16_t)(raw[j >> 1] >> (16 * (j & 1))));
}

// Eight values of a row turned by its position: dims d .. d + 7 of a head at x, of
// which `own` are loaded.  Each product and sum is rounded by itself (the library is
// compiled without contraction), as the definition has it.
template <bool F16>
__device__ __forceinline__ void turn8(const uint16_t *x, u32x4 own, int d, int rot, int inter, const float *cos, const float *sin, float *v)
{
    widen8<F16>(own, v);
    if (d >= rot) return;
    const int half = rot >> 1;
    if (inter) {
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const float c = cos[(d + j) >> 1], s = sin[(d + j) >> 1], a = v[j], b = v[j + 1];
            v[j] = a * c - b * s;
            v[j + 1] = b * c + a * s;
        }
        return;
    }
    // rot / 2 is a multiple of 8: the partners are eight in a row too
    const bool second = d >= half;
    const int t = second ? d - half : d;
    float y[8];
    widen8<F16>(load16(x + (second ? t : t + half)), y);
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float c = cos[t + j], s = sin[t + j];
        v[j] = second ? v[j] * c + y[j] * s : v[j] * c - y[j] * s;
    }
}
// The pair of halves (a, b) of dims t .. t + 7.
__device__ __forceinline__ void turn_pair(float *a, float *b, const float *cos, const float *sin)
{
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float c = cos[j], s = sin[j], x = a[j], y = b[j];
        a[j] = x * c - y * s;
        b[j] = y * c + x * s;
    }
}

// The queries of 16 tokens, heads h0 .. h1: a thread takes 8 dims (with their
// partners, so that the result may go over its source).  Many tokens: eight of them
// side by side, the angles kept over the heads; few: eight heads side by side, and as many tokens as there are threads left.
template <bool F16>
__device__ __forceinline__ void turn_queries(const KvAppendArgs &a, const Span &p, int blk, int h0, int h1, int D, bool few)
{
    const int half = a.rot >> 1, base = p.lo + blk * 16;
    const int units = a.interleaved ? D / 8 : (D - half) / 8;   // a unit below rot / 2 takes its partner along
    // threads side by side over a head: as many as have a unit (append of 13 x 300 rows of 20 + 2 x 4 heads of 64: eight of them 13.4 us, four 11.0)
    const int side = units <= 4 ? 4 : 8, groups = 64 / side;
    const int u0 = threadIdx.x & (side - 1), b0 = threadIdx.x / side;
    for (int u = u0; u < units; u += side) {
        const int d = u * 8, d0 = a.interleaved || d < half ? d : d + half, d1 = !a.interleaved && d < half ? d + half : -1;
        const bool turned = d0 < a.rot;
        for (int t = few ? b0 >> 3 : b0; t < 16; t += few ? groups >> 3 : groups) {
            const int pos = base + t;
            if (pos >= p.hi) break;
            const long long row = pos + p.shift;
            const uint16_t *x = (const uint16_t *)a.q + row * a.q_stride;
            uint16_t *y = (uint16_t *)a.q_out + row * a.qo_stride;
            float cos[8], sin[8];
            if (turned) {
                const long long at = (long long)pos * half + (a.interleaved ? d >> 1 : d);
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int e = a.interleaved ? j >> 1 : j;
                    cos[j] = a.cos[at + e];
                    sin[j] = a.sin[at + e];
                }
            }
            const auto load = [&](u32x4 (&raw)[2], int h) {
                raw[0] = load16(x + h * a.q_head + d0);
                if (d1 >= 0) raw[1] = load16(x + h * a.q_head + d1);
            };
            const auto turn = [&](const u32x4 (&raw)[2], int h) {
                float v[2][8];
                widen8<F16>(raw[0], v[0]);
                if (d1 >= 0) {
                    widen8<F16>(raw[1], v[1]);
                    turn_pair(v[0], v[1], cos, sin);
                } else if (turned) {
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const float m = v[0][j], n = v[0][j + 1];
                        v[0][j] = m * cos[j] - n * sin[j];
                        v[0][j + 1] = n * cos[j] + m * sin[j];
                    }
                }
#pragma unroll
                for (int w = 0; w < 2; w++) {
                    if (w == 1 && d1 < 0) break;
                    u32x4 o;
#pragma unroll
                    for (int j = 0; j < 4; j++) o[j] = pack2<F16>(v[w][2 * j], v[w][2 * j + 1]);
                    __builtin_memcpy(__builtin_assume_aligned(y + h * a.qo_head + (w ? d1 : d0), 2), &o, 16);
                }
            };
            if (few) {
                for (int h = h0 + (b0 & 7); h < h1; h += 8) {
                    u32x4 raw[2];
                    load(raw, h);
                    turn(raw, h);
                }
                continue;
            }
            // the result may be over its source, so that no load goes ahead of a store by itself: four heads are fetched, then turned
            // (4 x 8192 rows of 32 heads of 128 beside 8: 146 us, one by one 167; 2 x 1024 of 16 heads of 256 beside 16: 33 and 46)
            for (int h = h0; h < h1; h += 4) {
                u32x4 raw[4][2];
#pragma unroll
                for (int i = 0; i < 4; i++) load(raw[i], min(h + i, h1 - 1));
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (h + i < h1) turn(raw[i], h + i);
            }
        }
    }
}

// Eight values of a row to the output, in its type.
template <int TY>
__device__ __forceinline__ void put8(void *dst, long long at, const float *v)
{
    if constexpr (TY == MF_F32) {
        float *y = (float *)dst + at;
#pragma unroll
        for (int j = 0; j < 8; j++) y[j] = v[j];
    } else {
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; j++) o[j] = pack2<TY == MF_F16>(v[2 * j], v[2 * j + 1]);
        __builtin_memcpy(__builtin_assume_aligned((uint16_t *)dst + at, 2), &o, 16);
    }
}

// Launches of workgroups of 64 for n_seq sequences of `items` items and up to `span` tokens each: as many sequences to a
// launch as have room, and as many workgroups to an item as it has blocks of 16 or the launch has room; a kernel takes further blocks in turn.
template <class F>
inline hipError_t each_launch(int n_seq, int items, int span, const F &launch)
{
    const long long room = most_workgroups(64) / items, touched = (span + 14ll) / 16 + 1;
    for (int first = 0; first < n_seq;) {
        const int n = (int)(n_seq - first < room ? n_seq - first : room), blocks = (int)(touched < room / n ? touched : room / n);
        launch(first, (unsigned)((long long)n * items * blocks), blocks);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        first += n;
    }
    return hipSuccess;
}

}  // namespace mfs
