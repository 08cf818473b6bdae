// The paged cache in 8 bits: new rows into it (keys, and queries beside them,
// turned by their positions on the way), and rows of it read back.
//
// A wave takes one record (16 tokens of one head), whose keys share a scale and
// whose values do.  Lane l holds the dims 64 j + 16 (l / 16) .. + 15 of token l % 16:
// for keys 16 bytes of the record.  The values' order has 4 tokens in a dword; they
// are turned through 16 D bytes of LDS, [dim][token].  One wave owns a record, so
// nothing is written twice and no atomics are needed.
//
// Bound by the bytes where rows are many (4 prompts of 8192 tokens, 32 heads of queries over 8 of 128: 146 us for 742 MB, 5.1
// TB/s; read back 34 us), else by trips to memory, one after another: page number, rows, scale, codes (8 rows: 5.6 us,
// read back 4.3).
//
// A block that is begun (its earlier tokens were written by another call) keeps its
// scale where that is enough for the new tokens; where it is not the scale is doubled
// until it is, and the codes that are held are rounded to it.  Doubling bounds what
// a code loses over any number of calls: 1/2 + 1/4 + .. of a step, below one.
#include "mf_kv_rows.h"

namespace mfs {
namespace {

constexpr float kMostValue = 65504.f;

// A block's scale as it was and will be, and what takes codes from one to the other (1: they stay as they are).
struct Grown {
    float scale, inv, keep;
};
__device__ __forceinline__ Grown grow(uint32_t top, float old, bool begun)
{
    Grown g;
    const bool bad = top > 0x7f800000u;   // a NaN
    const float need = fmaxf(fminf(__uint_as_float(top), kMostValue) * (float)(1.0 / 127.0), kKv8LeastScale);
    // what is no scale is memory that was never written: the tokens before are zeros
    const bool held = begun && (old != old || (old >= kKv8LeastScale && old < kKv8MostScale));
    g.scale = need;
    if (held && old != kKv8LeastScale) {   // the least scale: zeros so far, or next to it
        const int ob = __float_as_int(old), nb = __float_as_int(need);
        // doubled no further than the largest value needs, so that none held is larger (in binary16, an infinity)
        g.scale = need <= old ? old : fminf(__int_as_float(ob + (((nb - ob + 0x7fffff) >> 23) << 23)), kMostValue * (float)(1.0 / 127.0));
    }
    if (bad || (held && old != old)) g.scale = NAN;
    g.keep = !begun || g.scale != g.scale || g.scale == old ? 1.f : held ? old / g.scale : 0.f;
    g.inv = g.scale != g.scale ? 0.f : 1.f / g.scale;
    return g;
}

__device__ __forceinline__ uint32_t code_of(float x, float inv)
{
    const float c = rintf(fminf(fmaxf(x, -kMostValue), kMostValue) * inv);
    return (uint32_t)(fminf(fmaxf(c, -127.f), 127.f) + 128.f);
}
// Four codes in a dword brought to another scale.
__device__ __forceinline__ uint32_t regrown(uint32_t w, float keep)
{
    uint32_t r = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const float c = rintf(((float)(w >> (8 * j) & 255) - 128.f) * keep);
        r |= (uint32_t)(fminf(fmaxf(c, -127.f), 127.f) + 128.f) << (8 * j);
    }
    return r;
}

template <int D>
__device__ __forceinline__ uint32_t top_of(const float (&v)[D / 64][16])
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < D / 64; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) top = max(top, __float_as_uint(v[j][e]) & 0x7fffffffu);
    return over_wave(top, [](uint32_t p, uint32_t q) { return max(p, q); });
}

template <bool F16, int D>
__device__ __forceinline__ void append_block(const KvAppendArgs &a, int s, int h, int blk, const Span &p, uint8_t *lds)
{
    constexpr int NC = D / 64;
    const long long record = kv8_record(a.g, a.b, s, h, blk);
    if (record < 0) return;   // the whole wave
    uint8_t *rec = a.g.pages + record * a.g.rec;
    KvScales *scales = kv8_scales(a.g) + record;
    const int lane = threadIdx.x & 63, tok = lane & 15, qt = lane >> 4, pos = blk * kKvBlock + tok;
    const bool live = pos >= p.lo && pos < p.hi, begun = p.lo > blk * kKvBlock;
    // tokens that are not written are computed as the last one that is
    const int at = max(p.lo, min(pos, p.hi - 1));
    const long long row = at + p.shift;
    const uint16_t *k = (const uint16_t *)a.k + row * a.k_stride + h * a.k_head, *x = (const uint16_t *)a.v + row * a.v_stride + h * a.v_head;
    u32x4 kraw[NC][2], vraw[NC][2];
#pragma unroll
    for (int j = 0; j < NC; j++)
#pragma unroll
        for (int e = 0; e < 2; e++) kraw[j][e] = load16(k + 64 * j + 16 * qt + 8 * e);
#pragma unroll
    for (int j = 0; j < NC; j++)
#pragma unroll
        for (int e = 0; e < 2; e++) vraw[j][e] = load16(x + 64 * j + 16 * qt + 8 * e);
    const KvScales old = *scales;
    uint32_t mine = 0;   // bytes of this lane's four tokens that are written
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const int q = blk * kKvBlock + 4 * qt + t;
        if (q >= p.lo && q < p.hi) mine |= 255u << (8 * t);
    }

    float v[NC][16];
    const float *cos = a.cos + (long long)at * (a.rot >> 1), *sin = a.sin + (long long)at * (a.rot >> 1);
    if (D >= 128 && a.rot == D && !a.interleaved) {
        // both halves are the lane's own
#pragma unroll
        for (int j = 0; j < NC; j++)
#pragma unroll
            for (int e = 0; e < 2; e++) widen8<F16>(kraw[j][e], v[j] + 8 * e);
#pragma unroll
        for (int j = 0; j < NC / 2; j++)
#pragma unroll
            for (int e = 0; e < 2; e++)
                turn_pair(v[j] + 8 * e, v[j + NC / 2] + 8 * e, cos + 64 * j + 16 * qt + 8 * e, sin + 64 * j + 16 * qt + 8 * e);
    } else if (D == 64 && a.rot == D && !a.interleaved) {
        // the halves are in lanes l and l ^ 32: both get both
        const bool second = lane >= 32;
#pragma unroll
        for (int e = 0; e < 2; e++) {
            u32x4 lo, hi;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const auto r = __builtin_amdgcn_permlane32_swap(kraw[0][e][i], kraw[0][e][i], false, false);
                lo[i] = r[0];
                hi[i] = r[1];
            }
            float x[8], y[8];
            widen8<F16>(lo, x);
            widen8<F16>(hi, y);
            turn_pair(x, y, cos + 16 * (qt & 1) + 8 * e, sin + 16 * (qt & 1) + 8 * e);
#pragma unroll
            for (int i = 0; i < 8; i++) v[0][8 * e + i] = second ? y[i] : x[i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < NC; j++)
#pragma unroll
            for (int e = 0; e < 2; e++) turn8<F16>(k, kraw[j][e], 64 * j + 16 * qt + 8 * e, a.rot, a.interleaved, cos, sin, v[j] + 8 * e);
    }
    const Grown gk = grow(top_of<D>(v), old.k, begun);   // cross-lane: every lane of the wave is here
    u32x4 *keys = (u32x4 *)rec + lane;
#pragma unroll
    for (int j = 0; j < NC; j++) {
        u32x4 w = {0, 0, 0, 0};
        if (live) {
#pragma unroll
            for (int e = 0; e < 16; e++) w[e >> 2] |= code_of(v[j][e], gk.inv) << (8 * (e & 3));
        } else if (gk.keep != 1.f) {
            w = keys[64 * j];
#pragma unroll
            for (int i = 0; i < 4; i++) w[i] = regrown(w[i], gk.keep);
        }
        if (live || gk.keep != 1.f) keys[64 * j] = w;
    }
#pragma unroll
    for (int j = 0; j < NC; j++)
#pragma unroll
        for (int e = 0; e < 2; e++) widen8<F16>(vraw[j][e], v[j] + 8 * e);
    const Grown gv = grow(top_of<D>(v), old.v, begun);
#pragma unroll
    for (int j = 0; j < NC; j++)
#pragma unroll
        for (int e = 0; e < 16; e++) lds[(64 * j + 16 * qt + e) * 16 + tok] = (uint8_t)code_of(v[j][e], gv.inv);
    __syncthreads();   // one wave a workgroup
    u32x4 *values = (u32x4 *)(rec + 16 * D) + lane;
    if (mine || gv.keep != 1.f) {
#pragma unroll
        for (int j = 0; j < NC; j++) {
            u32x4 w, o = {0, 0, 0, 0};
            if (mine != ~0u) o = values[64 * j];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                w[i] = *(const uint32_t *)(lds + (64 * j + 16 * i + tok) * 16 + 4 * qt);
                if (mine != ~0u) w[i] = (w[i] & mine) | ((gv.keep != 1.f ? regrown(o[i], gv.keep) : o[i]) & ~mine);
            }
            values[64 * j] = w;
        }
    }
    if (lane == 0) *scales = {gk.scale, gv.scale};
    __syncthreads();
}

// Work items as in the 4-bit cache's append.
template <bool F16, int D>
__global__ __launch_bounds__(64) void append8_kernel(KvAppendArgs a, int blocks, int slices, int few)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kKvBlock * D];
    const int items = a.g.n_kv_heads + slices;
    const int h = (int)(blockIdx.x % items), rest = (int)(blockIdx.x / items), s = a.first_seq + rest / blocks;
    const Span p = span_of(a.b, s);
    if (p.lo >= p.hi) return;
    if (h >= a.g.n_kv_heads) {
        const int part = h - a.g.n_kv_heads, h0 = part * a.n_heads / slices, h1 = (part + 1) * a.n_heads / slices;
        for (int b = rest % blocks; p.lo + b * 16 < p.hi; b += blocks) turn_queries<F16>(a, p, b, h0, h1, D, few);
        return;
    }
    for (int b = (p.lo >> 4) + rest % blocks; b * kKvBlock < p.hi; b += blocks) append_block<F16, D>(a, s, h, b, p, lds);
}

template <int TY, int D>   // TY: mf_dtype of the outputs
__global__ __launch_bounds__(64) void read8_kernel(KvReadArgs a, int blocks)
{
    constexpr int NC = D / 64;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kKvBlock * D];
    const int h = (int)(blockIdx.x % a.g.n_kv_heads), rest = (int)(blockIdx.x / a.g.n_kv_heads), s = a.first_seq + rest / blocks;
    const Span p = span_of(a.b, s);
    const int lane = threadIdx.x & 63, tok = lane & 15, qt = lane >> 4;
    for (int blk = (p.lo >> 4) + rest % blocks; blk * kKvBlock < p.hi; blk += blocks) {
        const int pos = blk * kKvBlock + tok;
        const bool live = pos >= p.lo && pos < p.hi;
        const long long record = kv8_record(a.g, a.b, s, h, blk);   // none: zeros
        const long long to = ((pos + p.shift) * a.g.n_kv_heads + h) * D;
        const uint8_t *rec = a.g.pages + (record < 0 ? 0 : record) * a.g.rec;
        KvScales sc = {0.f, 0.f};
        if (record >= 0) sc = kv8_scales(a.g)[record];
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            void *dst = kv ? a.v : a.k;
            if (!dst) continue;
            u32x4 w[NC];
#pragma unroll
            for (int j = 0; j < NC; j++) w[j] = record < 0 ? (u32x4){0, 0, 0, 0} : ((const u32x4 *)(rec + 16 * D * kv))[64 * j + lane];
            if (kv) {
                // the lane holds 4 tokens of a dim in a dword: to [dim][token]
                __syncthreads();
#pragma unroll
                for (int j = 0; j < NC; j++)
#pragma unroll
                    for (int i = 0; i < 4; i++) *(uint32_t *)(lds + (64 * j + 16 * i + tok) * 16 + 4 * qt) = w[j][i];
                __syncthreads();
            }
            const float scale = kv ? sc.v : sc.k;
#pragma unroll
            for (int j = 0; j < NC; j++)
#pragma unroll
                for (int e = 0; e < 16; e += 8) {
                    const int d = 64 * j + 16 * qt + e;
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const uint32_t c = kv ? lds[(d + i) * 16 + tok] : w[j][(e + i) >> 2] >> (8 * (i & 3)) & 255;
                        v[i] = scale * ((float)c - 128.f);
                    }
                    if (live) put8<TY>(dst, to + d, v);
                }
        }
    }
    // rows without a token of the cache
    for (long long r = p.row0 + rest % blocks; r < p.row1; r += blocks) {
        const long long at = r - p.shift;
        if (at >= p.lo && at < p.hi) {
            r += ((p.hi - 1 - at) / blocks) * blocks;   // on to the last of them
            continue;
        }
        const float zero[8] = {};
        for (int d = lane * 8; d < D; d += 64 * 8) {
            if (a.k) put8<TY>(a.k, (r * a.g.n_kv_heads + h) * D + d, zero);
            if (a.v) put8<TY>(a.v, (r * a.g.n_kv_heads + h) * D + d, zero);
        }
    }
}

template <int D>
void go_append(const KvAppendArgs &a, bool f16, unsigned grid, int blocks, int slices, int few, hipStream_t s)
{
    if (f16) hipLaunchKernelGGL((append8_kernel<true, D>), dim3(grid), dim3(64), 0, s, a, blocks, slices, few);
    else hipLaunchKernelGGL((append8_kernel<false, D>), dim3(grid), dim3(64), 0, s, a, blocks, slices, few);
}
template <int D>
void go_read(const KvReadArgs &a, int dtype, unsigned grid, int blocks, hipStream_t s)
{
    if (dtype == MF_F32) hipLaunchKernelGGL((read8_kernel<MF_F32, D>), dim3(grid), dim3(64), 0, s, a, blocks);
    else if (dtype == MF_BF16) hipLaunchKernelGGL((read8_kernel<MF_BF16, D>), dim3(grid), dim3(64), 0, s, a, blocks);
    else hipLaunchKernelGGL((read8_kernel<MF_F16, D>), dim3(grid), dim3(64), 0, s, a, blocks);
}

}  // namespace

hipError_t launch_kv8_append(const KvAppendArgs &args, bool f16, hipStream_t s)
{
    // eight heads of queries to a workgroup
    const int slices = args.q ? (args.n_heads + 7) / 8 : 0, few = args.b.max_new < 8;
    return each_launch(args.b.n_seq, args.g.n_kv_heads + slices, args.b.max_new, [&](int first, unsigned grid, int blocks) {
        KvAppendArgs a = args;
        a.first_seq = first;
        if (a.g.head_dim == 64) go_append<64>(a, f16, grid, blocks, slices, few, s);
        else if (a.g.head_dim == 128) go_append<128>(a, f16, grid, blocks, slices, few, s);
        else go_append<256>(a, f16, grid, blocks, slices, few, s);
    });
}

hipError_t launch_kv8_read(const KvReadArgs &args, int dtype, hipStream_t s)
{
    return each_launch(args.b.n_seq, args.g.n_kv_heads, args.b.max_new, [&](int first, unsigned grid, int blocks) {
        KvReadArgs a = args;
        a.first_seq = first;
        if (a.g.head_dim == 64) go_read<64>(a, dtype, grid, blocks, s);
        else if (a.g.head_dim == 128) go_read<128>(a, dtype, grid, blocks, s);
        else go_read<256>(a, dtype, grid, blocks, s);
    });
}

}  // namespace mfs
