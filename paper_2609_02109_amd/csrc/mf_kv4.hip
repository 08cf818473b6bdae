// The paged cache in 4 bits: new rows into it (keys, and queries beside them,
// turned by their positions on the way), and rows of it read back.
//
// A wave takes one record (16 tokens of one head).  Lane l holds the dims 32 i + 8
// (l / 16) .. + 7 of token l % 16: for keys eight codes of it are one dword of the
// record.  The values' order has 4 tokens in a dword; they are turned through 16 D
// bytes of LDS, [dim][token], of which four tokens are one word; a dword that holds
// other tokens' codes keeps those.  One wave owns a record, so nothing is written
// twice and no atomics are needed.
#include "mf_kv_rows.h"

namespace mfs {
namespace {

constexpr float kF16Max = 65504.f;

// Codes and scales of a token's values as the lane (token, l / 16) holds them: v[i][j] is dim 32 i + 8 (l / 16) + j.
template <int D, int G>
__device__ __forceinline__ void quantise(float v[D / 32][8], uint32_t code[D / 32][8], uint32_t meta[D / G])
{
    constexpr int IPG = G / 32;
#pragma unroll
    for (int g = 0; g < D / G; g++) {
        float lo = kF16Max, hi = -kF16Max, bad = 0.f;
#pragma unroll
        for (int i = g * IPG; i < (g + 1) * IPG; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) {
                if (v[i][j] != v[i][j]) bad = 1.f;
                v[i][j] = fminf(fmaxf(v[i][j], -kF16Max), kF16Max);
                lo = fminf(lo, v[i][j]);
                hi = fmaxf(hi, v[i][j]);
            }
        lo = quarters_min(lo);
        hi = quarters_max(hi);
        bad = quarters_max(bad);
        // two roundings, as the definition has it: left to itself the compiler makes one of them (v_fma_mixlo_f16)
        float step = (hi - lo) * (float)(1.0 / 15.0);
        asm("" : "+v"(step));
        const _Float16 scale = (_Float16)step, off = (_Float16)lo;
        const float s = (float)scale, o = (float)off, inv = s > 0.f ? 1.f / s : 0.f;
#pragma unroll
        for (int i = g * IPG; i < (g + 1) * IPG; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) code[i][j] = (uint32_t)fminf(fmaxf(rintf((v[i][j] - o) * inv), 0.f), 15.f);
        meta[g] = bad > 0.f ? 0x7e00u : bits<uint16_t>(scale) | (uint32_t)bits<uint16_t>(off) << 16;
    }
}

__device__ __forceinline__ uint32_t pack_codes(const uint32_t *c)
{
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 8; j++) w |= c[j] << (16 * (j & 1) + 4 * (j >> 1));
    return w;
}

// Bit of token t % 4 and dim d of a value dword (mf_serve.h).
constexpr __device__ int value_bit(int t, int d) { return 16 * (t & 1) + 4 * (2 * ((t >> 1) & 1) + ((d >> 4) & 1)); }

// Bytes of tokens 0 1 2 3 (two dims' codes each) to a value dword's order 0 2 1 3, and back.
__device__ __forceinline__ uint32_t value_order(uint32_t w) { return __builtin_amdgcn_perm(0u, w, 0x03010200u); }

// Where token t's scale of a group of the keys (0) or values (1) is in a record's tables.
template <int NG>
__device__ __forceinline__ int scale_at(int t, int kv, int g) { return (t >> 2) * 8 * NG + kv * 4 * NG + g * 4 + (t & 3); }

template <bool F16, int D, int G>
__device__ __forceinline__ void append_block(const KvAppendArgs &a, int s, int h, int blk, const Span &p, uint8_t *lds)
{
    constexpr int NS = D / 32, NG = D / G;
    uint8_t *rec = kv_record(a.g, a.b, s, h, blk);
    if (!rec) return;   // the whole wave
    const int lane = threadIdx.x & 63, tok = lane & 15, qt = lane >> 4, pos = blk * kKvBlock + tok;
    const bool live = pos >= p.lo && pos < p.hi;
    // tokens that are not written are computed as the last one that is
    const int at = max(p.lo, min(pos, p.hi - 1));
    const long long row = at + p.shift;
    const uint16_t *k = (const uint16_t *)a.k + row * a.k_stride + h * a.k_head, *x = (const uint16_t *)a.v + row * a.v_stride + h * a.v_head;
    u32x4 kraw[NS], vraw[NS];
#pragma unroll
    for (int i = 0; i < NS; i++) kraw[i] = load16(k + 32 * i + 8 * qt);
#pragma unroll
    for (int i = 0; i < NS; i++) vraw[i] = load16(x + 32 * i + 8 * qt);
    uint32_t mine = 0;   // tokens of this lane's four that are written
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const int q = blk * kKvBlock + 4 * qt + t;
        if (q >= p.lo && q < p.hi) mine |= 1u << t;
    }
    Words<NS> old;
    uint8_t *values = rec + 8 * D + lane * (D / 8);
    if (mine && mine != 15) old = load_words<NS>(values);

    float v[NS][8];
    uint32_t code[NS][8], meta[NG];
    uint16_t *table = (uint16_t *)(rec + 16 * D);   // scales, key offsets, value offsets (mf_serve.h)
    const float *cos = a.cos + (long long)at * (a.rot >> 1), *sin = a.sin + (long long)at * (a.rot >> 1);
    if (a.rot == D && !a.interleaved) {
        // both halves are the lane's own
#pragma unroll
        for (int i = 0; i < NS; i++) widen8<F16>(kraw[i], v[i]);
#pragma unroll
        for (int i = 0; i < NS / 2; i++) turn_pair(v[i], v[i + NS / 2], cos + 32 * i + 8 * qt, sin + 32 * i + 8 * qt);
    } else {
#pragma unroll
        for (int i = 0; i < NS; i++) turn8<F16>(k, kraw[i], 32 * i + 8 * qt, a.rot, a.interleaved, cos, sin, v[i]);
    }
    quantise<D, G>(v, code, meta);   // cross-lane: every lane of the wave is here
    if (live) {
        uint32_t w[NS];
#pragma unroll
        for (int i = 0; i < NS; i++) w[i] = pack_codes(code[i]);
        __builtin_memcpy(__builtin_assume_aligned(rec + lane * (D / 8), 8), w, D / 8);
#pragma unroll
        for (int g = 0; g < NG; g++)
            if ((g & 3) == qt) {
                table[scale_at<NG>(tok, 0, g)] = (uint16_t)meta[g];
                table[32 * NG + tok * NG + g] = (uint16_t)(meta[g] >> 16);
            }
    }
#pragma unroll
    for (int i = 0; i < NS; i++) widen8<F16>(vraw[i], v[i]);
    quantise<D, G>(v, code, meta);
    if (live) {
#pragma unroll
        for (int g = 0; g < NG; g++)
            if ((g & 3) == qt) {
                table[scale_at<NG>(tok, 1, g)] = (uint16_t)meta[g];
                table[48 * NG + g * 16 + tok] = (uint16_t)(meta[g] >> 16);
            }
    }
#pragma unroll
    for (int i = 0; i < NS; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) lds[(32 * i + 8 * qt + j) * 16 + tok] = (uint8_t)code[i][j];
    __syncthreads();   // one wave a workgroup
    if (mine) {
        uint32_t keep = 0;
#pragma unroll
        for (int t = 0; t < 4; t++)
            if (!(mine >> t & 1)) keep |= 0xffu << value_bit(t, 0);
        uint32_t w[NS];
#pragma unroll
        for (int i = 0; i < NS; i++) {
            const uint32_t even = *(const uint32_t *)(lds + (32 * i + tok) * 16 + 4 * qt), odd = *(const uint32_t *)(lds + (32 * i + 16 + tok) * 16 + 4 * qt);
            w[i] = value_order(even | odd << 4);
            if (mine != 15) w[i] = (w[i] & ~keep) | (old.w[i] & keep);
        }
        __builtin_memcpy(__builtin_assume_aligned(values, 8), w, D / 8);
    }
    __syncthreads();
}

// Work item: (sequence, 16 positions, head), the numbers past the heads standing for
// slices of the queries' heads: few tokens or many, there is a wave for each 16 of a head.
// Bound by the bytes of rows and queries from some thousand rows on (32768 rows of 32 + 2 x
// 8 heads of 128: 142 us for 747 MB, 5.3 TB/s, a copy 5.2), below that by one trip to
// memory after another (a row each of 8 requests: 5.8 us).
template <bool F16, int D, int G>
__global__ __launch_bounds__(64) void append_kernel(KvAppendArgs a, int blocks, int slices, int few)
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
    for (int b = (p.lo >> 4) + rest % blocks; b * kKvBlock < p.hi; b += blocks) append_block<F16, D, G>(a, s, h, b, p, lds);
}

// Rows back, a wave per 16 positions of a head as in the append; bound by the bytes written
// (32768 rows of 2 x 8 heads of 128: 49 us for 210 MB, 4.3 TB/s) or by the trip to
// memory (8 rows: 4.3 us).
template <int TY, int D, int G>   // TY: mf_dtype of the outputs
__global__ __launch_bounds__(64) void read_kernel(KvReadArgs a, int blocks)
{
    constexpr int NS = D / 32, NG = D / G;
    __shared__ __attribute__((aligned(16))) uint8_t lds[kKvBlock * D];
    const int h = (int)(blockIdx.x % a.g.n_kv_heads), rest = (int)(blockIdx.x / a.g.n_kv_heads), s = a.first_seq + rest / blocks;
    const Span p = span_of(a.b, s);
    const int lane = threadIdx.x & 63, tok = lane & 15, qt = lane >> 4;
    for (int blk = (p.lo >> 4) + rest % blocks; blk * kKvBlock < p.hi; blk += blocks) {
        const int pos = blk * kKvBlock + tok;
        const bool live = pos >= p.lo && pos < p.hi;
        const uint8_t *rec = kv_record(a.g, a.b, s, h, blk);   // none: zeros
        const long long to = ((pos + p.shift) * a.g.n_kv_heads + h) * D;
        const uint16_t *table = rec ? (const uint16_t *)(rec + 16 * D) : nullptr;
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            void *dst = kv ? a.v : a.k;
            if (!dst) continue;
            Words<NS> w = {};
            float sc[NG] = {}, off[NG] = {};
            if (rec) {
                w = load_words<NS>(rec + 8 * D * kv + lane * (D / 8));
#pragma unroll
                for (int g = 0; g < NG; g++) {
                    sc[g] = to_float<true>(table[scale_at<NG>(tok, kv, g)]);
                    off[g] = to_float<true>(table[kv ? 48 * NG + g * 16 + tok : 32 * NG + tok * NG + g]);
                }
            }
            if (kv) {
                // the lane holds 4 tokens of two dims a dword: to [dim][token]
                __syncthreads();
#pragma unroll
                for (int i = 0; i < NS; i++) {
                    const uint32_t x = value_order(w.w[i]);
                    *(uint32_t *)(lds + (32 * i + tok) * 16 + 4 * qt) = x & 0x0f0f0f0fu;
                    *(uint32_t *)(lds + (32 * i + 16 + tok) * 16 + 4 * qt) = x >> 4 & 0x0f0f0f0fu;
                }
                __syncthreads();
            }
#pragma unroll
            for (int i = 0; i < NS; i++) {
                const int d = 32 * i + 8 * qt;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const uint32_t c = kv ? lds[(d + j) * 16 + tok] : w.w[i] >> (16 * (j & 1) + 4 * (j >> 1)) & 15;
                    v[j] = off[32 * i / G] + sc[32 * i / G] * (float)c;
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

template <bool F16, int D, int G>
void go_append(const KvAppendArgs &a, unsigned grid, int blocks, int slices, int few, hipStream_t s)
{
    hipLaunchKernelGGL((append_kernel<F16, D, G>), dim3(grid), dim3(64), 0, s, a, blocks, slices, few);
}
template <int TY, int D, int G>
void go_read(const KvReadArgs &a, unsigned grid, int blocks, hipStream_t s)
{
    hipLaunchKernelGGL((read_kernel<TY, D, G>), dim3(grid), dim3(64), 0, s, a, blocks);
}

}  // namespace

#define MFS_FOR_SHAPE(g, CALL)                                                                      \
    if ((g).head_dim == 64) { if ((g).group == 32) { CALL(64, 32); } else { CALL(64, 64); } }       \
    else if ((g).head_dim == 128) {                                                                 \
        if ((g).group == 32) { CALL(128, 32); } else if ((g).group == 64) { CALL(128, 64); } else { CALL(128, 128); } } \
    else { if ((g).group == 32) { CALL(256, 32); } else if ((g).group == 64) { CALL(256, 64); } else { CALL(256, 128); } }

hipError_t launch_kv4_append(const KvAppendArgs &args, bool f16, hipStream_t s)
{
    // eight heads of queries to a workgroup
    const int slices = args.q ? (args.n_heads + 7) / 8 : 0, few = args.b.max_new < 8;
    return each_launch(args.b.n_seq, args.g.n_kv_heads + slices, args.b.max_new, [&](int first, unsigned grid, int blocks) {
        KvAppendArgs a = args;
        a.first_seq = first;
#define CALL(D, G) f16 ? go_append<true, D, G>(a, grid, blocks, slices, few, s) : go_append<false, D, G>(a, grid, blocks, slices, few, s)
        MFS_FOR_SHAPE(a.g, CALL)
#undef CALL
    });
}

hipError_t launch_kv4_read(const KvReadArgs &args, int dtype, hipStream_t s)
{
    return each_launch(args.b.n_seq, args.g.n_kv_heads, args.b.max_new, [&](int first, unsigned grid, int blocks) {
        KvReadArgs a = args;
        a.first_seq = first;
#define CALL(D, G) dtype == MF_F32 ? go_read<MF_F32, D, G>(a, grid, blocks, s) \
                                   : dtype == MF_BF16 ? go_read<MF_BF16, D, G>(a, grid, blocks, s) : go_read<MF_F16, D, G>(a, grid, blocks, s)
        MFS_FOR_SHAPE(a.g, CALL)
#undef CALL
    });
}

}  // namespace mfs
