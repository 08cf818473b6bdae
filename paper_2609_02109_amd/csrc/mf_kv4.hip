// The paged cache in 4 bits: new rows into it (keys, and queries beside them,
// turned by their positions on the way), and rows of it read back.
//
// A wave takes one record (16 tokens of one head).  For keys, lane l holds the
// dims 32 i + 8 (l / 16) .. + 7 of token l % 16: eight codes of it are one dword
// of the record, so a lane writes what it computed, 4 lanes a token.  The
// values' order has 4 tokens in a dword; they are turned through 16 D bytes of
// LDS, and a dword that holds other tokens' codes keeps those.  One wave owns
// a record, so nothing is written twice and no atomics are needed.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

constexpr float kF16Max = 65504.f;

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

// Eight values of a row turned by its position: dims d .. d + 7 of a head at x.
// Each product and sum is rounded by itself (the library is compiled without
// contraction), as the definition has it.
template <bool F16>
__device__ __forceinline__ void turn8(const uint16_t *x, int d, int rot, int inter, const float *cos, const float *sin, float *v)
{
    const u32x4 own = load16(x + d);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = to_float<F16>((uint16_t)(own[j >> 1] >> (16 * (j & 1))));
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
    const u32x4 far = load16(x + (second ? t : t + half));
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float c = cos[t + j], s = sin[t + j], y = to_float<F16>((uint16_t)(far[j >> 1] >> (16 * (j & 1))));
        v[j] = second ? v[j] * c + y * s : v[j] * c - y * s;
    }
}

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
        _Float16 scale = (_Float16)((hi - lo) * (float)(1.0 / 15.0)), off = (_Float16)lo;
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
__device__ __forceinline__ int value_bit(int t, int d) { return 16 * (t & 1) + 4 * (2 * ((t >> 1) & 1) + ((d >> 4) & 1)); }

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
    const long long row = pos + p.shift;
    float v[NS][8];
    uint32_t code[NS][8], meta[NG];
    uint16_t *table = (uint16_t *)(rec + 16 * D);   // scales, key offsets, value offsets (mf_serve.h)
    if (live) {
        const uint16_t *k = (const uint16_t *)a.k + row * a.k_stride + h * a.k_head;
        const float *cos = a.cos ? a.cos + (long long)pos * (a.rot >> 1) : nullptr;
        const float *sin = a.cos ? a.sin + (long long)pos * (a.rot >> 1) : nullptr;
#pragma unroll
        for (int i = 0; i < NS; i++) turn8<F16>(k, 32 * i + 8 * qt, a.rot, a.interleaved, cos, sin, v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < NS; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) v[i][j] = 0.f;
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
        const uint16_t *x = (const uint16_t *)a.v + row * a.v_stride + h * a.v_head;
#pragma unroll
        for (int i = 0; i < NS; i++) turn8<F16>(x, 32 * i + 8 * qt, 0, 0, nullptr, nullptr, v[i]);
    }
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
    for (int i = 0; i < NS; i++) {
        u32x2 b = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; j++) b[j >> 2] |= code[i][j] << (8 * (j & 3));
        *(u32x2 *)(lds + tok * D + 32 * i + 8 * qt) = b;
    }
    __syncthreads();   // one wave a workgroup
    uint32_t mine = 0;   // tokens of this lane's four that are written
#pragma unroll
    for (int t = 0; t < 4; t++) {
        const int q = blk * kKvBlock + 4 * qt + t;
        if (q >= p.lo && q < p.hi) mine |= 1u << t;
    }
    if (mine) {
        uint32_t *out = (uint32_t *)(rec + 8 * D + lane * (D / 8));
#pragma unroll
        for (int i = 0; i < NS; i++) {
            uint32_t w = 0, keep = 0;
#pragma unroll
            for (int t = 0; t < 4; t++)
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    const int d = 32 * i + 16 * u + tok, bit = value_bit(t, d);
                    if (mine >> t & 1) w |= (uint32_t)lds[(4 * qt + t) * D + d] << bit;
                    else keep |= 15u << bit;
                }
            if (keep) w |= out[i] & keep;
            out[i] = w;
        }
    }
    __syncthreads();
}

template <bool F16>
__device__ __forceinline__ void turn_queries(const KvAppendArgs &a, const Span &p, int blk, int D)
{
    // 8 dims of every head of 16 tokens; a pair of halves is one thread's, so that the result may go over its source
    const int base = p.lo + blk * 16, half = a.rot >> 1;
    const int units = a.interleaved ? D / 8 : (D - half) / 8;   // a unit below rot / 2 takes its partner along
    for (int e = (int)threadIdx.x; e < 16 * a.n_heads * units; e += (int)blockDim.x) {
        const int u = e % units, th = e / units, h = th % a.n_heads, pos = base + th / a.n_heads;
        if (pos < p.lo || pos >= p.hi) continue;
        const long long row = pos + p.shift;
        const uint16_t *x = (const uint16_t *)a.q + row * a.q_stride + h * a.q_head;
        uint16_t *y = (uint16_t *)a.q_out + row * a.qo_stride + h * a.qo_head;
        const float *cos = a.cos + (long long)pos * half, *sin = a.sin + (long long)pos * half;
        int d[2] = {u * 8, -1};
        if (!a.interleaved) {
            if (d[0] < half) d[1] = d[0] + half;
            else d[0] += half;
        }
        float v[2][8];
        turn8<F16>(x, d[0], a.rot, a.interleaved, cos, sin, v[0]);
        if (d[1] >= 0) turn8<F16>(x, d[1], a.rot, a.interleaved, cos, sin, v[1]);
        for (int w = 0; w < 2; w++) {
            if (d[w] < 0) continue;
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; j++) o[j] = pack2<F16>(v[w][2 * j], v[w][2 * j + 1]);
            __builtin_memcpy(__builtin_assume_aligned(y + d[w], 2), &o, 16);
        }
    }
}

// Work item: (sequence, 16 positions, head), the last head number standing for the queries.
template <bool F16, int D, int G>
__global__ __launch_bounds__(64) void append_kernel(KvAppendArgs a, int blocks, int heads)
{
    __shared__ __attribute__((aligned(16))) uint8_t lds[kKvBlock * D];
    const int h = (int)(blockIdx.x % heads), rest = (int)(blockIdx.x / heads), s = rest / blocks;
    const Span p = span_of(a.b, s);
    if (p.lo >= p.hi) return;
    if (h == a.g.n_kv_heads) {
        for (int b = rest % blocks; p.lo + b * 16 < p.hi; b += blocks) turn_queries<F16>(a, p, b, D);
        return;
    }
    for (int b = (p.lo >> 4) + rest % blocks; b * kKvBlock < p.hi; b += blocks) append_block<F16, D, G>(a, s, h, b, p, lds);
}

template <int TY, int D, int G>   // TY: mf_dtype of the outputs
__global__ __launch_bounds__(64) void read_kernel(KvReadArgs a, int blocks)
{
    constexpr int NS = D / 32, NG = D / G;
    const int h = (int)(blockIdx.x % a.g.n_kv_heads), rest = (int)(blockIdx.x / a.g.n_kv_heads), s = rest / blocks;
    const Span p = span_of(a.b, s);
    const int lane = threadIdx.x & 63, tok = lane & 15, qt = lane >> 4;
    // every row of the step is written: those without a token of the cache with zeros
    for (long long r = p.row0 + 16ll * (rest % blocks); r < p.row1; r += 16ll * blocks) {
        // rows r .. r + 15 are tokens of one record or two
        const long long row = r + tok, at = row - p.shift;
        if (row >= p.row1) continue;
        const bool live = at >= p.lo && at < p.hi;
        const int pos = live ? (int)at : 0, in = pos & 15;
        const uint8_t *rec = live ? kv_record(a.g, a.b, s, h, pos >> 4) : nullptr;
        const long long to = (row * a.g.n_kv_heads + h) * D;
#pragma unroll
        for (int kv = 0; kv < 2; kv++) {
            void *dst = kv ? a.v : a.k;
            if (!dst) continue;
#pragma unroll
            for (int i = 0; i < NS; i++) {
                const int d = 32 * i + 8 * qt;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = 0.f;
                if (rec) {
                    const uint16_t *table = (const uint16_t *)(rec + 16 * D);
                    const int g = d / G;
                    const float sc = to_float<true>(table[scale_at<NG>(in, kv, g)]),
                                off = to_float<true>(table[kv ? 48 * NG + g * 16 + in : 32 * NG + in * NG + g]);
                    const uint32_t w = kv ? 0u : ((const uint32_t *)(rec + (qt * 16 + in) * (D / 8)))[i];
#pragma unroll
                    for (int j = 0; j < 8; j++) {
                        const uint32_t c = kv ? ((const uint32_t *)(rec + 8 * D + ((in >> 2) * 16 + ((d + j) & 15)) * (D / 8)))[i] >> value_bit(in, d + j)
                                              : w >> (16 * (j & 1) + 4 * (j >> 1));
                        v[j] = off + sc * (float)(c & 15);
                    }
                }
                if (TY == MF_F32) {
                    float *y = (float *)dst + to + d;
#pragma unroll
                    for (int j = 0; j < 8; j++) y[j] = v[j];
                } else {
                    u32x4 o;
#pragma unroll
                    for (int j = 0; j < 4; j++) o[j] = pack2<TY == MF_F16>(v[2 * j], v[2 * j + 1]);
                    __builtin_memcpy(__builtin_assume_aligned((uint16_t *)dst + to + d, 2), &o, 16);
                }
            }
        }
    }
}

template <bool F16, int D, int G>
void go_append(const KvAppendArgs &a, unsigned grid, int blocks, int heads, hipStream_t s)
{
    hipLaunchKernelGGL((append_kernel<F16, D, G>), dim3(grid), dim3(64), 0, s, a, blocks, heads);
}
template <int TY, int D, int G>
void go_read(const KvReadArgs &a, unsigned grid, int blocks, hipStream_t s)
{
    hipLaunchKernelGGL((read_kernel<TY, D, G>), dim3(grid), dim3(64), 0, s, a, blocks);
}

// Workgroups a sequence gets for its blocks of 16, so that the grid stays within 2^30; a kernel takes further blocks in turn.
int blocks_for(long long span, long long others)
{
    long long b = (span + 14) / 16 + 1;   // 16-blocks that span tokens can touch
    const long long most = (1ll << 30) / (others > 0 ? others : 1);
    return (int)(b < most ? b : most > 1 ? most : 1);
}

}  // namespace

#define MFS_FOR_SHAPE(g, CALL)                                                                      \
    if ((g).head_dim == 64) { if ((g).group == 32) { CALL(64, 32); } else { CALL(64, 64); } }       \
    else if ((g).head_dim == 128) {                                                                 \
        if ((g).group == 32) { CALL(128, 32); } else if ((g).group == 64) { CALL(128, 64); } else { CALL(128, 128); } } \
    else { if ((g).group == 32) { CALL(256, 32); } else if ((g).group == 64) { CALL(256, 64); } else { CALL(256, 128); } }

hipError_t launch_kv4_append(const KvAppendArgs &a, bool f16, hipStream_t s)
{
    const int heads = a.g.n_kv_heads + (a.q ? 1 : 0);
    const int blocks = blocks_for(a.b.max_new, (long long)a.b.n_seq * heads);
    const unsigned grid = (unsigned)((long long)a.b.n_seq * heads * blocks);
#define CALL(D, G) f16 ? go_append<true, D, G>(a, grid, blocks, heads, s) : go_append<false, D, G>(a, grid, blocks, heads, s)
    MFS_FOR_SHAPE(a.g, CALL)
#undef CALL
    return hipGetLastError();
}

hipError_t launch_kv4_read(const KvReadArgs &a, int dtype, hipStream_t s)
{
    const int blocks = blocks_for(a.b.max_new, (long long)a.b.n_seq * a.g.n_kv_heads);
    const unsigned grid = (unsigned)((long long)a.b.n_seq * a.g.n_kv_heads * blocks);
#define CALL(D, G) dtype == MF_F32 ? go_read<MF_F32, D, G>(a, grid, blocks, s) \
                                   : dtype == MF_BF16 ? go_read<MF_BF16, D, G>(a, grid, blocks, s) : go_read<MF_F16, D, G>(a, grid, blocks, s)
    MFS_FOR_SHAPE(a.g, CALL)
#undef CALL
    return hipGetLastError();
}

}  // namespace mfs
