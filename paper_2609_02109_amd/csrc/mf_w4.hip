// Products with 4-bit weights and group scales: y = x W^T + bias,
// W[n][k] = s (c - z).  With P = sum_k (16 + c) x and X = sum_k x over a group,
// both from matrix instructions, the group's part is s (P - (16 + z) X): the
// codes go into the instruction as they are, and scale and zero point cost two
// fp32 operations a group and output instead of one a weight.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

__device__ __forceinline__ uint32_t low_nibbles(uint32_t v)
{
    v &= 0x0f0f0f0fu;
    v = (v | v >> 4) & 0x00ff00ffu;
    return (v | v >> 8) & 0xffffu;
}

// A wave per record: 16 rows of 64 bytes of codes in, 1 KB in a row out, then the scales.
// Once a weight (134 MB of codes: 87 us; a workgroup a record, by single bytes, 106).
__global__ __launch_bounds__(256) void w4_pack_kernel(W4PackArgs a)
{
    const int tiles = (a.n_out + kW4Tile - 1) / kW4Tile, chunks = (a.n_in + kW4Chunk - 1) / kW4Chunk, rec = w4_record(a.group), gpc = kW4Chunk / a.group;
    const long long row_bytes = a.n_in / 2, groups = a.n_in / a.group;
    const int lane = threadIdx.x & 63, chunk = (int)blockIdx.x * 4 + wave_id();
    if (chunk >= chunks) return;
    for (int tile = (int)blockIdx.y; tile < tiles; tile += (int)gridDim.y) {
        uint8_t *out = a.packed + ((long long)tile * chunks + chunk) * rec;
        const int n = tile * kW4Tile + (lane & 15);
        u32x4 w = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int k = chunk * kW4Chunk + i * 32 + (lane >> 4) * 8;
            if (n < a.n_out && k < a.n_in) {
                uint32_t v;
                __builtin_memcpy(&v, a.codes + n * row_bytes + k / 2, 4);
                w[i] = low_nibbles(v) | low_nibbles(v >> 4) << 16;
            }
        }
        ((u32x4 *)out)[lane] = w;
        if (lane >= 16 * gpc) continue;
        const int g = chunk * gpc + (lane >> 4);
        uint32_t m = 0;
        if (n < a.n_out && g < groups) {
            const long long at = n * groups + g;
            const float z = 16.f + (float)(a.zeros ? a.zeros[at] & 15 : 8);
            m = a.scales[at] | (uint32_t)(a.f16 ? from_float<true>(z) : from_float<false>(z)) << 16;
        }
        ((uint32_t *)(out + kW4Codes))[lane] = m;
    }
}

// Four outputs n .. n + 3 of row m: bias, rounding, and the edge.
template <bool F16>
__device__ __forceinline__ void store4(const W4Args &a, int m, int n, f32x4 sum)
{
    uint16_t *y = (uint16_t *)a.y + (long long)m * a.y_stride + n;
    const int many = a.n_out - n < 4 ? a.n_out - n : 4;
    if (a.bias)
        for (int r = 0; r < many; r++) sum[r] += to_float<F16>(((const uint16_t *)a.bias)[n + r]);
    if (many == 4 && ((uintptr_t)y & 7) == 0) {
        *(u32x2 *)y = (u32x2){pack2<F16>(sum[0], sum[1]), pack2<F16>(sum[2], sum[3])};
    } else {
        for (int r = 0; r < many; r++) y[r] = from_float<F16>(sum[r]);
    }
}

// A wave's share of a chunk: codes and scales of NT tiles of 16 outputs.
template <int G, int NT>
struct W4Chunk {
    static constexpr int GPC = kW4Chunk / G;
    u32x4 w[NT], meta[NT][GPC];
    __device__ __forceinline__ void load(const uint8_t *const (&wp)[NT], long long at, int lane)
    {
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const uint8_t *r = wp[t] + at;
            w[t] = *(const u32x4 *)(r + lane * 16);
#pragma unroll
            for (int g = 0; g < GPC; g++) meta[t][g] = *(const u32x4 *)(r + kW4Codes + g * 64 + (lane >> 4) * 16);
        }
    }
};

// Few rows (bound by the weights' bytes: 8 rows of 32768 x 8192 in groups of 128 take 30 us
// for 140 MB, 4.7 TB/s; small layers by the trip to memory and the sum through LDS: 1 x 4096
// x 4096 4.5 us).
// A workgroup takes NT tiles of 16 outputs and MT tiles of 16 rows; its NW waves
// take every NW-th chunk of 128 inputs, the next chunk on its way while one is
// computed, and add up through LDS at the end, in wave order.  The operand of the
// rows has 16 rows in 16 neighbouring lanes, which as a load from memory are 16
// lines for 256 bytes (8 TB/s over the card, which bounded every product of 8
// rows and more): the wave reads whole rows and turns them through LDS of its own.
template <bool F16, int G, int MT, int NT, int NW>
__global__ __launch_bounds__(NW * 64) void w4_kernel(W4Args a)
{
    constexpr int GPC = kW4Chunk / G, IPG = G / 32, REC = w4_record(G);
    // rows as 16-byte pieces, piece p of row r at p ^ r, so that neither side meets a bank twice; later the sums
    constexpr int STAGE = MT * 16 * 16, SUMS = MT * NT * 64;
    __shared__ u32x4 lds[NW * (STAGE > SUMS ? STAGE : SUMS)];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW4Tile - 1) / kW4Tile, chunks = (a.n_in + kW4Chunk - 1) / kW4Chunk;
    const int tile0 = (int)blockIdx.x * NT, m0 = (int)blockIdx.y * MT * 16;
    const uint8_t *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int tile = tile0 + t < n_tiles ? tile0 + t : n_tiles - 1;   // past the end: computed again, not stored
        wp[t] = a.packed + (long long)tile * chunks * REC;
    }
    u32x4 *stage = lds + wave * STAGE;
    const uint16_t *xp[MT * 4];
#pragma unroll
    for (int j = 0; j < MT * 4; j++) {
        const int m = m0 + 4 * j + qt;
        xp[j] = (const uint16_t *)a.x + (long long)(m < a.rows ? m : a.rows - 1) * a.x_stride;
    }
    const CodeBits cb = code_bits<F16>();
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    // rows 4 j + lane / 16, piece lane % 16: past the rows the last one (it is not stored), past the
    // inputs the row's last piece (its scale is 0)
    u32x4 raw[MT * 4];
    const auto load_x = [&](int c) {
        const int k = min(c * kW4Chunk + col * 8, a.n_in - 8);
#pragma unroll
        for (int j = 0; j < MT * 4; j++) {
            if (m0 + 4 * j >= a.rows) break;
            raw[j] = load16(xp[j] + k);
        }
    };
    f32x4 acc[MT][NT] = {};
    W4Chunk<G, NT> now;
    if (wave < chunks) {
        now.load(wp, (long long)wave * REC, lane);
        load_x(wave);
    }
    for (int c = wave; c < chunks; c += NW) {
        // the waves' pieces are their own: the order of a wave's own accesses is enough
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int j = 0; j < MT * 4; j++) {
            if (m0 + 4 * j >= a.rows) break;
            const int r = 4 * j + qt;
            stage[r * 16 + (col ^ (r & 15))] = raw[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        W4Chunk<G, NT> next;
        const bool more = c + NW < chunks;
        if (more) {
            next.load(wp, (long long)(c + NW) * REC, lane);
            load_x(c + NW);
        }
#pragma unroll
        for (int g = 0; g < GPC; g++) {
            u32x4 x[MT][IPG];
            f32x4 X[MT];
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int i = 0; i < IPG; i++) {
                    x[m][i] = stage[(m * 16 + col) * 16 + ((4 * (g * IPG + i) + qt) ^ col)];
                    X[m] = mfma<F16>(ones8<F16>(), x[m][i], i ? X[m] : zero);
                }
#pragma unroll
            for (int t = 0; t < NT; t++) {
                f32x4 P[MT];
#pragma unroll
                for (int i = 0; i < IPG; i++) {
                    const u32x4 A = codes8<F16>(now.w[t][g * IPG + i], cb);
#pragma unroll
                    for (int m = 0; m < MT; m++) P[m] = mfma<F16>(A, x[m][i], i ? P[m] : zero);
                }
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float s = to_float<F16>((uint16_t)now.meta[t][g][r]), z = to_float<F16>((uint16_t)(now.meta[t][g][r] >> 16));
#pragma unroll
                    for (int m = 0; m < MT; m++) acc[m][t][r] = fmaf(s, fmaf(-z, X[m][r], P[m][r]), acc[m][t][r]);
                }
            }
        }
        if (more) now = next;
    }
    f32x4 *red = (f32x4 *)lds;
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int t = 0; t < NT; t++) red[(wave * MT * NT + m * NT + t) * 64 + lane] = acc[m][t];
    __syncthreads();
    for (int e = (int)threadIdx.x; e < SUMS; e += NW * 64) {
        const int l = e & 63, mt = e >> 6, m = m0 + (mt / NT) * 16 + (l & 15);
        const int n = (tile0 + mt % NT) * kW4Tile + (l >> 4) * 4;
        f32x4 sum = red[e];
#pragma unroll
        for (int v = 1; v < NW; v++) sum += red[v * SUMS + e];
        if (m < a.rows && n < a.n_out) store4<F16>(a, m, n, sum);
    }
}

// Sum of eight 16-bit values (dot products of pairs with ones, in fp32).
template <bool F16>
__device__ __forceinline__ float sum8(u32x4 v)
{
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if (F16) s = __builtin_amdgcn_fdot2(bits<f16x2>(v[j]), bits<f16x2>(0x3c003c00u), s, false);
        else s = __builtin_amdgcn_fdot2_f32_bf16(bits<bf16x2>(v[j]), bits<bf16x2>(0x3f803f80u), s, false);
    }
    return s;
}

// A neighbour's value: quad_perm, row_half_mirror, row_mirror.
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// Many rows (bound by the issue of two waves a SIMD: at 64 x 32768 x 8192, 48 us, vector
// instructions take 43 % of the cycles, matrix ones 27 %, and little of the two runs at
// once; the codes' conversion and scale and zero point are most of the first.  Four chunks
// in LDS for one barrier took as long: 57 us, at 512 rows 87 for 82).
// All NW waves of a workgroup take the same chunk, for NT tiles of 16
// outputs each, so that the rows come from memory once for 16 NW NT outputs.  A
// chunk of MT x 16 rows goes into LDS (pieces as above) with its groups' sums
// while the one before is computed; rows and weights are DEEP chunks ahead in
// registers (loads return in order: the one that is awaited has to be as old as
// all the others).  blockIdx.y: the part of the inputs, blockIdx.z: the block of rows.
template <bool F16, int G, int MT, int NT, int NW, int DEEP>
__global__ __launch_bounds__(NW * 64) void w4_rows_kernel(W4Args a, int splits, float *part)
{
    constexpr int GPC = kW4Chunk / G, IPG = G / 32, REC = w4_record(G), ROWS = MT * 16, PIECES = ROWS * 16, MINE = PIECES / (NW * 64);
    static_assert(MINE >= 1 && MINE * NW * 64 == PIECES && DEEP % 2 == 0, "whole pieces a thread, rounds end where they began");
    __shared__ u32x4 stage[2][PIECES];
    __shared__ float sums[2][GPC][ROWS];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW4Tile - 1) / kW4Tile, chunks = (a.n_in + kW4Chunk - 1) / kW4Chunk;
    const int tile0 = ((int)blockIdx.x * NW + wave) * NT, m0 = (int)blockIdx.z * ROWS;
    const int rounds = (chunks + DEEP - 1) / DEEP;
    const int c0 = (int)((long long)rounds * blockIdx.y / splits) * DEEP, c1 = min((int)((long long)rounds * (blockIdx.y + 1) / splits) * DEEP, chunks);
    const uint8_t *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int tile = tile0 + t < n_tiles ? tile0 + t : n_tiles - 1;   // past the end: computed again, not stored
        wp[t] = a.packed + (long long)tile * chunks * REC;
    }
    // this thread's pieces: rows r0 + j * (NW * 4), piece threadIdx.x % 16
    const int r0 = (int)threadIdx.x >> 4, piece = (int)threadIdx.x & 15;
    const uint16_t *xp[MINE];
#pragma unroll
    for (int j = 0; j < MINE; j++) {
        const int m = m0 + r0 + j * NW * 4;
        xp[j] = (const uint16_t *)a.x + (long long)(m < a.rows ? m : a.rows - 1) * a.x_stride;
    }
    // always a load, so that the compiler can count them: past the rows the last one (it is not stored),
    // past the inputs the row's last piece (its scale is 0), past the part some chunk (it is not used)
    u32x4 raw[DEEP][MINE];
    const auto fetch = [&](u32x4 (&raw)[MINE], int c) {
        const int k = min(c * kW4Chunk + piece * 8, a.n_in - 8);
#pragma unroll
        for (int j = 0; j < MINE; j++) raw[j] = load16(xp[j] + k);
    };
    const auto put = [&](const u32x4 (&raw)[MINE], int buf) {
#pragma unroll
        for (int j = 0; j < MINE; j++) {
            const int r = r0 + j * NW * 4;
            stage[buf][r * 16 + (piece ^ (r & 15))] = raw[j];
            float s = sum8<F16>(raw[j]);
            // over the group's pieces, which are neighbouring lanes: within four, the other four, the other eight
            s += dpp<0xb1>(s);
            s += dpp<0x4e>(s);
            if (G >= 64) s += dpp<0x141>(s);
            if (G >= 128) s += dpp<0x140>(s);
            if (piece % (G / 8) == 0) sums[buf][piece / (G / 8)][r] = s;
        }
    };
    const CodeBits cb = code_bits<F16>();
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    f32x4 acc[MT][NT] = {};
    W4Chunk<G, NT> w[DEEP];
    // in the order of the loop, so that at its head the compiler counts the same loads from both sides
    fetch(raw[0], c0);
#pragma unroll
    for (int d = 0; d < DEEP; d++) {
        if (d == DEEP - 1) put(raw[0], 0);
        fetch(raw[(d + 1) % DEEP], c0 + d + 1);
        w[d].load(wp, (long long)min(c0 + d, chunks - 1) * REC, lane);
    }
    lds_barrier();
    for (int cc = c0; cc < c1; cc += DEEP) {
#pragma unroll
        for (int d = 0; d < DEEP; d++) {
            const int c = cc + d, buf = d & 1;   // DEEP is even
            // A round's chunks past the end are fetched and not computed: a way out of the loop from
            // here has every load awaited at its head (64 x 32768 x 8192, groups of 64: 83 us, so 66).
            // Groups of 32 do leave it: without, they need more registers than there are.
            if (G == 32 && c >= c1) break;
            put(raw[(d + 1) % DEEP], buf ^ 1);   // chunk c + 1
            fetch(raw[(d + 1) % DEEP], c + 1 + DEEP);
            if (G == 32 || c < c1) {
#pragma unroll
                for (int g = 0; g < GPC; g++) {
                    u32x4 x[MT][IPG];
                    float X[MT];
#pragma unroll
                    for (int m = 0; m < MT; m++) {
                        X[m] = sums[buf][g][m * 16 + col];
#pragma unroll
                        for (int i = 0; i < IPG; i++) x[m][i] = stage[buf][(m * 16 + col) * 16 + ((4 * (g * IPG + i) + qt) ^ col)];
                    }
#pragma unroll
                    for (int t = 0; t < NT; t++) {
                        f32x4 P[MT];
#pragma unroll
                        for (int i = 0; i < IPG; i++) {
                            const u32x4 A = codes8<F16>(w[d].w[t][g * IPG + i], cb);
#pragma unroll
                            for (int m = 0; m < MT; m++) P[m] = mfma<F16>(A, x[m][i], i ? P[m] : zero);
                        }
#pragma unroll
                        for (int r = 0; r < 4; r++) {
                            const float s = to_float<F16>((uint16_t)w[d].meta[t][g][r]), z = to_float<F16>((uint16_t)(w[d].meta[t][g][r] >> 16));
#pragma unroll
                            for (int m = 0; m < MT; m++) acc[m][t][r] = fmaf(s, fmaf(-z, X[m], P[m][r]), acc[m][t][r]);
                        }
                    }
                }
            }
            w[d].load(wp, (long long)min(c + DEEP, chunks - 1) * REC, lane);
            lds_barrier();
        }
    }
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int n = (tile0 + t) * kW4Tile + qt * 4;
        if (n >= a.n_out) continue;
#pragma unroll
        for (int mt = 0; mt < MT; mt++) {
            const int m = m0 + mt * 16 + col;
            if (m >= a.rows) continue;
            if (splits == 1) store4<F16>(a, m, n, acc[mt][t]);
            else *(f32x4 *)(part + ((long long)blockIdx.y * a.rows + m) * (n_tiles * kW4Tile) + n) = acc[mt][t];
        }
    }
}

// Adds the parts up, in order (bytes: 17 MB for 64 x 32768 in 2 parts, 4.5 us).
template <bool F16>
__global__ __launch_bounds__(256) void w4_join_kernel(W4Args a, int splits, const float *part)
{
    const int quads = (a.n_out + 3) / 4;
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    if (e >= (long long)quads * a.rows) return;
    const int m = (int)(e / quads), n = (int)(e % quads) * 4;
    const long long row = (long long)((a.n_out + kW4Tile - 1) / kW4Tile) * kW4Tile;
    f32x4 sum = *(const f32x4 *)(part + m * row + n);
    for (int p = 1; p < splits; p++) sum += *(const f32x4 *)(part + ((long long)p * a.rows + m) * row + n);
    store4<F16>(a, m, n, sum);
}

template <bool F16, int G, int MT, int NT, int NW>
hipError_t go_few(const W4Args &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW4Tile - 1) / kW4Tile);
    hipLaunchKernelGGL((w4_kernel<F16, G, MT, NT, NW>), dim3((tiles + NT - 1) / NT), dim3(NW * 64), 0, s, a);
    return hipGetLastError();
}

template <bool F16, int G, int MT, int NT, int NW, int DEEP>
hipError_t go_rows(const W4Args &a, const W4Plan &p, float *part, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW4Tile - 1) / kW4Tile), per = NW * NT;
    hipLaunchKernelGGL((w4_rows_kernel<F16, G, MT, NT, NW, DEEP>), dim3((tiles + per - 1) / per, p.splits, (a.rows + MT * 16 - 1) / (MT * 16)),
                       dim3(NW * 64), 0, s, a, p.splits, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const long long quads = (long long)((a.n_out + 3) / 4) * a.rows;
    hipLaunchKernelGGL((w4_join_kernel<F16>), dim3((unsigned)((quads + 255) / 256)), dim3(256), 0, s, a, p.splits, part);
    return hipGetLastError();
}

template <bool F16, int G>
hipError_t pick(const W4Args &a, const W4Plan &p, float *part, hipStream_t s)
{
    // what the registers of two waves a SIMD hold
    constexpr int DEEP = 4, DEEP2 = G == 128 ? 4 : 2;
    switch (p.form) {
        case kW4One16: return go_few<F16, G, 1, 1, 16>(a, s);
        case kW4One8: return go_few<F16, G, 1, 1, 8>(a, s);
        case kW4Four4: return go_few<F16, G, 1, 4, 4>(a, s);
        case kW4Two8: return go_few<F16, G, 2, 1, 8>(a, s);
        case kW4Rows32: return go_rows<F16, G, 2, 1, 8, DEEP>(a, p, part, s);
        case kW4Rows64: return go_rows<F16, G, 4, 1, 8, DEEP>(a, p, part, s);
        case kW4Rows64x2: return go_rows<F16, G, 4, 2, 8, DEEP2>(a, p, part, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_w4_pack(const W4PackArgs &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW4Tile - 1) / kW4Tile), chunks = (unsigned)((a.n_in + kW4Chunk - 1) / kW4Chunk);
    hipLaunchKernelGGL(w4_pack_kernel, dim3((chunks + 3) / 4, tiles < 16384 ? tiles : 16384), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Forms, with both sides measured (us, bfloat16, outputs x inputs):
// * up to 16 rows the waves of a workgroup share one tile of outputs (8 waves; 1 x
//   4096 x 4096: 3.9, 16 waves 4.2; but 16 where few tiles have many inputs: 16 x 4096 x
//   16384: 15.0, 8 waves 16.6).  Past 4 rows and 1024 tiles it is the rows, read again for
//   every tile, that count: four tiles (16 x 28672 x 4096: 15.5, one 21.9).
// * up to 32 rows of small layers the same with two tiles of rows (groups of 64, this way
//   and by rows, up to the limit: 32 x 1024 x 4096: 6.4, 9.6; 32 x 4096 x 4096: 7.2, 11.1;
//   past it: 32 x 4096 x 8192: 11.1, 13.7; 32 x 8192 x 4096: 12.2, 12.5; 32 x 2048 x 16384:
//   17.4, 15.8; 32 x 8192 x 8192: 21.9, 16.6).
// * otherwise by rows, two tiles of outputs a wave where that leaves workgroups enough (64 x
//   32768 x 8192: 57, one 66; 512 x 8192 x 8192: 84, one 108; 64 x 4096 x 4096: 16, two 20), the inputs in as many parts as give every
//   compute unit a workgroup (32 x 8192 x 8192 in 4: 18, whole 40).
W4Plan w4_plan(int rows, int n_out, int n_in)
{
    W4Plan p;
    p.splits = 1;
    p.ws_bytes = 0;
    const long long tiles = (n_out + kW4Tile - 1) / kW4Tile, chunks = (n_in + kW4Chunk - 1) / kW4Chunk;
    if (rows <= 16) {
        p.form = rows > 4 && tiles >= 1024 ? kW4Four4 : tiles <= 256 && chunks > 64 ? kW4One16 : kW4One8;
    } else if (rows <= 32 && tiles * chunks <= 256 * 32) {
        p.form = kW4Two8;
    } else {
        p.form = rows <= 32 ? kW4Rows32 : tiles * ((rows + 63) / 64) >= 1024 ? kW4Rows64x2 : kW4Rows64;
        const long long per = p.form == kW4Rows64x2 ? 16 : 8, groups = (tiles + per - 1) / per * ((rows + 63) / 64);
        long long k = (256 + groups - 1) / groups;
        if (k > chunks / 4) k = chunks / 4;
        p.splits = k < 1 ? 1 : (int)k;
        if (p.splits > 1) p.ws_bytes = (size_t)p.splits * rows * tiles * kW4Tile * sizeof(float);
    }
    return p;
}

hipError_t launch_w4(const W4Args &a, const W4Plan &p, int group, bool f16, float *part, hipStream_t s)
{
    if (f16) return group == 32 ? pick<true, 32>(a, p, part, s) : group == 64 ? pick<true, 64>(a, p, part, s) : pick<true, 128>(a, p, part, s);
    return group == 32 ? pick<false, 32>(a, p, part, s) : group == 64 ? pick<false, 64>(a, p, part, s) : pick<false, 128>(a, p, part, s);
}

}  // namespace mfs
