// Products of 8-bit rows with 8-bit weights: y[m][n] = (sum_k x[m][k] w[n][k])
// xs[m] ws[n] + bias[n].  The sum is a whole number, exact in the 32 bits that
// the matrix instructions add up in, so that no order of it makes a difference;
// the scales cost two multiplications an output.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes from any address.
__device__ __forceinline__ i32x4 load16b(const void *p)
{
    i32x4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// D += A B, 16 x 16 x 64: lane l holds A[l % 16][16 (l / 16) ..+16], B[16 (l / 16) ..+16][l % 16], D[4 (l / 16) + r][l % 16].
__device__ __forceinline__ i32x4 mfma8(i32x4 a, i32x4 b, i32x4 c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0); }

// Once a weight: a wave per record, 16 rows of 64 codes in, 1 KB in a row out.
__global__ __launch_bounds__(256) void w8_pack_kernel(W8PackArgs a)
{
    const int tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in);
    const int lane = threadIdx.x & 63, chunk = (int)blockIdx.x * 4 + wave_id();
    if (chunk == 0 && blockIdx.x == 0) {
        float *scales = (float *)(a.packed + (long long)tiles * chunks * kW8Record);
        for (long long n = (long long)blockIdx.y * 64 + lane; n < a.n_out; n += (long long)gridDim.y * 64) scales[n] = a.scales[n];
    }
    if (chunk >= chunks) return;
    for (int tile = (int)blockIdx.y; tile < tiles; tile += (int)gridDim.y) {
        const int n = tile * kW8Tile + (lane & 15), k = chunk * kW8Chunk + (lane >> 4) * 16;
        i32x4 w = {0, 0, 0, 0};
        if (n < a.n_out && k < a.n_in) w = load16b(a.codes + (long long)n * a.n_in + k);   // inputs are a multiple of 16
        ((i32x4 *)(a.packed + ((long long)tile * chunks + chunk) * kW8Record))[lane] = w;
    }
}

// Outputs n .. n + 3 of row m.
template <bool F16>
__device__ __forceinline__ void store4(const W8Args &a, int m, int n, i32x4 acc)
{
    const float xs = a.x_scales[m];
    const int many = min(4, a.n_out - n);
    uint16_t *y = (uint16_t *)a.y + (long long)m * a.y_stride + n;
    float v[4];
    for (int r = 0; r < 4; r++) {
        if (r >= many) break;
        v[r] = (float)acc[r] * xs * a.w_scales[n + r];
        if (a.bias) v[r] += to_float<F16>(((const uint16_t *)a.bias)[n + r]);
    }
    if (many == 4) {
        const u32x2 o = {pack2<F16>(v[0], v[1]), pack2<F16>(v[2], v[3])};
        __builtin_memcpy(__builtin_assume_aligned(y, 2), &o, 8);
    } else {
        for (int r = 0; r < many; r++) y[r] = from_float<F16>(v[r]);
    }
}

// Few rows (bound by the weights' bytes).  A workgroup takes NT tiles of 16 outputs and MT tiles of 16 rows; its NW
// waves take every NW-th chunk of 64 D inputs, the next one on its way while one is computed, and add up through LDS.
template <bool F16, int MT, int NT, int NW, int D>
__global__ __launch_bounds__(NW * 64) void w8_few_kernel(W8Args a)
{
    constexpr int SUMS = MT * NT * 64;
    __shared__ i32x4 lds[NW * SUMS];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in);
    const int tile0 = (int)blockIdx.x * NT, m0 = (int)blockIdx.y * MT * 16;
    const uint8_t *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int tile = min(tile0 + t, n_tiles - 1);   // past the end: computed again, not stored
        wp[t] = a.packed + (long long)tile * chunks * kW8Record + lane * 16;
    }
    const int8_t *xp[MT];
#pragma unroll
    for (int m = 0; m < MT; m++) xp[m] = a.x + (long long)min(m0 + 16 * m + col, a.rows - 1) * a.x_stride;
    i32x4 acc[MT][NT] = {}, w[NT][D], x[MT][D];
    // past the inputs: the last record's or the row's last codes, not used or times a weight of 0
    const auto load = [&](i32x4 (&w)[NT][D], i32x4 (&x)[MT][D], int c) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            const int at = min(c + d, chunks - 1);
#pragma unroll
            for (int t = 0; t < NT; t++) w[t][d] = *(const i32x4 *)(wp[t] + (long long)at * kW8Record);
#pragma unroll
            for (int m = 0; m < MT; m++) x[m][d] = load16b(xp[m] + min(at * kW8Chunk + qt * 16, a.n_in - 16));
        }
    };
    if (wave * D < chunks) load(w, x, wave * D);
    for (int c = wave * D; c < chunks; c += NW * D) {
        i32x4 wn[NT][D], xn[MT][D];
        load(wn, xn, c + NW * D);
#pragma unroll
        for (int d = 0; d < D; d++) {
            if (c + d >= chunks) break;
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int t = 0; t < NT; t++) acc[m][t] = mfma8(w[t][d], x[m][d], acc[m][t]);
        }
#pragma unroll
        for (int d = 0; d < D; d++) {
#pragma unroll
            for (int t = 0; t < NT; t++) w[t][d] = wn[t][d];
#pragma unroll
            for (int m = 0; m < MT; m++) x[m][d] = xn[m][d];
        }
    }
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int t = 0; t < NT; t++) lds[(wave * MT * NT + m * NT + t) * 64 + lane] = acc[m][t];
    __syncthreads();
    for (int e = (int)threadIdx.x; e < SUMS; e += NW * 64) {
        const int l = e & 63, mt = e >> 6, m = m0 + (mt / NT) * 16 + (l & 15), n = (tile0 + mt % NT) * kW8Tile + (l >> 4) * 4;
        i32x4 sum = lds[e];
#pragma unroll
        for (int v = 1; v < NW; v++) sum += lds[v * SUMS + e];
        if (m < a.rows && n < a.n_out) store4<F16>(a, m, n, sum);
    }
}

// Many rows: a workgroup of four waves takes 128 rows and 128 outputs, a wave 64 of each.  128 inputs of the rows go
// into LDS at a time while the ones before are computed; the weights come as operands from memory.
template <bool F16>
__global__ __launch_bounds__(256) void w8_tiles_kernel(W8Args a)
{
    // rows of eight 16-byte pieces, piece p of row r at p ^ (r % 8)
    __shared__ i32x4 stage[2][128 * 8];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in), steps = (chunks + 1) / 2;
    const int m0 = (int)blockIdx.y * 128, tile0 = (int)blockIdx.x * 8 + (wave >> 1) * 4, mw = (wave & 1) * 64;
    const uint8_t *wp[4];
#pragma unroll
    for (int t = 0; t < 4; t++) wp[t] = a.packed + (long long)min(tile0 + t, n_tiles - 1) * chunks * kW8Record + lane * 16;
    const int r0 = (int)threadIdx.x >> 3, piece = (int)threadIdx.x & 7;
    const int8_t *xp[4];
#pragma unroll
    for (int j = 0; j < 4; j++) xp[j] = a.x + (long long)min(m0 + r0 + 32 * j, a.rows - 1) * a.x_stride;
    i32x4 raw[4], w[2][4], acc[4][4] = {};
    const auto fetch = [&](int s) {
        const int k = min(s * 128 + piece * 16, a.n_in - 16);
#pragma unroll
        for (int j = 0; j < 4; j++) raw[j] = load16b(xp[j] + k);
    };
    const auto weights = [&](int s) {
#pragma unroll
        for (int d = 0; d < 2; d++)
#pragma unroll
            for (int t = 0; t < 4; t++) w[d][t] = *(const i32x4 *)(wp[t] + (long long)min(2 * s + d, chunks - 1) * kW8Record);
    };
    const auto put = [&](int buf) {
#pragma unroll
        for (int j = 0; j < 4; j++) stage[buf][(r0 + 32 * j) * 8 + (piece ^ (r0 & 7))] = raw[j];
    };
    fetch(0);
    put(0);
    __syncthreads();
    for (int s = 0; s < steps; s++) {
        weights(s);
        if (s + 1 < steps) fetch(s + 1);
#pragma unroll
        for (int d = 0; d < 2; d++) {
            if (2 * s + d >= chunks) break;
            i32x4 x[4];
#pragma unroll
            for (int m = 0; m < 4; m++) x[m] = stage[s & 1][(mw + 16 * m + col) * 8 + ((4 * d + qt) ^ (col & 7))];
#pragma unroll
            for (int m = 0; m < 4; m++)
#pragma unroll
                for (int t = 0; t < 4; t++) acc[m][t] = mfma8(w[d][t], x[m], acc[m][t]);
        }
        if (s + 1 < steps) put((s + 1) & 1);
        __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < 4; m++)
#pragma unroll
        for (int t = 0; t < 4; t++) {
            const int row = m0 + mw + 16 * m + col, n = (tile0 + t) * kW8Tile + qt * 4;
            if (row < a.rows && n < a.n_out) store4<F16>(a, row, n, acc[m][t]);
        }
}

template <bool F16, int MT, int NT, int NW, int D>
hipError_t go_few(const W8Args &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW8Tile - 1) / kW8Tile);
    hipLaunchKernelGGL((w8_few_kernel<F16, MT, NT, NW, D>), dim3((tiles + NT - 1) / NT, (a.rows + MT * 16 - 1) / (MT * 16)), dim3(NW * 64), 0, s, a);
    return hipGetLastError();
}

template <bool F16>
hipError_t pick(const W8Args &a, const W8Plan &p, hipStream_t s)
{
    switch (p.form) {
        case kW8Few1: return go_few<F16, 1, 1, 8, 2>(a, s);
        case kW8Few2: return go_few<F16, 2, 1, 8, 2>(a, s);
        case kW8Few4: return go_few<F16, 4, 1, 8, 2>(a, s);
        case kW8Tiles: break;
    }
    hipLaunchKernelGGL((w8_tiles_kernel<F16>), dim3((unsigned)((a.n_out + 127) / 128), (a.rows + 127) / 128), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_w8_pack(const W8PackArgs &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW8Tile - 1) / kW8Tile), chunks = (unsigned)w8_chunks(a.n_in);
    hipLaunchKernelGGL(w8_pack_kernel, dim3((chunks + 3) / 4, tiles < 16384 ? tiles : 16384), dim3(256), 0, s, a);
    return hipGetLastError();
}

W8Plan w8_plan(int rows, int n_out, int n_in)
{
    W8Plan p;
    p.ws_bytes = 0;
    p.form = rows <= 16 ? kW8Few1 : rows <= 32 ? kW8Few2 : rows <= 64 ? kW8Few4 : kW8Tiles;
    return p;
}

hipError_t launch_w8(const W8Args &a, const W8Plan &p, bool f16, void *, hipStream_t s) { return f16 ? pick<true>(a, p, s) : pick<false>(a, p, s); }

}  // namespace mfs
