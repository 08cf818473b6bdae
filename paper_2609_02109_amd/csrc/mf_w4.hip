// Products with 4-bit weights and group scales: y = x W^T + bias,
// W[n][k] = s (c - z).  With P = sum_k (16 + c) x and X = sum_k x over a group,
// both from matrix instructions, the group's part is s (P - (16 + z) X): the
// codes go into the instruction as they are, and scale and zero point cost two
// fp32 operations a group and output instead of one a weight.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

// One thread per dword of a record: code dwords first, then scales.
__global__ void w4_pack_kernel(W4PackArgs a)
{
    const int chunks = (a.n_in + kW4Chunk - 1) / kW4Chunk, rec = w4_record(a.group), gpc = kW4Chunk / a.group;
    const uint8_t *codes = a.codes;
    const long long row_bytes = a.n_in / 2, groups = a.n_in / a.group;
    for (long long t = blockIdx.x; t < (long long)((a.n_out + kW4Tile - 1) / kW4Tile) * chunks; t += gridDim.x) {
        const int tile = (int)(t / chunks), chunk = (int)(t % chunks);
        uint32_t *out = (uint32_t *)(a.packed + t * rec);
        for (int e = (int)threadIdx.x; e < rec / 4; e += (int)blockDim.x) {
            uint32_t w = 0;
            if (e < kW4Codes / 4) {
                const int lane = e >> 2, i = e & 3;
                const int n = tile * kW4Tile + (lane & 15), k = chunk * kW4Chunk + i * 32 + (lane >> 4) * 8;
                if (n < a.n_out && k < a.n_in) {
                    const uint8_t *src = codes + (long long)n * row_bytes + k / 2;
                    for (int j = 0; j < 4; j++) w |= (uint32_t)(src[j] & 15) << (4 * j) | (uint32_t)(src[j] >> 4) << (16 + 4 * j);
                }
            } else {
                const int m = e - kW4Codes / 4;
                const int n = tile * kW4Tile + (m & 15), g = chunk * gpc + (m >> 4);
                if (n < a.n_out && g < groups) {
                    const long long at = (long long)n * groups + g;
                    const float z = 16.f + (float)(a.zeros ? a.zeros[at] & 15 : 8);
                    w = a.scales[at] | (uint32_t)(a.f16 ? from_float<true>(z) : from_float<false>(z)) << 16;
                }
            }
            out[e] = w;
        }
    }
}

// A workgroup takes NT tiles of 16 outputs and MT tiles of 16 rows; its NW waves
// take every NW-th chunk of 128 inputs and add up through LDS at the end, in
// wave order.
template <bool F16, int G, int MT, int NT, int NW>
__global__ __launch_bounds__(NW * 64) void w4_kernel(W4Args a)
{
    constexpr int GPC = kW4Chunk / G, IPG = G / 32, REC = w4_record(G);
    __shared__ f32x4 red[NW][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW4Tile - 1) / kW4Tile, chunks = (a.n_in + kW4Chunk - 1) / kW4Chunk;
    const int tile0 = (int)blockIdx.x * NT, m0 = (int)blockIdx.y * MT * 16;
    const uint8_t *wp[NT];
    for (int t = 0; t < NT; t++) {
        const int tile = tile0 + t < n_tiles ? tile0 + t : n_tiles - 1;   // past the end: computed again, not stored
        wp[t] = a.packed + (long long)tile * chunks * REC;
    }
    const uint16_t *xp[MT];
    for (int t = 0; t < MT; t++) {
        const int m = m0 + t * 16 + col;
        xp[t] = (const uint16_t *)a.x + (long long)(m < a.rows ? m : a.rows - 1) * a.x_stride + qt * 8;
    }
    const CodeBits cb = code_bits<F16>();
    f32x4 acc[MT][NT] = {};
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    for (int c = wave; c < chunks; c += NW) {
        u32x4 w[NT], meta[NT][GPC], x[MT][4];
#pragma unroll
        for (int t = 0; t < NT; t++) {
            const uint8_t *r = wp[t] + (long long)c * REC;
            w[t] = *(const u32x4 *)(r + lane * 16);
#pragma unroll
            for (int g = 0; g < GPC; g++) meta[t][g] = *(const u32x4 *)(r + kW4Codes + g * 64 + qt * 16);
        }
#pragma unroll
        for (int t = 0; t < MT; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int k = c * kW4Chunk + i * 32;
                x[t][i] = (u32x4){0, 0, 0, 0};
                if (k < a.n_in) x[t][i] = load16(xp[t] + k);
            }
#pragma unroll
        for (int g = 0; g < GPC; g++) {
            f32x4 X[MT];
#pragma unroll
            for (int m = 0; m < MT; m++) {
                X[m] = zero;
#pragma unroll
                for (int i = 0; i < IPG; i++) X[m] = mfma<F16>(ones8<F16>(), x[m][g * IPG + i], X[m]);
            }
#pragma unroll
            for (int t = 0; t < NT; t++) {
                f32x4 P[MT];
#pragma unroll
                for (int i = 0; i < IPG; i++) {
                    const u32x4 A = codes8<F16>(w[t][g * IPG + i], cb);
#pragma unroll
                    for (int m = 0; m < MT; m++) P[m] = mfma<F16>(A, x[m][g * IPG + i], i ? P[m] : zero);
                }
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    const float s = to_float<F16>((uint16_t)meta[t][g][r]), z = to_float<F16>((uint16_t)(meta[t][g][r] >> 16));
#pragma unroll
                    for (int m = 0; m < MT; m++) acc[m][t][r] = fmaf(s, fmaf(-z, X[m][r], P[m][r]), acc[m][t][r]);
                }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int t = 0; t < NT; t++) red[wave][m * NT + t][lane] = acc[m][t];
    __syncthreads();
    for (int e = (int)threadIdx.x; e < MT * NT * 64; e += NW * 64) {
        const int l = e & 63, mt = e >> 6, m = m0 + (mt / NT) * 16 + (l & 15);
        const int n = (tile0 + mt % NT) * kW4Tile + (l >> 4) * 4;
        f32x4 sum = red[0][mt][l];
#pragma unroll
        for (int v = 1; v < NW; v++) sum += red[v][mt][l];
        if (m >= a.rows || n >= a.n_out) continue;
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
}

template <bool F16, int G, int MT, int NT, int NW>
hipError_t go(const W4Args &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW4Tile - 1) / kW4Tile);
    // rows past 65535 blocks of 16 MT are launched in parts
    W4Args p = a;
    const int most = 65535 * MT * 16;
    for (int m = 0; m < a.rows; m += most) {
        p.rows = a.rows - m < most ? a.rows - m : most;
        p.x = (const uint16_t *)a.x + (long long)m * a.x_stride;
        p.y = (uint16_t *)a.y + (long long)m * a.y_stride;
        const dim3 grid((tiles + NT - 1) / NT, (unsigned)((p.rows + MT * 16 - 1) / (MT * 16)));
        hipLaunchKernelGGL((w4_kernel<F16, G, MT, NT, NW>), grid, dim3(NW * 64), 0, s, p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <bool F16, int G>
hipError_t pick(const W4Args &a, hipStream_t s)
{
    if (a.rows <= 16) return go<F16, G, 1, 1, 16>(a, s);
    if (a.rows <= 32) return go<F16, G, 2, 2, 8>(a, s);
    return go<F16, G, 4, 2, 8>(a, s);
}

}  // namespace

hipError_t launch_w4_pack(const W4PackArgs &a, hipStream_t s)
{
    const long long recs = (long long)((a.n_out + kW4Tile - 1) / kW4Tile) * ((a.n_in + kW4Chunk - 1) / kW4Chunk);
    const unsigned grid = (unsigned)(recs < 65536 ? recs : 65536);
    hipLaunchKernelGGL(w4_pack_kernel, dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_w4(const W4Args &a, int group, bool f16, hipStream_t s)
{
    if (f16) return group == 32 ? pick<true, 32>(a, s) : group == 64 ? pick<true, 64>(a, s) : pick<true, 128>(a, s);
    return group == 32 ? pick<false, 32>(a, s) : group == 64 ? pick<false, 64>(a, s) : pick<false, 128>(a, s);
}

}  // namespace mfs
