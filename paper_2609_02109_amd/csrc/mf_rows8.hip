// Rows of activations in 8 bits: the norm (with the residual's addition), the
// gate, or the row as it is, each with the row's largest value and its codes in
// the same pass; and what codes stand for.
//
// A row belongs to T threads, which hold it in registers as fp32 (8 V values each)
// between the sum of squares, the largest value and the codes: what comes from
// memory comes once.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

// Elements k .. k + 7 of a row of n, zeros past it.
__device__ __forceinline__ u32x4 load8(const uint16_t *x, int k, int n)
{
    if (k + 8 <= n) return load16(x + k);
    uint32_t w[4] = {0, 0, 0, 0};
    for (int j = 0; k + j < n; j++) w[j >> 1] |= (uint32_t)x[k + j] << (16 * (j & 1));
    return (u32x4){w[0], w[1], w[2], w[3]};
}
__device__ __forceinline__ void store8(uint16_t *y, int k, int n, u32x4 v)
{
    if (k + 8 <= n) {
        __builtin_memcpy(__builtin_assume_aligned(y + k, 2), &v, 16);
        return;
    }
    for (int j = 0; k + j < n; j++) y[k + j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
}
template <bool F16>
__device__ __forceinline__ void widen8(u32x4 raw, float *v)
{
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = to_float<F16>((uint16_t)(raw[j >> 1] >> (16 * (j & 1))));
}

// g sigmoid(g) u, within (4 + |g|) 2^-24 of itself: far below half a code.  Below -88 the quotient's end is reached, 0.
__device__ __forceinline__ float gated(float g, float u)
{
    return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * u;
}

// Over the T threads of a row, through LDS where they are more than a wave.
template <int T, class X, class F>
__device__ __forceinline__ X over_row(X v, X (&lds)[T / 64], const F &f)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = f(v, (X)__shfl_xor(v, d));
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) lds[wave_id()] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < T / 64; w++) v = f(v, lds[w]);
    }
    return v;
}

template <bool F16, int OP, int T, int V>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rows8_kernel(Rows8Args a)
{
    constexpr int PER = T < 256 ? 256 / T : 1;   // rows of a workgroup
    __shared__ float sums[T / 64];
    __shared__ uint32_t tops[T / 64];
    const int t = (int)threadIdx.x % T, n = a.n;
    for (long long row = (long long)blockIdx.x * PER + (int)threadIdx.x / T; row < a.rows; row += (long long)gridDim.x * PER) {
        const uint16_t *x = (const uint16_t *)a.x + row * a.x_stride, *y = (const uint16_t *)a.y + row * a.y_stride;
        float v[V][8];
        u32x4 raw[V], with[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int k = 8 * (t + i * T);
            raw[i] = with[i] = (u32x4){0, 0, 0, 0};
            if (k >= n) continue;
            raw[i] = load8(x, k, n);
            if (OP == kRowsGate || (OP == kRowsNorm && a.y)) with[i] = load8(y, k, n);
        }
        float sum = 0.f;
        uint32_t top = 0;   // the largest magnitude's bits: infinities and NaN are above all others
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int k = 8 * (t + i * T);
            widen8<F16>(raw[i], v[i]);
            float u[8];
            if (OP == kRowsGate || OP == kRowsNorm) widen8<F16>(with[i], u);
            if (OP == kRowsGate) {
#pragma unroll
                for (int j = 0; j < 8; j++) v[i][j] = gated(v[i][j], u[j]);
            }
            if (OP == kRowsNorm) {
                if (a.y) {
                    u32x4 h;
#pragma unroll
                    for (int j = 0; j < 4; j++) h[j] = pack2<F16>(v[i][2 * j] + u[2 * j], v[i][2 * j + 1] + u[2 * j + 1]);
                    if (k < n) store8((uint16_t *)a.sum + row * a.sum_stride, k, n, h);
                    widen8<F16>(h, v[i]);   // what is carried on is what is normed
                }
#pragma unroll
                for (int j = 0; j < 8; j++) sum += v[i][j] * v[i][j];
            }
        }
        if (OP == kRowsNorm) {
            sum = over_row<T>(sum, sums, [](float p, float q) { return p + q; });
            const float r = 1.f / sqrtf(sum / (float)n + a.eps);
#pragma unroll
            for (int i = 0; i < V; i++) {
                const int k = 8 * (t + i * T);
                if (k >= n) continue;
                float w[8];
                widen8<F16>(load8((const uint16_t *)a.weight, k, n), w);
#pragma unroll
                for (int j = 0; j < 8; j++) v[i][j] = v[i][j] * r * w[j];
            }
            if (!(sum < INFINITY)) top = 0x7fffffffu;
        }
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) top = max(top, __float_as_uint(v[i][j]) & 0x7fffffffu);
        top = over_row<T>(top, tops, [](uint32_t p, uint32_t q) { return max(p, q); });
        const bool bad = top >= 0x7f800000u;
        float scale = __uint_as_float(top) * (float)(1.0 / 127.0);
        if (scale < 0x1p-126f) scale = 0.f;   // below it 1 / scale may leave fp32
        const float inv = scale > 0.f && !bad ? 1.f / scale : 0.f;
        if (t == 0) a.scales[row] = bad ? NAN : scale;
        int8_t *out = a.codes + row * a.codes_stride;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int k = 8 * (t + i * T);
            if (k >= n) continue;
            uint32_t c[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const int q = bad ? 0 : (int)fminf(fmaxf(rintf(v[i][j] * inv), -127.f), 127.f);
                c[j >> 2] |= (uint32_t)(q & 255) << (8 * (j & 3));
            }
            if (k + 8 <= n) {
                __builtin_memcpy(out + k, c, 8);
            } else {
                for (int j = 0; k + j < n; j++) out[k + j] = (int8_t)(c[j >> 2] >> (8 * (j & 3)));
            }
        }
    }
}

// 8 values a thread.
template <int TY>
__global__ __launch_bounds__(256) void values8_kernel(Values8Args a)
{
    const int pieces = (a.n + 7) / 8;
    const long long all = a.rows * pieces;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < all; e += (long long)gridDim.x * 256) {
        const long long row = e / pieces;
        const int k = (int)(e - row * pieces) * 8, many = min(8, a.n - k);
        const int8_t *c = a.codes + row * a.codes_stride + k;
        const float s = a.scales[row];
        int8_t q[8] = {};
        if (many == 8) __builtin_memcpy(q, c, 8);
        else
            for (int j = 0; j < many; j++) q[j] = c[j];
        const long long at = row * a.out_stride + k;
        if constexpr (TY == MF_F32) {
            for (int j = 0; j < many; j++) ((float *)a.out)[at + j] = (float)q[j] * s;
        } else {
            u32x4 o;
#pragma unroll
            for (int j = 0; j < 4; j++) o[j] = pack2<TY == MF_F16>((float)q[2 * j] * s, (float)q[2 * j + 1] * s);
            store8((uint16_t *)a.out + at, 0, many, o);
        }
    }
}

template <bool F16, int OP, int T, int V>
hipError_t go(const Rows8Args &a, hipStream_t s)
{
    constexpr int PER = T < 256 ? 256 / T : 1, THREADS = T < 256 ? 256 : T;
    const long long groups = (a.rows + PER - 1) / PER, most = most_workgroups(THREADS);
    hipLaunchKernelGGL((rows8_kernel<F16, OP, T, V>), dim3((unsigned)(groups < most ? groups : most)), dim3(THREADS), 0, s, a);
    return hipGetLastError();
}

template <bool F16, int OP>
hipError_t pick(const Rows8Args &a, hipStream_t s)
{
    if (a.n <= 512) return go<F16, OP, 64, 1>(a, s);
    if (a.n <= 1024) return go<F16, OP, 64, 2>(a, s);
    if (a.n <= 2048) return go<F16, OP, 256, 1>(a, s);
    if (a.n <= 4096) return go<F16, OP, 256, 2>(a, s);
    if (a.n <= 8192) return go<F16, OP, 256, 4>(a, s);
    if (a.n <= 16384) return go<F16, OP, 256, 8>(a, s);
    if (a.n <= 65536) return go<F16, OP, 1024, 8>(a, s);
    return go<F16, OP, 1024, 16>(a, s);
}

}  // namespace

hipError_t launch_rows8(const Rows8Args &a, Rows8Op op, bool f16, hipStream_t s)
{
    if (op == kRowsNorm) return f16 ? pick<true, kRowsNorm>(a, s) : pick<false, kRowsNorm>(a, s);
    if (op == kRowsGate) return f16 ? pick<true, kRowsGate>(a, s) : pick<false, kRowsGate>(a, s);
    return f16 ? pick<true, kRowsPlain>(a, s) : pick<false, kRowsPlain>(a, s);
}

hipError_t launch_values8(const Values8Args &a, int dtype, hipStream_t s)
{
    const long long groups = (a.rows * ((a.n + 7) / 8) + 255) / 256, most = most_workgroups(256);
    const dim3 grid((unsigned)(groups < most ? groups : most));
    if (dtype == MF_F32) hipLaunchKernelGGL((values8_kernel<MF_F32>), grid, dim3(256), 0, s, a);
    else if (dtype == MF_BF16) hipLaunchKernelGGL((values8_kernel<MF_BF16>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((values8_kernel<MF_F16>), grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace mfs
