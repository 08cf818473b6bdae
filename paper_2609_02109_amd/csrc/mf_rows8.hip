// Rows of activations in 8 bits: the norm (with the residual's addition), the
// gate, or the row as it is, each with the row's largest value and its codes in
// the same pass; and what codes stand for.
//
// A row belongs to T threads, which hold it in registers as fp32 (8 V values each)
// between the sum of squares, the largest value and the codes: what comes from
// memory comes once.  Bound by the bytes from some hundred rows on (8192 rows of
// 8192, norm with a residual: 87 us for 470 MB, 5.4 TB/s; 4500 of 10240, gate:
// 42 to 44 us for 230 MB, 5.2 to 5.5 TB/s, and 37 where the 256 MB cache has them from the call before; what
// they stand for, 8192 of 8192: 36 us for 201 MB), below that by the trip to memory and the waves' meetings (one row of
// 4096: 2.9 us).
#include "mf_serve_dev.h"

namespace mfs {
namespace {

// Elements k .. k + 7 of a row of n, zeros past it.
__device__ __forceinline__ u32x4 load8(const uint16_t *x, int k, int n)
{
    if (k + 8 <= n) return load16(x + k);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 7; j++)   // with indexes that are known: else the array is in memory
        if (k + j < n) w[j >> 1] |= (uint32_t)x[k + j] << (16 * (j & 1));
    return (u32x4){w[0], w[1], w[2], w[3]};
}
__device__ __forceinline__ void store8(uint16_t *y, int k, int n, u32x4 v)
{
    if (k + 8 <= n) {
        __builtin_memcpy(__builtin_assume_aligned(y + k, 2), &v, 16);
        return;
    }
#pragma unroll
    for (int j = 0; j < 7; j++)
        if (k + j < n) y[k + j] = (uint16_t)(v[j >> 1] >> (16 * (j & 1)));
}
template <bool F16>
__device__ __forceinline__ void widen8(u32x4 raw, float *v)
{
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = to_float<F16>((uint16_t)(raw[j >> 1] >> (16 * (j & 1))));
}

// g sigmoid(g) u, within (4 + 1.3 |g|) 2^-24 of itself: far below half a code.  Below -88 the quotient's end is reached, 0.
__device__ __forceinline__ float gated(float g, float u)
{
    return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f)) * u;
}

// Over the T threads of a row, through LDS where they are more than a wave.
template <int T, class X, class F>
__device__ __forceinline__ X over_row(X v, X (&lds)[T / 64], const F &f)
{
    v = over_wave(v, f);
    if constexpr (T > 64) {
        if ((threadIdx.x & 63) == 0) lds[wave_id()] = v;
        lds_barrier();
        v = lds[0];
#pragma unroll
        for (int w = 1; w < T / 64; w++) v = f(v, lds[w]);
    }
    return v;
}

// Eight codes of a row from k on.
__device__ __forceinline__ void put_codes(int8_t *out, int k, int n, const Row8 &r, const float *v)
{
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 8; j++) c[j >> 2] |= code8(r, v[j]) << (8 * (j & 3));
    if (k + 8 <= n) {
        __builtin_memcpy(out + k, c, 8);
        return;
    }
#pragma unroll
    for (int j = 0; j < 7; j++)
        if (k + j < n) out[k + j] = (int8_t)(c[j >> 2] >> (8 * (j & 3)));
}
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float add(float p, float q) { return p + q; }
__device__ __forceinline__ uint32_t larger(uint32_t p, uint32_t q) { return max(p, q); }

// Eight elements of y before the norm's factors, in fp32: x, the sum of x and the residual (stored on the way), or the gate.
template <bool F16, int OP>
__device__ __forceinline__ void begin8(const Rows8Args &a, long long row, int k, u32x4 x, u32x4 y, float *v)
{
    widen8<F16>(x, v);
    if (OP == kRowsPlain || (OP == kRowsNorm && !a.y)) return;
    float u[8];
    widen8<F16>(y, u);
    if (OP == kRowsGate) {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = gated(v[j], u[j]);
        return;
    }
    u32x4 h;
#pragma unroll
    for (int j = 0; j < 4; j++) h[j] = pack2<F16>(v[2 * j] + u[2 * j], v[2 * j + 1] + u[2 * j + 1]);
    store8((uint16_t *)a.sum + row * a.sum_stride, k, a.n, h);
    widen8<F16>(h, v);   // what is carried on is what is normed
}
template <bool F16>
__device__ __forceinline__ void weigh8(u32x4 weight, float r, float *v)
{
    float w[8];
    widen8<F16>(weight, w);
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] = v[j] * r * w[j];
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
        u32x4 raw[V], with[V], weight[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int k = 8 * (t + i * T);
            raw[i] = with[i] = weight[i] = (u32x4){0, 0, 0, 0};
            if (k >= n) continue;
            raw[i] = load8(x, k, n);
            if (OP == kRowsGate || (OP == kRowsNorm && a.y)) with[i] = load8(y, k, n);
        }
        if (OP == kRowsNorm) {
#pragma unroll
            for (int i = 0; i < V; i++)
                if (8 * (t + i * T) < n) weight[i] = load8((const uint16_t *)a.weight, 8 * (t + i * T), n);
        }
        float sum = 0.f;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; i++) {
            const int k = 8 * (t + i * T);
#pragma unroll
            for (int j = 0; j < 8; j++) v[i][j] = 0.f;
            if (k < n) begin8<F16, OP>(a, row, k, raw[i], with[i], v[i]);
            if (OP == kRowsNorm) {
#pragma unroll
                for (int j = 0; j < 8; j++) sum += v[i][j] * v[i][j];
            }
        }
        if (OP == kRowsNorm) {
            sum = over_row<T>(sum, sums, add);
            const float r = 1.f / sqrtf(sum / (float)n + a.eps);
#pragma unroll
            for (int i = 0; i < V; i++)
                if (8 * (t + i * T) < n) weigh8<F16>(weight[i], r, v[i]);
            if (!(sum < INFINITY)) top = 0x7fffffffu;
        }
#pragma unroll
        for (int i = 0; i < V; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) top = max(top, magnitude(v[i][j]));
        const Row8 r = row8_of(over_row<T>(top, tops, larger));
        if (t == 0) a.scales[row] = r.scale;
        int8_t *out = a.codes + row * a.codes_stride;
#pragma unroll
        for (int i = 0; i < V; i++)
            if (8 * (t + i * T) < n) put_codes(out, 8 * (t + i * T), n, r, v[i]);
        if (T > 64 && row + gridDim.x < a.rows) lds_barrier();   // the next row's largest value goes where this one's is read
    }
}

// Rows that registers do not hold: three passes over them (two without a norm), the later ones over what the caches have.
template <bool F16, int OP>
__global__ __launch_bounds__(1024) void rows8_wide_kernel(Rows8Args a)
{
    constexpr int T = 1024;
    __shared__ float sums[T / 64];
    __shared__ uint32_t tops[T / 64];
    const int n = a.n;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const uint16_t *x = (const uint16_t *)a.x + row * a.x_stride, *y = (const uint16_t *)a.y + row * a.y_stride;
        const uint16_t *h = OP == kRowsNorm && a.y ? (const uint16_t *)a.sum + row * a.sum_stride : x;
        const u32x4 none = {0, 0, 0, 0};
        float sum = 0.f, r = 1.f;
        if (OP == kRowsNorm) {
            for (int k = 8 * (int)threadIdx.x; k < n; k += 8 * T) {
                float v[8];
                begin8<F16, OP>(a, row, k, load8(x, k, n), a.y ? load8(y, k, n) : none, v);
#pragma unroll
                for (int j = 0; j < 8; j++) sum += v[j] * v[j];
            }
            sum = over_row<T>(sum, sums, add);
            r = 1.f / sqrtf(sum / (float)n + a.eps);
        }
        // what a thread has stored of h is its own to read
        const auto get = [&](int k, float *v) {
            if (OP == kRowsNorm) {
                widen8<F16>(load8(h, k, n), v);
                weigh8<F16>(load8((const uint16_t *)a.weight, k, n), r, v);
            } else {
                begin8<F16, OP>(a, row, k, load8(x, k, n), OP == kRowsGate ? load8(y, k, n) : none, v);
            }
        };
        uint32_t top = !(sum < INFINITY) ? 0x7fffffffu : 0u;
        for (int k = 8 * (int)threadIdx.x; k < n; k += 8 * T) {
            float v[8];
            get(k, v);
#pragma unroll
            for (int j = 0; j < 8; j++) top = max(top, magnitude(v[j]));
        }
        const Row8 q = row8_of(over_row<T>(top, tops, larger));
        if (threadIdx.x == 0) a.scales[row] = q.scale;
        for (int k = 8 * (int)threadIdx.x; k < n; k += 8 * T) {
            float v[8];
            get(k, v);
            put_codes(a.codes + row * a.codes_stride, k, n, q, v);
        }
        if (row + gridDim.x < a.rows) lds_barrier();   // as above
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
#pragma unroll
            for (int j = 0; j < 7; j++)
                if (j < many) q[j] = c[j];
        const long long at = row * a.out_stride + k;
        if constexpr (TY == MF_F32) {
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (j < many) ((float *)a.out)[at + j] = (float)q[j] * s;
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

// As many threads to a row as leave each one or two pieces of eight, whether rows are few or many (us, norm with a residual and
// gate, the same rows again, of which the caches have a part; T threads of V pieces): 1 x 4096: 512 of one 2.9 and 2.5, 256 of two
// 3.4 and 2.9; 8192 x 4096: 36.5 and 26.2, 38.3 and 26.5; 8192 x 8192: 512 of two 85 and 61, 256 of four 94 and 62, 1024 of one 86
// and 63; 4500 x 10240: 1024 of two 82 and 37, 256 of eight 116 and 47.  Short rows: 8192 x 1024: 64 of two 12.1 and 9.1, 256 of one
// 13.6 and 11.4; 1 x 1024: 3.0, 2.5.
// Wider ones, which go over their rows two and three times, from memory: 1 x 28672: 7.7 and 8.2; 512 x 28672: 29 and 21 for 103 and 73 MB;
// 4096 x 28672: 182 and 152 for 822 and 587 MB, 4.5 and 3.9 TB/s; 512 x 131072: 132 and 110.
template <bool F16, int OP>
hipError_t pick(const Rows8Args &a, hipStream_t s)
{
    if (a.n <= 512) return go<F16, OP, 64, 1>(a, s);
    if (a.n <= 1024) return go<F16, OP, 64, 2>(a, s);
    if (a.n <= 2048) return go<F16, OP, 256, 1>(a, s);
    if (a.n <= 4096) return go<F16, OP, 512, 1>(a, s);
    if (a.n <= 8192) return go<F16, OP, 512, 2>(a, s);
    if (a.n <= 16384) return go<F16, OP, 1024, 2>(a, s);
    const long long most = most_workgroups(1024);
    hipLaunchKernelGGL((rows8_wide_kernel<F16, OP>), dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(1024), 0, s, a);
    return hipGetLastError();
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
