// Products of 8-bit rows with 8-bit weights: y[m][n] = (sum_k x[m][k] w[n][k])
// xs[m] ws[n] + bias[n].  The sum is a whole number, exact in the 32 bits that
// the matrix instructions add up in, so that no order of it makes a difference;
// the scales cost two multiplications an output.
#include "mf_serve_dev.h"

namespace mfs {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Rows in 16 bits that a product for few rows puts into 8 itself, which every workgroup does, as far as their codes have room in
// LDS: up to four (4 x 4096 x 4096: 7.8 us; by a launch of their own about as much in a graph, and 3 us more to call); eight
// are slower (8 x 28672 x 4096: 28.4, by a launch of their own 25.4).
constexpr int kW8Rows16 = 4, kW8Lds = 32768;

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
        for (long long n = (long long)blockIdx.y * 64 + lane; n < (long long)tiles * kW8Tile; n += (long long)gridDim.y * 64) scales[n] = n < a.n_out ? a.scales[n] : 0.f;
    }
    if (chunk >= chunks) return;
    for (int tile = (int)blockIdx.y; tile < tiles; tile += (int)gridDim.y) {
        const int n = tile * kW8Tile + (lane & 15), k = chunk * kW8Chunk + (lane >> 4) * 16;
        i32x4 w = {0, 0, 0, 0};
        if (n < a.n_out && k < a.n_in) w = load16b(a.codes + (long long)n * a.n_in + k);   // inputs are a multiple of 16
        ((i32x4 *)(a.packed + ((long long)tile * chunks + chunk) * kW8Record))[lane] = w;
    }
}

// What outputs n .. n + 3 of row m are taken times and added to; fetched ahead of its use.
template <bool F16>
struct Ends {
    float xs;
    f32x4 ws;
    uint32_t bias[2];
    __device__ __forceinline__ void fetch(const W8Args &a, int m, int n)
    {
        bias[0] = bias[1] = 0;
        if (m >= a.rows || n >= a.n_out) return;
        if (a.x_scales) xs = a.x_scales[m];   // else the kernel knows
        fetch(a, n);
    }
    __device__ __forceinline__ void fetch(const W8Args &a, int n)
    {
        bias[0] = bias[1] = 0;
        if (n >= a.n_out) return;
        ws = *(const f32x4 *)(a.w_scales + n);   // whole tiles of scales
        if (!a.bias) return;
        const uint16_t *b = (const uint16_t *)a.bias + n;
        if (n + 4 <= a.n_out) __builtin_memcpy(bias, __builtin_assume_aligned(b, 2), 8);
        else
#pragma unroll
            for (int r = 0; r < 3; r++)   // with indexes that are known: else the array is in memory
                if (n + r < a.n_out) bias[r >> 1] |= (uint32_t)b[r] << (16 * (r & 1));
    }
    __device__ __forceinline__ u32x2 outputs(const W8Args &a, i32x4 acc) const
    {
        float v[4];
#pragma unroll
        for (int r = 0; r < 4; r++) {
            v[r] = (float)acc[r] * xs * ws[r];
            if (a.bias) v[r] += to_float<F16>((uint16_t)(bias[r >> 1] >> (16 * (r & 1))));
        }
        return (u32x2){pack2<F16>(v[0], v[1]), pack2<F16>(v[2], v[3])};
    }
    __device__ __forceinline__ void store(const W8Args &a, int m, int n, i32x4 acc) const
    {
        if (m >= a.rows || n >= a.n_out) return;
        uint16_t *y = (uint16_t *)a.y + (long long)m * a.y_stride + n;
        const u32x2 o = outputs(a, acc);
        if (n + 4 <= a.n_out) __builtin_memcpy(__builtin_assume_aligned(y, 2), &o, 8);
        else
#pragma unroll
            for (int r = 0; r < 3; r++)
                if (n + r < a.n_out) y[r] = (uint16_t)(o[r >> 1] >> (16 * (r & 1)));
    }
};

// Up to 1 << SH rows in 16 bits into 8, in LDS: as many of the NW waves to each, 4 values a thread and turn.
template <bool F16, int NW, int SH>
__device__ __forceinline__ void rows_to_8(const W8Args &a, i32x4 *codes, uint32_t *tops, float *scales)
{
    constexpr int WAVES = NW >> SH, PER = WAVES * 64, MOST = (kW8Lds >> SH) / 4 / PER;   // w8_takes_16
    const int lane = threadIdx.x & 63, wave = wave_id(), m = wave / WAVES, t = (int)threadIdx.x % PER;
    const bool row_here = m < a.rows;
    const uint16_t *row = (const uint16_t *)a.x16 + (long long)m * a.x_stride;
    uint32_t v[MOST][2], top = 0;
#pragma unroll
    for (int i = 0; i < MOST; i++) {
        const int k = 4 * (t + i * PER);
        v[i][0] = v[i][1] = 0;
        if (row_here && k < a.n_in) __builtin_memcpy(v[i], __builtin_assume_aligned(row + k, 2), 8);
    }
    const auto value = [&](int i, int j) { return to_float<F16>((uint16_t)(v[i][j >> 1] >> (16 * (j & 1)))); };
#pragma unroll
    for (int i = 0; i < MOST; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) top = max(top, __float_as_uint(value(i, j)) & 0x7fffffffu);
    top = over_wave(top, [](uint32_t p, uint32_t q) { return max(p, q); });
    if (lane == 0) tops[wave] = top;
    lds_barrier();
#pragma unroll
    for (int i = 0; i < WAVES; i++) top = max(top, tops[m * WAVES + i]);
    const Row8 r = row8_of(top);
    if (t == 0 && row_here) scales[m] = r.scale;
#pragma unroll
    for (int i = 0; i < MOST; i++) {
        const int k = 4 * (t + i * PER);
        uint32_t c = 0;
#pragma unroll
        for (int j = 0; j < 4; j++) c |= code8(r, value(i, j)) << (8 * j);
        if (row_here && k < a.n_in) ((uint32_t *)codes)[(m * a.n_in + k) / 4] = c;
    }
}

// Few rows (up to 16; bound by the weights' bytes, and below some 32 MB of them by two trips to memory and the sum through
// LDS).  A workgroup takes NT tiles of 16 outputs; its NW waves take every NW-th D chunks of 64 inputs, each chunk's place in
// the registers fetched again where it has been used, and add up through LDS.  1 x 4096 x 4096: 5.0 us for 16.8 MB, 3.4 TB/s;
// 16 x 28672 x 4096: 24.2 us for 117 MB, 4.9 TB/s.
// X16: rows that come in 16 bits, up to kW8Rows16, are put into 8 in LDS by every workgroup, with the
// first weights on their way (1 x 4096 x 4096: 6.0 us; a launch of its own takes 2.5 more than the 5.0, and its gap).
template <bool F16, int NT, int NW, int D, bool X16>
__global__ __launch_bounds__(NW * 64) void w8_few_kernel(W8Args a)
{
    constexpr int SUMS = NT * 64, Q = (NT + NW - 1) / NW;
    __shared__ i32x4 lds[NW * SUMS];
    __shared__ i32x4 codes[X16 ? kW8Lds / 16 : 1];   // rows of n_in
    __shared__ uint32_t tops[X16 ? NW : 1];
    __shared__ float scales[X16 ? kW8Rows16 : 1];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in);
    const int tile0 = (int)blockIdx.x * NT;
    const uint8_t *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int tile = min(tile0 + t, n_tiles - 1);   // past the end: computed again, not stored
        wp[t] = a.packed + (long long)tile * chunks * kW8Record + lane * 16;
    }
    const int8_t *xp = X16 ? nullptr : a.x + (long long)min(col, a.rows - 1) * a.x_stride;
    i32x4 acc[NT] = {}, w[NT][D], x[D];
    const auto load_x = [&](int c, int d) {
        if (c + d >= chunks) return;
        const int k = min((c + d) * kW8Chunk + qt * 16, a.n_in - 16);   // past the inputs: codes times weights of 0
        if (X16) x[d] = codes[(min(col, a.rows - 1) * a.n_in + k) / 16];
        else x[d] = load16b(xp + k);
    };
    const auto load = [&](int c, int d) {
        if (c + d >= chunks) return;
#pragma unroll
        for (int t = 0; t < NT; t++) w[t][d] = *(const i32x4 *)(wp[t] + (long long)(c + d) * kW8Record);
    };
#pragma unroll
    for (int d = 0; d < D; d++) {
        load(wave * D, d);
        if (!X16) load_x(wave * D, d);
    }
    // this thread's outputs
    Ends<F16> ends[Q];
    int em[Q], en[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int e = (int)threadIdx.x + q * NW * 64, l = e & 63, mt = e >> 6;
        em[q] = e < SUMS ? l & 15 : a.rows;
        en[q] = (tile0 + mt) * kW8Tile + (l >> 4) * 4;
        ends[q].fetch(a, em[q], en[q]);
    }
    if constexpr (X16) {
        if (a.rows == 1) rows_to_8<F16, NW, 0>(a, codes, tops, scales);
        else if (a.rows == 2) rows_to_8<F16, NW, 1>(a, codes, tops, scales);
        else rows_to_8<F16, NW, 2>(a, codes, tops, scales);
        lds_barrier();
#pragma unroll
        for (int d = 0; d < D; d++) load_x(wave * D, d);
    }
    for (int c = wave * D; c < chunks; c += NW * D) {
#pragma unroll
        for (int d = 0; d < D; d++) {
            if (c + d < chunks) {
#pragma unroll
                for (int t = 0; t < NT; t++) acc[t] = mfma8(w[t][d], x[d], acc[t]);
            }
            load(c + NW * D, d);
            load_x(c + NW * D, d);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; t++) lds[(wave * NT + t) * 64 + lane] = acc[t];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int e = (int)threadIdx.x + q * NW * 64;
        if (e >= SUMS) break;
        i32x4 sum = lds[e];
#pragma unroll
        for (int v = 1; v < NW; v++) sum += lds[v * SUMS + e];
        if (X16 && em[q] < a.rows) ends[q].xs = scales[em[q]];
        ends[q].store(a, em[q], en[q], sum);
    }
}

// Many rows: WM x WN waves, each with MT tiles of 16 rows and NT of 16 outputs.  The rows go through LDS, 128 inputs
// a step, in three buffers: a step reads one, the next one is whole, and the one after is being written, so that a wave's
// operands are read ahead over the barrier between steps.  The weights come as operands from memory, 64
// inputs fetched where those before them in the registers have been used.  Bound by the matrix instructions: 4096 x 8192 x
// 8192 in 217 us, 2.5 POP/s (a library's product of 8192^3: 2.1), which are busy 61 % of the cycles, vector
// instructions 25 %; a compute unit holds one workgroup (96 KB of LDS), which waits at a barrier a step.
template <bool F16, int MT, int NT, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64, WM * WN <= 4 ? 1 : 2) void w8_tiles_kernel(W8Args a)
{
    constexpr int BM = WM * MT * 16, BN = WN * NT, THREADS = WM * WN * 64, MINE = BM * 8 / THREADS, HALF = MT / 2;
    static_assert(MINE * THREADS == BM * 8 && MT % 2 == 0, "whole pieces a thread, two halves of rows");
    // rows of eight 16-byte pieces, piece p of row r at p ^ (r % 8)
    __shared__ i32x4 stage[3 * BM * 8];
    const int lane = threadIdx.x & 63, wave = wave_id(), col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in), steps = chunks / 2;
    const int nb = (n_tiles + BN - 1) / BN, mb = (a.rows + BM - 1) / BM;
    // Workgroups go to the eight L2 caches in turn: each gets neighbouring blocks, 4 of rows by some of outputs
    int id = (int)blockIdx.x;
    const int all = nb * mb, per = (all + 7) / 8, cut = all & 7;
    {
        const int x = id & 7, i = id >> 3;
        id = cut == 0 || x < cut ? x * per + i : cut * per + (x - cut) * (per - 1) + i;
    }
    const int band = id / (4 * nb), rows_here = min(4, mb - band * 4), in = id - band * 4 * nb;
    const int m0 = (band * 4 + in % rows_here) * BM, tile0 = in / rows_here * BN + wave / WM * NT, mw = wave % WM * MT * 16;
    const uint8_t *wp[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) wp[t] = a.packed + (long long)min(tile0 + t, n_tiles - 1) * chunks * kW8Record + lane * 16;
    const int r0 = (int)threadIdx.x >> 3, piece = (int)threadIdx.x & 7;
    const int8_t *xp[MINE];
#pragma unroll
    for (int j = 0; j < MINE; j++) xp[j] = a.x + (long long)min(m0 + r0 + THREADS / 8 * j, a.rows - 1) * a.x_stride;
    i32x4 raw[MINE], w[2][NT], x[2][HALF], acc[MT][NT] = {};
    // past the inputs codes times weights of 0, past the last step ones that are not used
    const auto fetch = [&](i32x4 (&raw)[MINE], int s) {
        const int k = min(s * 128 + piece * 16, a.n_in - 16);
#pragma unroll
        for (int j = 0; j < MINE; j++) raw[j] = load16b(xp[j] + k);
    };
    const auto weights = [&](int s, int d) {
        const long long at = (long long)(2 * min(s, steps - 1) + d) * kW8Record;
#pragma unroll
        for (int t = 0; t < NT; t++) w[d][t] = *(const i32x4 *)(wp[t] + at);
    };
    const auto put = [&](const i32x4 (&raw)[MINE], int at) {
#pragma unroll
        for (int j = 0; j < MINE; j++) stage[at + (r0 + THREADS / 8 * j) * 8 + (piece ^ (r0 & 7))] = raw[j];
    };
    const auto rows = [&](i32x4 (&x)[HALF], int at, int d, int h) {
#pragma unroll
        for (int m = 0; m < HALF; m++) x[m] = stage[at + (mw + 16 * (h * HALF + m) + col) * 8 + ((4 * d + qt) ^ (col & 7))];
    };
    const auto compute = [&](const i32x4 (&x)[HALF], int d, int h) {
#pragma unroll
        for (int m = 0; m < HALF; m++)
#pragma unroll
            for (int t = 0; t < NT; t++) acc[h * HALF + m][t] = mfma8(w[d][t], x[m], acc[h * HALF + m][t]);
    };
    constexpr int ONE = BM * 8;
    {
        // in the order of the loop (rows, then weights), so that at its head no load is awaited for another's sake
        i32x4 one[MINE], two[MINE];
        fetch(one, 0);
        fetch(two, 1);
        fetch(raw, 2);
        __builtin_amdgcn_sched_barrier(0);
        weights(0, 0);
        weights(0, 1);
        __builtin_amdgcn_sched_barrier(0);
        put(one, 0);
        put(two, ONE);
    }
    lds_barrier();
    int now = 0, next = ONE, after = 2 * ONE;
    rows(x[0], now, 0, 0);
    for (int s = 0; s < steps; s++) {
        // in this order: left to itself the compiler puts every load at the end of the step
        const auto pin = [] { __builtin_amdgcn_sched_barrier(0); };
        rows(x[1], now, 0, 1);
        pin();
        compute(x[0], 0, 0);
        pin();
        put(raw, after);   // step s + 2
        fetch(raw, s + 3);
        rows(x[0], now, 1, 0);
        pin();
        compute(x[1], 0, 1);
        pin();
        weights(s + 1, 0);
        rows(x[1], now, 1, 1);
        pin();
        compute(x[0], 1, 0);
        pin();
        rows(x[0], next, 0, 0);
        pin();
        compute(x[1], 1, 1);
        pin();
        weights(s + 1, 1);
        pin();
        lds_barrier();
        const int done = now;
        now = next;
        next = after;
        after = done;
    }
    // no load goes ahead of a store by itself: all scales first (4096 x 4096 x 1024: 26.8 us, each with its store 32.4)
    Ends<F16> ends[NT];
    float xs[MT];
#pragma unroll
    for (int t = 0; t < NT; t++) ends[t].fetch(a, (tile0 + t) * kW8Tile + qt * 4);
#pragma unroll
    for (int m = 0; m < MT; m++) xs[m] = a.x_scales[min(m0 + mw + 16 * m + col, a.rows - 1)];
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
            // of two tiles' outputs 4 qt .. + 3 of a row to outputs 8 qt .. + 7, so that lanes side by side have 64 bytes of it
            // (the same: 23.2 us, with 32 bytes 26.8)
            ends[t].xs = ends[t + 1].xs = xs[m];
            const u32x2 p = ends[t].outputs(a, acc[m][t]), q = ends[t + 1].outputs(a, acc[m][t + 1]);
            u32x4 o;
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const auto far = __builtin_amdgcn_permlane32_swap(p[i], q[i], false, false);
                const auto near = __builtin_amdgcn_permlane16_swap(far[0], far[1], false, false);
                o[i] = near[0];
                o[2 + i] = near[1];
            }
            const int row = m0 + mw + 16 * m + col, n = (tile0 + t) * kW8Tile + qt * 8;
            if (row >= a.rows || n >= a.n_out) continue;
            uint16_t *y = (uint16_t *)a.y + (long long)row * a.y_stride + n;
            if (n + 8 <= a.n_out) __builtin_memcpy(__builtin_assume_aligned(y, 2), &o, 16);
            else
#pragma unroll
                for (int j = 0; j < 7; j++)
                    if (n + j < a.n_out) y[j] = (uint16_t)(o[j >> 1] >> (16 * (j & 1)));
        }
}

// Some rows (up to a few hundred; bound by trips to memory).  A workgroup's waves are KP parts of the inputs times TW tiles
// of 16 outputs.  The waves of a part share the rows: 128 inputs of them go into LDS (pieces as in w8_tiles_kernel) while the
// inputs before are computed, so that they come from memory once for 16 TW outputs; rows and weights are DEEP steps
// ahead in registers (loads return in order: the one that is awaited has to be as old as all the
// others).  At the end the parts add up through LDS.  blockIdx.y: the block of rows.  77 x 5003 x 4112: 10.3 us, of which 4.4
// are the bytes.
template <bool F16, int MT, int KP, int TW, int DEEP>
__global__ __launch_bounds__(KP * TW * 64) void w8_rows_kernel(W8Args a)
{
    constexpr int ROWS = MT * 16, PIECES = ROWS * 8, THREADS = TW * 64, MINE = (PIECES + THREADS - 1) / THREADS;
    constexpr int SUMS = TW * MT * 64, Q = (MT + KP - 1) / KP, STAGE = KP * 2 * PIECES;
    static_assert(DEEP % 2 == 0, "rounds end where they began");
    __shared__ i32x4 lds[STAGE > KP * SUMS ? STAGE : KP * SUMS];
    const int lane = threadIdx.x & 63, wave = wave_id(), kp = wave / TW, tw = wave % TW, col = lane & 15, qt = lane >> 4;
    const int n_tiles = (a.n_out + kW8Tile - 1) / kW8Tile, chunks = (int)w8_chunks(a.n_in), steps = chunks / 2;
    const int tile0 = (int)blockIdx.x * TW, m0 = (int)blockIdx.y * ROWS;
    // every part takes as many steps, so that barriers meet; c1: its end
    const int many = (steps + KP - 1) / KP, c0 = kp * many, c1 = min(c0 + many, steps);
    const uint8_t *wp = a.packed + (long long)min(tile0 + tw, n_tiles - 1) * chunks * kW8Record + lane * 16;
    i32x4 *stage = lds + kp * 2 * PIECES;
    const int t0 = tw * 64 + lane, r0 = t0 >> 3, piece = t0 & 7;
    const int8_t *xp[MINE];
#pragma unroll
    for (int j = 0; j < MINE; j++) xp[j] = a.x + (long long)min(m0 + r0 + j * THREADS / 8, a.rows - 1) * a.x_stride;
    // always a load, so that the compiler can count them: past the rows the last one (it is not stored),
    // past the inputs some codes (weights of 0, or not used), past the part some step (it is not used)
    i32x4 raw[DEEP][MINE], w[DEEP][2];
    const auto fetch = [&](i32x4 (&raw)[MINE], int c) {
        const int k = min(c * 128 + piece * 16, a.n_in - 16);
#pragma unroll
        for (int j = 0; j < MINE; j++) raw[j] = load16b(xp[j] + k);
    };
    const auto put = [&](const i32x4 (&raw)[MINE], int buf) {
#pragma unroll
        for (int j = 0; j < MINE; j++) {
            const int r = r0 + j * THREADS / 8;
            if (PIECES % THREADS == 0 || r < ROWS) stage[buf * PIECES + r * 8 + (piece ^ (r & 7))] = raw[j];
        }
    };
    const auto weights = [&](i32x4 (&w)[2], int c) {
#pragma unroll
        for (int d = 0; d < 2; d++) w[d] = *(const i32x4 *)(wp + (long long)(2 * min(c, steps - 1) + d) * kW8Record);
    };
    // this thread's outputs
    Ends<F16> ends[Q];
    int em[Q], en[Q];
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int e = (int)threadIdx.x + q * KP * THREADS, l = e & 63, mt = e >> 6;
        em[q] = e < SUMS ? m0 + mt / TW * 16 + (l & 15) : a.rows;
        en[q] = (tile0 + mt % TW) * kW8Tile + (l >> 4) * 4;
        ends[q].fetch(a, em[q], en[q]);
    }
    i32x4 acc[MT] = {};
    // in the order of the loop, so that at its head the compiler counts the same loads from both sides
    fetch(raw[0], c0);
#pragma unroll
    for (int d = 0; d < DEEP; d++) {
        if (d == DEEP - 1) put(raw[0], 0);
        fetch(raw[(d + 1) % DEEP], c0 + d + 1);
        weights(w[d], c0 + d);
    }
    lds_barrier();
    const auto compute = [&](const i32x4 (&w)[2], int c, int buf) {
        if (c >= c1) return;
#pragma unroll
        for (int h = 0; h < 2; h++) {
#pragma unroll
            for (int m = 0; m < MT; m++)
                acc[m] = mfma8(w[h], stage[buf * PIECES + (m * 16 + col) * 8 + ((4 * h + qt) ^ (col & 7))], acc[m]);
        }
    };
    int c = c0;
    for (; c + DEEP <= c0 + many; c += DEEP) {
#pragma unroll
        for (int d = 0; d < DEEP; d++) {
            put(raw[(d + 1) % DEEP], (d & 1) ^ 1);   // step c + d + 1
            fetch(raw[(d + 1) % DEEP], c + d + 1 + DEEP);
            compute(w[d], c + d, d & 1);
            weights(w[d], c + d + DEEP);
            lds_barrier();
        }
    }
#pragma unroll
    for (int d = 0; d < DEEP - 1; d++) {   // what is left of a round
        if (c + d >= c0 + many) break;
        put(raw[d + 1], (d & 1) ^ 1);
        compute(w[d], c + d, d & 1);
        lds_barrier();
    }
    // the loop's last barrier is behind the last reads of the rows
#pragma unroll
    for (int m = 0; m < MT; m++) lds[(kp * MT * TW + m * TW + tw) * 64 + lane] = acc[m];
    lds_barrier();
#pragma unroll
    for (int q = 0; q < Q; q++) {
        const int e = (int)threadIdx.x + q * KP * THREADS;
        if (e >= SUMS) break;
        i32x4 sum = lds[e];
#pragma unroll
        for (int v = 1; v < KP; v++) sum += lds[v * SUMS + e];
        ends[q].store(a, em[q], en[q], sum);
    }
}

template <bool F16, int NT, int NW, int D>
hipError_t go_few(const W8Args &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW8Tile - 1) / kW8Tile);
    if (a.x_scales) hipLaunchKernelGGL((w8_few_kernel<F16, NT, NW, D, false>), dim3((tiles + NT - 1) / NT), dim3(NW * 64), 0, s, a);
    else hipLaunchKernelGGL((w8_few_kernel<F16, NT, NW, D, true>), dim3((tiles + NT - 1) / NT), dim3(NW * 64), 0, s, a);
    return hipGetLastError();
}

template <bool F16, int MT, int NT, int WM, int WN>
hipError_t go_tiles(const W8Args &a, hipStream_t s)
{
    constexpr int BM = WM * MT * 16, BN = WN * NT * 16;
    const long long blocks = (long long)((a.n_out + BN - 1) / BN) * ((a.rows + BM - 1) / BM);
    hipLaunchKernelGGL((w8_tiles_kernel<F16, MT, NT, WM, WN>), dim3((unsigned)blocks), dim3(WM * WN * 64), 0, s, a);
    return hipGetLastError();
}

template <bool F16, int MT, int KP, int TW, int DEEP>
hipError_t go_rows(const W8Args &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW8Tile - 1) / kW8Tile);
    const unsigned nb = (tiles + TW - 1) / TW, mb = (a.rows + MT * 16 - 1) / (MT * 16);
    // workgroups go to the eight L2 caches in turn: with a multiple of 8 in a row all blocks of rows of the same outputs to the
    // same one (77 x 5000 x 4096: 10.2 us, else 11.8; 130 x 4100 x 4096: 9.9 and 13.4); what is past the outputs stores nothing
    hipLaunchKernelGGL((w8_rows_kernel<F16, MT, KP, TW, DEEP>), dim3(mb == 1 ? nb : (nb + 7) / 8 * 8, mb), dim3(KP * TW * 64), 0, s, a);
    return hipGetLastError();
}

template <bool F16>
hipError_t pick(const W8Args &a, hipStream_t s)
{
    switch (w8_form(a.rows, a.n_out, a.n_in)) {
        case kW8Few16: return go_few<F16, 1, 16, 2>(a, s);
        case kW8Few8x2: return go_few<F16, 2, 8, 2>(a, s);
        case kW8Rows32x1: return go_rows<F16, 2, 4, 1, 4>(a, s);
        case kW8Rows32: return go_rows<F16, 2, 2, 2, 4>(a, s);
        case kW8Rows32x4: return go_rows<F16, 2, 2, 4, 4>(a, s);
        case kW8Block32: return go_rows<F16, 2, 4, 2, 2>(a, s);
        case kW8Block64: return go_rows<F16, 4, 4, 2, 2>(a, s);
        case kW8Block64x4: return go_rows<F16, 4, 2, 4, 2>(a, s);
        case kW8Block128x4: return go_rows<F16, 8, 2, 4, 2>(a, s);
        case kW8Tiles128: return go_tiles<F16, 4, 4, 2, 4>(a, s);
        case kW8Tiles256: return go_tiles<F16, 8, 4, 2, 4>(a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_w8_pack(const W8PackArgs &a, hipStream_t s)
{
    const unsigned tiles = (unsigned)((a.n_out + kW8Tile - 1) / kW8Tile), chunks = (unsigned)w8_chunks(a.n_in);
    hipLaunchKernelGGL(w8_pack_kernel, dim3((chunks + 3) / 4, tiles < 16384 ? tiles : 16384), dim3(256), 0, s, a);
    return hipGetLastError();
}

// Forms, with both sides measured (us, outputs x inputs, weights from memory):
// * up to 16 rows a workgroup a tile of outputs, 16 waves (1 x 4096 x 4096: 5.0, 8 waves 5.6); of many outputs two tiles, so
//   that the rows are read half as often (16 x 8192 x 8192: 13.3, one 16.2; 16 x 28672 x 4096: 24.2, one 28.5).
// * up to 32 the rows go through LDS, of few outputs for one tile with the inputs in four parts (32 x 4096 x 4096: 6.7; 22 x 1970 x
//   16320: 15.4, two tiles and two parts 18.9), for two tiles (32 x 4096 x 4096: 7.1, the form for 16 rows with two of them 7.8; 32 x 8192 x
//   8192: 15.2 and 23), or four of many outputs (32 x 28672 x 4096: 25.8, two 28.7).
// * past that blocks of rows and outputs, by what each form would take: a + b k + (c + d k) r us, k its inputs over 4096, r its
//   blocks over the 256 compute units (tiles, of which a unit holds one: rounded up).  Fitted to 75 sizes of 33 to 4096 rows, 260
//   to 29000 outputs and 400 to 14000 inputs, timed with every form: within 10 to 15 % of them, and the form that it takes is
//   1.8 % behind the best at the mean and 23 % at most.  Blocks of 32 x 32, 64 x 32, 64 x 64, 128 x 64, 128 x 256, 256 x 256:
//   64 x 4096 x 4096: 6.7, 8.5, 9.5, 14, 27, 45; 512 x 4096 x 4096: 32, 27, 18, 18, 29, 46; 1032 x 14180 x 1600: 128, 108, 60, 67, 38, 54;
//   4096 x 8192 x 8192: 1350, 750, 490, 410, 260, 217.
W8Form w8_form(int rows, int n_out, int n_in)
{
    const long long tiles = (n_out + kW8Tile - 1) / kW8Tile;
    if (rows <= 16) return tiles <= 256 ? kW8Few16 : kW8Few8x2;
    if (rows <= 32) return tiles <= 256 ? kW8Rows32x1 : tiles <= 1024 ? kW8Rows32 : kW8Rows32x4;
    const struct {
        W8Form form;
        int rows, outputs;
        float a, b, c, d;
    } forms[] = {{kW8Block32, 32, 32, 2.8f, 1.5f, 0.6f, 4.1f},    {kW8Block64, 64, 32, 2.8f, 2.9f, 1.3f, 5.3f},
                 {kW8Block64x4, 64, 64, 3.4f, 4.5f, 1.3f, 6.6f},  {kW8Block128x4, 128, 64, 3.6f, 8.7f, 3.3f, 8.1f},
                 {kW8Tiles128, 128, 256, 0.f, 0.f, 6.6f, 25.9f},  {kW8Tiles256, 256, 256, 0.f, 0.f, 9.2f, 39.2f}};
    W8Form best = kW8Block32;
    float least = INFINITY;
    const float k = (float)n_in / 4096.f;
    for (const auto &f : forms) {
        const long long blocks = ((rows + f.rows - 1ll) / f.rows) * ((n_out + f.outputs - 1ll) / f.outputs);
        const bool tiles = f.form == kW8Tiles128 || f.form == kW8Tiles256;
        const float r = tiles ? (float)((blocks + 255) / 256) : (float)blocks / 256.f, us = f.a + f.b * k + (f.c + f.d * k) * r;
        if (us < least) {
            least = us;
            best = f.form;
        }
    }
    return best;
}

// Three rows have the threads of four.
bool w8_takes_16(int rows, int n_in) { return rows <= kW8Rows16 && (rows == 3 ? 4ll : rows) * n_in <= kW8Lds; }

hipError_t launch_w8(const W8Args &a, bool f16, hipStream_t s) { return f16 ? pick<true>(a, s) : pick<false>(a, s); }

}  // namespace mfs
