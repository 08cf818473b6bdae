// Attention over the 4-bit cache: how the work is laid over the card, and the
// join of the parts of long contexts (the kernel itself is in mf_kv4_attn.h).
#include "mf_kv4_attn.h"

namespace mfs {

hipError_t launch_attn_d64(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn_d128(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn_d256(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

KvPlan kv4_plan(const KvGeom &g, const KvBatch &b, int n_heads, int window)
{
    KvPlan p;
    const long long rows = (long long)b.max_new * (n_heads / g.n_kv_heads);   // of a sequence and key head, at most
    p.rows_by_wave = rows > (g.head_dim < 256 ? 32 : 16);
    p.rt = p.rows_by_wave || rows > 16 ? 2 : 1;
    const int wg_rows = attn_rows(p.rt, p.rows_by_wave);
    p.row_tiles = (rows + wg_rows - 1) / wg_rows;
    p.items = p.row_tiles * b.n_seq * g.n_kv_heads;
    long long span = b.max_kv;   // tokens that a work item goes over, at most
    if (window > 0 && (long long)window + b.max_new + kAttnStep < span) span = (long long)window + b.max_new + kAttnStep;
    const long long steps = (span + kAttnStep - 1) / kAttnStep;
    // some 1024 workgroups in all, eight steps each at least
    long long splits = p.items > 0 ? (1024 + p.items - 1) / p.items : 1;
    if (splits > (steps + 7) / 8) splits = (steps + 7) / 8;
    if (splits < 1) splits = 1;
    const long long per = (steps + splits - 1) / splits;
    p.chunk = (int)(per * kAttnStep);
    p.splits = per > 0 ? (int)((steps + per - 1) / per) : 1;
    if (p.splits < 1) p.splits = 1;
    p.ws_bytes = p.splits > 1 ? (size_t)p.items * p.splits * wg_rows * (g.head_dim + 2) * sizeof(float) : 0;
    return p;
}

namespace {

// A wave per row: the parts' sums, each scaled to the common maximum, in order.
template <bool F16, int D>
__global__ __launch_bounds__(64) void attn_join_kernel(KvAttnArgs a, int wg_rows)
{
    const int item = (int)(blockIdx.x / wg_rows), rr = (int)(blockIdx.x % wg_rows);
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const int q0 = a.b.q_start[s];
    const long long q1 = a.b.q_start[s + 1];
    const int n = q0 < 0 || q0 >= a.b.rows || q1 <= q0 ? 0 : (int)((q1 < a.b.rows ? q1 : a.b.rows) - q0);
    const long long row = (long long)tile * wg_rows + rr;
    if (row >= (long long)n * a.per_kv) return;
    const int i = (int)(row / a.per_kv), head = h * a.per_kv + (int)(row - (long long)i * a.per_kv), lane = threadIdx.x;
    const f32x2 *ml = (const f32x2 *)(a.part + (long long)a.items * a.splits * wg_rows * D);
    const long long at = (long long)item * a.splits * wg_rows + rr;
    float m = -INFINITY;
    for (int p = 0; p < a.splits; p++) m = fmaxf(m, ml[at + (long long)p * wg_rows][0]);
    float l = 0.f, o[D / 64] = {};
    for (int p = 0; p < a.splits; p++) {
        const f32x2 part = ml[at + (long long)p * wg_rows];
        const float x = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(part[0] - m);
        l += part[1] * x;
        const float *y = a.part + (at + (long long)p * wg_rows) * D;
#pragma unroll
        for (int d = 0; d < D / 64; d++) o[d] += y[d * 64 + lane] * x;
    }
    uint16_t *out = (uint16_t *)a.out + (long long)(q0 + i) * a.out_stride + (long long)head * a.out_head;
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no token; a NaN stays one
#pragma unroll
    for (int d = 0; d < D / 64; d++) out[d * 64 + lane] = from_float<F16>(o[d] * inv);
    if (a.lse && lane == 0)
        a.lse[(long long)(q0 + i) * a.n_heads + head] =
            l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

template <int D>
void go_join(const KvAttnArgs &a, int wg_rows, bool f16, hipStream_t s)
{
    const dim3 grid((unsigned)((long long)a.items * wg_rows));
    if (f16) hipLaunchKernelGGL((attn_join_kernel<true, D>), grid, dim3(64), 0, s, a, wg_rows);
    else hipLaunchKernelGGL((attn_join_kernel<false, D>), grid, dim3(64), 0, s, a, wg_rows);
}

}  // namespace

hipError_t launch_kv4_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    const hipError_t e = a.g.head_dim == 64 ? launch_attn_d64(a, p, f16, s) : a.g.head_dim == 128 ? launch_attn_d128(a, p, f16, s) : launch_attn_d256(a, p, f16, s);
    if (e != hipSuccess || a.splits == 1) return e;
    const int wg_rows = attn_rows(p.rt, p.rows_by_wave);
    if (a.g.head_dim == 64) go_join<64>(a, wg_rows, f16, s);
    else if (a.g.head_dim == 128) go_join<128>(a, wg_rows, f16, s);
    else go_join<256>(a, wg_rows, f16, s);
    return hipGetLastError();
}

}  // namespace mfs
