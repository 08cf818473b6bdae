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
    // two tiles of rows a wave where the registers of two waves a SIMD hold them (heads of
    // 256: one; two took 164 us where one takes 122, 4 x 300 query tokens over 2000 to 4000)
    p.rows_by_wave = rows > (g.head_dim < 256 ? 32 : 16);
    p.rt = g.head_dim < 256 && rows > 16 ? 2 : 1;
    long long span = b.max_kv;   // tokens that rows of an item go over, at most
    if (window > 0 && (long long)window + b.max_new + kAttnStep < span) span = (long long)window + b.max_new + kAttnStep;
    const long long heads = (long long)b.n_seq * g.n_kv_heads;
    p.splits = 1;
    p.chunk = 0;
    p.slots = 0;
    p.whole = false;
    p.waves = kAttnWaves;
    if (p.rows_by_wave) {
        const int wg_rows = attn_rows(p.rt, true);
        p.row_tiles = (rows + wg_rows - 1) / wg_rows;
        const long long items = p.row_tiles * heads, steps = (span + kAttnStep - 1) / kAttnStep;
        long long splits = items > 0 ? (512 + items - 1) / items : 1;
        if (splits > (steps + 31) / 32) splits = (steps + 31) / 32;
        if (splits > 1) {
            const long long per = (steps + splits - 1) / splits;
            p.chunk = (int)(per * kAttnStep);
            p.splits = (int)((steps + per - 1) / per);
        }
        p.workgroups = items * p.splits;
        p.slots = p.splits > 1 ? p.workgroups : 0;
        p.slot_rows = wg_rows;
    } else {
        p.row_tiles = 1;
        // Whole heads have neither shares to find nor parts to join, which is 3 us and more,
        // but the longest decides.  us, whole and in shares, heads of 128 and one length:
        //   1 x 8 of 1000: 11.0, 12.2; of 1500: 12.9, 12.6; of 4000: 22.7, 12.2
        //   16 x 8 of 2000: 16.5, 22.3; of 3000: 20.8, 21.4; of 6000: 32.1, 31.1
        //   16 x 16 of 4000: 27.2, 36.7; 200 x 8 of 500: 29, 56; of 2000: 94, 120
        // (heads of 64, 16 x 16 of all lengths up to 4000: 19.8, 25.4).  Past 4096 tokens many
        // heads of one length would still be faster whole (16 x 16 of 6000: 37.1, 46.4), of all
        // lengths hardly (31.8, 33.7).
        const long long longest = heads * 16 < 1024 ? 1024 : heads * 16 < 4096 ? heads * 16 : 4096;
        p.whole = span <= longest;
        if (p.whole) {
            // few heads: more waves to each (1 x 8 of 1000: 8 waves 10.5, 4 11.5; 200 x 8 of 600: 47 and 27)
            p.waves = heads < 512 ? 8 : 4;
            p.workgroups = heads;
        } else {
            // as many as are on the card at once, by the kernels' registers; two units each at least
            const int per_cu = p.rt == 2 || g.head_dim == 256 ? 2 : g.head_dim == 64 ? 4 : g.group == 32 ? 2 : 3;
            const long long units = (span + kAttnUnit - 1) / kAttnUnit, most = (units * heads + 1) / 2;
            p.workgroups = most < 256 * per_cu ? most : 256 * per_cu;
            p.slots = 2 * p.workgroups;
        }
        p.slot_rows = (int)rows;
    }
    p.ws_bytes = (size_t)(p.slots * p.slot_rows) * (g.head_dim + 2) * sizeof(float);
    return p;
}

namespace {

constexpr int kJoinWaves = 4;

// Adds up `parts` parts of a row (latency: 4 parts on their way at a time, 1 x 60000 tokens
// 28.6 -> 27.0 us in all): part i is in slot first (i = 0) or rest + i * step.
// The workgroup's threads take four dims and every so many parts each.
template <bool F16, int D>
__device__ __forceinline__ void join_row(const KvAttnArgs &a, long long first, long long rest, long long step, int parts, int srow,
                                         long long qrow, int head)
{
    constexpr int T = D / 4, PG = kJoinWaves * 64 / T;   // threads over a row, parts at a time
    __shared__ f32x4 so[PG][T];
    __shared__ f32x2 sm[PG];
    const int t = threadIdx.x % T, g = threadIdx.x / T;
    const f32x2 *ml = (const f32x2 *)(a.part + (long long)a.slots * a.slot_rows * D);
    float base = kNoBase, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    // four parts on their way at a time; past the last its like, with no weight
    for (int i = g; i < parts; i += 4 * PG) {
        f32x2 m[4];
        f32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int k = min(i + j * PG, parts - 1);
            const long long at = (k ? rest + k * step : first) * a.slot_rows + srow;
            m[j] = ml[at];
            v[j] = *(const f32x4 *)(a.part + at * D + 4 * t);
        }
        float to = base;
#pragma unroll
        for (int j = 0; j < 4; j++) to = fmaxf(to, m[j][0]);
        const float x = __builtin_amdgcn_exp2f(base - to);
        base = to;
        l *= x;
        o *= x;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (i + j * PG >= parts) break;
            const float y = __builtin_amdgcn_exp2f(m[j][0] - to);
            l += m[j][1] * y;
#pragma unroll
            for (int r = 0; r < 4; r++) o[r] += v[j][r] * y;
        }
    }
    so[g][t] = o;
    if (t == 0) sm[g] = (f32x2){base, l};
    __syncthreads();
    if (g != 0) return;
    const int n = parts < PG ? parts : PG;
    for (int i = 0; i < n; i++) base = fmaxf(base, sm[i][0]);
    l = 0.f;
    o = (f32x4){0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n; i++) {
        const float x = __builtin_amdgcn_exp2f(sm[i][0] - base);
        l += sm[i][1] * x;
        o += so[i][t] * x;
    }
    uint16_t *out = (uint16_t *)a.out + qrow * a.out_stride + (long long)head * a.out_head + 4 * t;
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no token; a NaN stays one
#pragma unroll
    for (int r = 0; r < 4; r++) out[r] = from_float<F16>(o[r] * inv);
    if (a.lse && t == 0) a.lse[qrow * a.n_heads + head] = l == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// A workgroup per row that work items may have.
template <bool F16, int D>
__global__ __launch_bounds__(kJoinWaves * 64) void join_rows_kernel(KvAttnArgs a)
{
    const int wg = a.first + (int)blockIdx.x, item = wg / a.slot_rows, rr = wg % a.slot_rows;
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
    const long long row = (long long)tile * a.slot_rows + rr;
    if (row >= (long long)sr.n * a.per_kv) return;
    const int i = (int)(row / a.per_kv);
    join_row<F16, D>(a, (long long)item * a.splits, (long long)item * a.splits, 1, a.splits, rr, sr.q0 + i,
                     h * a.per_kv + (int)(row - (long long)i * a.per_kv));
}

// Few parts, up to what join_row takes at a time: D / 4 threads a row add them up as it does, bit for bit, four dims
// each, and a workgroup takes several rows (1 x 2000 over 2000 of the 4-bit cache, 32 heads over 8 of 128, two parts: 121 us in
// all, by a workgroup a row 171).
template <bool F16, int D>
__global__ __launch_bounds__(kJoinWaves * 64) void join_few_kernel(KvAttnArgs a)
{
    constexpr int T = D / 4, ROWS = kJoinWaves * 64 / T;
    // rows of a workgroup are of one item: an item's slots are a multiple of 64 rows
    const long long r0 = ((long long)a.first + blockIdx.x) * ROWS;
    const int item = (int)(r0 / a.slot_rows), rr = (int)(r0 - (long long)item * a.slot_rows) + (int)threadIdx.x / T, t = threadIdx.x % T;
    const int tile = item % a.row_tiles, sh = item / a.row_tiles, h = sh % a.g.n_kv_heads, s = sh / a.g.n_kv_heads;
    const SeqRows sr = seq_rows(a.b, seq_raw(a.b, s));
    const long long row = (long long)tile * a.slot_rows + rr;
    if (row >= (long long)sr.n * a.per_kv) return;
    const f32x2 *ml = (const f32x2 *)(a.part + (long long)a.slots * a.slot_rows * D);
    const long long first = (long long)item * a.splits * a.slot_rows + rr;
    float base = kNoBase, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.splits; i++) base = fmaxf(base, ml[first + (long long)i * a.slot_rows][0]);
    const float end = ml[first + (long long)(a.splits - 1) * a.slot_rows][0];
    for (int i = 0; i < a.splits; i += 4) {
        f32x2 m[4];
        f32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const long long at = first + (long long)min(i + j, a.splits - 1) * a.slot_rows;
            m[j] = ml[at];
            v[j] = *(const f32x4 *)(a.part + at * D + 4 * t);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (i + j >= a.splits) break;
            // by way of the last part's base, as join_row has it: the same bits
            const float to = fmaxf(m[j][0], end), y = __builtin_amdgcn_exp2f(m[j][0] - to), x = __builtin_amdgcn_exp2f(to - base);
            l += m[j][1] * y * x;
            o += v[j] * y * x;
        }
    }
    const int i = (int)(row / a.per_kv), head = h * a.per_kv + (int)(row - (long long)i * a.per_kv);
    const long long qrow = sr.q0 + i;
    const float inv = l == 0.f ? 0.f : 1.f / l;   // no token; a NaN stays one
    uint16_t y[4];
#pragma unroll
    for (int r = 0; r < 4; r++) y[r] = from_float<F16>(o[r] * inv);
    __builtin_memcpy((uint16_t *)a.out + qrow * a.out_stride + (long long)head * a.out_head + 4 * t, y, 8);
    if (a.lse && t == 0) a.lse[qrow * a.n_heads + head] = l == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
}

// A workgroup per row of a sequence and head: its parts are those of the workgroups
// whose shares the head's units lie in.
template <bool F16, int D>
__global__ __launch_bounds__(kJoinWaves * 64) void join_tokens_kernel(KvAttnArgs a)
{
    const int wg = a.first + (int)blockIdx.x, item = wg / a.slot_rows, rr = wg % a.slot_rows;
    const int h = item % a.g.n_kv_heads, s = item / a.g.n_kv_heads, lane = threadIdx.x & 63;
    const SeqRaw raw = seq_raw(a.b, s);
    const SeqRows sr = seq_rows(a.b, raw);
    if (rr >= (long long)sr.n * a.per_kv) return;
    long long total = 0, before = 0;
    for (int s0 = 0; s0 < a.b.n_seq; s0 += 64) {
        const Lanes l = lanes_at(a, s0, lane);
        if (s >= s0 && s < s0 + 64) before = total + __builtin_amdgcn_readlane(l.upto - l.units, s - s0);
        total += l.all;
    }
    const long long share = (total * a.g.n_kv_heads + a.workgroups - 1) / a.workgroups, units = units_of(a, raw);
    const long long b0 = before * a.g.n_kv_heads + h * units, w0 = b0 / share, w1 = (b0 + units - 1) / share;
    if (w0 == w1) return;   // one workgroup had it whole
    const int i = rr / a.per_kv;
    join_row<F16, D>(a, 2 * w0 + 1, 2 * w0, 2, (int)(w1 - w0 + 1), rr, sr.q0 + i, h * a.per_kv + rr - i * a.per_kv);
}

template <int D>
hipError_t go_join(const KvAttnArgs &a, const KvPlan &p, bool f16, long long items, hipStream_t s)
{
    const auto go = [&](void (*kernel)(KvAttnArgs)) { return each_launch(kernel, a, items * a.slot_rows, kJoinWaves * 64, s); };
    constexpr int few = kJoinWaves * 64 / (D / 4);
    // a thread goes over its row's parts one after another, which pays where there are rows for all compute units: a workgroup a row
    // and several rows to one, us, of the 4-bit cache (rows that tiles have x parts): 1024 x 8: 30.4, 33.7; 2048 x 8: 32.2, 34.6; 4096 x 3:
    // 33.1, 30.9; 8192 x 8: 55.3, 51.4; of the 8-bit one: 4096 x 16: 38.0, 42.3; 7168 x 9: 33.3, 31.3; 1024 x 16: 14.0, 21.2
    if (p.rows_by_wave && a.splits <= few && items * a.slot_rows > 512 * (long long)a.splits)
        return each_launch(f16 ? join_few_kernel<true, D> : join_few_kernel<false, D>, a, items * a.slot_rows / few, kJoinWaves * 64, s);
    if (p.rows_by_wave) return f16 ? go(join_rows_kernel<true, D>) : go(join_rows_kernel<false, D>);
    return f16 ? go(join_tokens_kernel<true, D>) : go(join_tokens_kernel<false, D>);
}

}  // namespace

hipError_t launch_kv_join(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    if (p.slots == 0) return hipSuccess;
    const long long items = p.row_tiles * a.b.n_seq * a.g.n_kv_heads;
    return a.g.head_dim == 64 ? go_join<64>(a, p, f16, items, s) : a.g.head_dim == 128 ? go_join<128>(a, p, f16, items, s) : go_join<256>(a, p, f16, items, s);
}

hipError_t launch_kv4_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    const hipError_t e = a.g.head_dim == 64 ? launch_attn_d64(a, p, f16, s) : a.g.head_dim == 128 ? launch_attn_d128(a, p, f16, s) : launch_attn_d256(a, p, f16, s);
    return e != hipSuccess ? e : launch_kv_join(a, p, f16, s);
}

}  // namespace mfs
