// Attention over the 8-bit cache: how the work is laid over the card (the kernel
// itself is in mf_kv8_attn.h, the join of parts in mf_kv4_attn.hip).
#include "mf_kv_attn.h"

namespace mfs {

hipError_t launch_attn8_d64(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn8_d128(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn8_d256(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

// By rows: tiles of 64 rt rows, each over `splits` parts of its tokens.  As many parts as leave all workgroups on the card at
// once (two a compute unit; of heads of 64 four), of about eight steps of 32 tokens at the least; a half of that and so on where it
// takes less: parts are written and read (9 x 213 query tokens over 466, 8 over 2 heads of 256: two parts 34 us, one 25).
// us: about what that takes, by figures of heads of 128 that were set by hand beside those below; heads of 64 and of 256 go by them
// too, though a step of theirs has half the work and twice.  Every sequence counts as one of max_new tokens: one long piece of
// a prompt beside decodes leaves no parts (512 over 20000 beside three of one token: 698 us, apart 205 and 30).
struct RowsPlan {
    long long row_tiles, items, splits;
    float us;
};
static RowsPlan rows_plan(int rt, long long rows, long long heads, int head_dim, long long span, long long max_new)
{
    const int wg_rows = attn_rows(rt, true);
    RowsPlan p;
    p.row_tiles = (rows + wg_rows - 1) / wg_rows;
    p.items = p.row_tiles * heads;
    p.us = INFINITY;
    const long long steps = (span + kAttnStep - 1) / kAttnStep, mean = steps - max_new / 2 / kAttnStep, room = head_dim == 64 ? 1024 : 512;
    long long splits = p.items > 0 ? room / p.items : 1;
    if (splits > (mean + 4) / 8) splits = (mean + 4) / 8;
    if (splits < 1) splits = 1;
    for (; splits >= 1; splits /= 2) {
        const float rounds = (float)((p.items * splits + room - 1) / room), parts = (float)(p.items * splits * wg_rows) * (float)(head_dim + 2) * 4.f;
        // a beginning, the steps, and where there are parts their writing, reading and a launch
        const float us = rounds * (9.f + (float)steps / (float)splits * (rt == 1 ? 0.84f : 1.15f)) + (splits > 1 ? 4.f + 2.f * parts / 4e6f : 0.f);
        if (us < p.us) {
            p.us = us;
            p.splits = splits;
        }
    }
    return p;
}

KvPlan kv8_plan(const KvGeom &g, const KvBatch &b, int n_heads, int window)
{
    KvPlan p;
    const long long rows = (long long)b.max_new * (n_heads / g.n_kv_heads);   // of a sequence and key head, at most
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
        // Of heads of 128 a wave takes one tile of 16 rows or two, which share operands (us, one and two, in the best number of parts; 32
        // over 8 heads): 1 x 16 query tokens over 4000: 17, 21; 1 x 300 over 3000: 45, 46; 4 x 64 over 3000: 38, 41; 1 x 1000 over 1000: 34, 40;
        // 4 x 100 over 3000: 55, 53; 1 x 512 over 8000: 121, 100; 2 x 1500 over 3000: 189, 193; 2 x 1024 over 11000: 473, 396.  Of heads of 64
        // one (16 heads, 2 x 500 over 2000: 34, 37; 2 x 1024 over 12000: 190, 197), of heads of 256 two have no room.
        RowsPlan r = rows_plan(1, rows, heads, g.head_dim, span, b.max_new);
        p.rt = 1;
        if (g.head_dim == 128) {
            const RowsPlan two = rows_plan(2, rows, heads, g.head_dim, span, b.max_new);
            if (two.us < r.us) r = two, p.rt = 2;
        }
        const long long steps = (span + kAttnStep - 1) / kAttnStep;
        p.row_tiles = r.row_tiles;
        if (r.splits > 1) {
            const long long per = (steps + r.splits - 1) / r.splits;
            p.chunk = (int)(per * kAttnStep);
            p.splits = (int)((steps + per - 1) / per);
        }
        p.workgroups = r.items * p.splits;
        p.slots = p.splits > 1 ? p.workgroups : 0;
        p.slot_rows = attn_rows(p.rt, true);
    } else {
        p.row_tiles = 1;
        // Whole heads have neither shares to find nor parts to join, which is 3 us and more, but the longest decides, and
        // few heads leave most of the card idle.  us, whole and in shares (heads of 128; one length, then all lengths up to it):
        //   4 x 8 of 1500: 11.7, 11.9 and 11.7, 14.3; of 3000: 17.6, 14.4 and 17.3, 14.7
        //   8 x 8 of 2000: 14.5, 15.6 and 13.3, 13.0; of 4000: 22.1, 20.3 and 21.5, 19.3
        //   16 x 8 of 8000: 41.5, 47.7 and 37.1, 34.6; of 16000: 101.7, 100.7 and 91.6, 70.1
        //   32 x 8 of 8000: 91.5, 100.3 and 55.7, 61.8; of 20000: 221.5, 236.1 and 143.5, 135.8
        // (heads of 64: 16 x 8 of 8000: 29.8, 31.0 and 29.3, 24.6; of 256: 16 x 8 of 8000: 99.7, 103.4 and 84.5, 62.3)
        p.whole = span <= (heads < 64 ? 1536 : heads < 128 ? 2048 : 8192);
        if (p.whole) {
            // few heads: more waves to each (1 x 8 of 1500: 8 waves 11.5, 4 12.4; 128 x 8 of 500: 33.2 and 24.5)
            p.waves = heads < 512 ? 8 : 4;
            p.workgroups = heads;
        } else {
            // two workgroups a compute unit, two units each at least (24 x 8 of 10000: 97.8 us, three 98.5, four 107.1)
            const long long units = (span + kAttnUnit - 1) / kAttnUnit, most = (units * heads + 1) / 2;
            p.workgroups = most < 512 ? most : 512;
            p.slots = 2 * p.workgroups;
        }
        p.slot_rows = (int)rows;
    }
    p.ws_bytes = (size_t)(p.slots * p.slot_rows) * (g.head_dim + 2) * sizeof(float);
    return p;
}

hipError_t launch_kv8_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    const hipError_t e = a.g.head_dim == 64 ? launch_attn8_d64(a, p, f16, s) : a.g.head_dim == 128 ? launch_attn8_d128(a, p, f16, s) : launch_attn8_d256(a, p, f16, s);
    return e != hipSuccess ? e : launch_kv_join(a, p, f16, s);
}

}  // namespace mfs
