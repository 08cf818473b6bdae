// Attention over the 8-bit cache: how the work is laid over the card (the kernel
// itself is in mf_kv8_attn.h, the join of parts in mf_kv4_attn.hip).
#include "mf_kv_attn.h"

namespace mfs {

hipError_t launch_attn8_d64(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn8_d128(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_attn8_d256(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

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
