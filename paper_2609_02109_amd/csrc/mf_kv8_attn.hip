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
        const long long longest = heads * 16 < 1024 ? 1024 : heads * 16 < 4096 ? heads * 16 : 4096;
        p.whole = span <= longest;
        if (p.whole) {
            p.waves = heads < 512 ? 8 : 4;
            p.workgroups = heads;
        } else {
            // as many as are on the card at once, by the kernels' registers; two units each at least
            const int per_cu = p.rt == 2 || g.head_dim == 256 ? 2 : g.head_dim == 64 ? 4 : 3;
            const long long units = (span + kAttnUnit - 1) / kAttnUnit, most = (units * heads + 1) / 2;
            p.workgroups = most < 256 * per_cu ? most : 256 * per_cu;
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
