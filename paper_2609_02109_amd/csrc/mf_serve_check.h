// What the served steps' C entries (mf_serve_api.cpp, mf_serve8_api.cpp) check arguments with.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "mf_serve.h"

namespace mfs {

// A C caller may pass any int as an enum: read through its representation.
inline int as_int(const mf_dtype &d)
{
    int v;
    static_assert(sizeof v == sizeof d, "mf_dtype is int-sized");
    std::memcpy(&v, &d, sizeof v);
    return v;
}

inline bool half_type(int d) { return d == MF_BF16 || d == MF_F16; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
inline mf_status of(hipError_t e) { return e == hipSuccess ? MF_OK : MF_EDEVICE; }

// Rows of `heads` times D elements at these strides: no two overlap, and the
// furthest element stays within 2^62 elements.
inline bool strides_fit(int64_t rows, int64_t stride, int64_t heads, int64_t head, int64_t d, bool out)
{
    const int64_t most = (int64_t)1 << 40;
    if (stride < 0 || head < 0 || stride > most || head > most) return false;
    if (!out) return true;
    // outputs: heads inside rows or rows inside heads
    if (heads > 1 && head < d) return false;
    if (rows > 1 && stride < d) return false;
    return heads <= 1 || rows <= 1 || stride >= (heads - 1) * head + d || head >= (rows - 1) * stride + d;
}

// Pieces of len bytes in up to two levels of steps, the larger one first; at 0: none.
struct Place {
    typedef __int128 wide;   // a piece may begin 2^70 bytes behind the first
    wide at, end;
    int64_t len, n[2], step[2];
    int levels;
    // Piece i of the first level.
    Place piece(wide i) const
    {
        const wide from = at + i * step[0];
        return {from, from + len + (levels > 1 ? wide(n[1] - 1) * step[1] : 0), len, {n[1], 0}, {step[1], 0}, levels - 1};
    }
};
inline Place place(const void *p, int64_t len, int64_t n = 1, int64_t step = 0, int64_t n2 = 1, int64_t step2 = 0)
{
    const Place::wide at = (Place::wide)(uintptr_t)p;
    Place r = {at, at + len, len, {0, 0}, {0, 0}, 0};
    const bool swap = step2 > step;
    for (int i = 0; i < 2; i++) {
        const int64_t many = (i == 0) == swap ? n2 : n, by = (i == 0) == swap ? step2 : step;
        if (many <= 1 || by == 0) continue;   // the same bytes again
        r.end += (Place::wide)(many - 1) * by;
        r.n[r.levels] = many;
        r.step[r.levels++] = by;
    }
    return r;
}
inline Place::wide floor_of(Place::wide a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); }

// Whether x and y have no byte together.  Ones that lie between one another in more than a few pieces at different steps are
// taken to have.
inline bool apart(const Place &x, const Place &y)
{
    typedef Place::wide wide;
    if (x.end <= y.at || y.end <= x.at) return true;
    if (x.levels == 0 && y.levels == 0) return false;
    const auto most = [](wide p, wide q) { return p > q ? p : q; };
    if (x.levels > 0 && y.levels > 0 && x.step[0] == y.step[0]) {
        // piece i of x and j of y meet or not by j - i alone
        const int64_t step = x.step[0];
        const Place p = x.piece(0), q = y.piece(0);
        const wide lo = most(floor_of(p.at - q.end, step) + 1, -wide(x.n[0] - 1));
        const wide hi = -most(floor_of(q.at - p.end, step) + 1, -wide(y.n[0] - 1));
        if (hi - lo >= 16) return false;
        for (wide d = lo; d <= hi; d++)
            if (!apart(p, y.piece(d))) return false;
        return true;
    }
    const bool of_x = y.levels == 0 || (x.levels > 0 && x.step[0] > y.step[0]);
    const Place &a = of_x ? x : y, &b = of_x ? y : x, first = a.piece(0);
    const wide lo = most(floor_of(b.at - first.end, a.step[0]) + 1, 0);
    const wide hi = -most(floor_of(a.at - b.end, a.step[0]) + 1, -wide(a.n[0] - 1));
    if (hi - lo >= 16) return false;
    for (wide i = lo; i <= hi; i++)
        if (!apart(a.piece(i), b)) return false;
    return true;
}
inline bool apart(const Place &x, std::initializer_list<Place> all)
{
    for (const Place &y : all)
        if (x.at != 0 && y.at != 0 && !apart(x, y)) return false;
    return true;
}

// The batch of a call over a cache's pages; `run`: its device arrays too.
inline mf_status check_batch(int page_size, const void *d_pages, const mf_kv4_batch *b, bool run, KvBatch &o)
{
    if (!b) return MF_EINVAL;
    if (b->n_seq < 0 || b->max_new < 0 || b->max_kv < 0 || b->rows < 0 || b->table_cols < 0) return MF_EINVAL;
    if (b->n_seq > (1 << 20) || b->rows > (1 << 30) || b->max_kv > (1 << 30)) return MF_EUNSUPPORTED;
    if ((int64_t)b->max_kv > (int64_t)b->table_cols * page_size) return MF_EINVAL;
    if (b->table_stride < 0 || b->table_stride > ((int64_t)1 << 40) || (b->n_seq > 1 && b->table_stride < b->table_cols)) return MF_EINVAL;
    if (run && b->n_seq > 0 && b->rows > 0) {
        if (!d_pages || !aligned(d_pages, 256)) return MF_EINVAL;
        if (!b->d_q_start || !b->d_kv_len || !aligned(b->d_q_start, 4) || !aligned(b->d_kv_len, 4)) return MF_EINVAL;
        if (b->table_cols > 0 && (!b->d_page_table || !aligned(b->d_page_table, 4))) return MF_EINVAL;
    }
    o.n_seq = b->n_seq;
    o.max_new = b->max_new < b->rows ? b->max_new : (int)b->rows;
    o.max_kv = b->max_kv;
    o.rows = (int)b->rows;
    o.q_start = b->d_q_start;
    o.kv_len = b->d_kv_len;
    o.table = b->d_page_table;
    o.table_stride = b->table_stride;
    return MF_OK;
}

// Where a step's rows of `heads` times D elements lie, a cache's pages, and what a batch has on the device.
inline Place place_of_rows(const void *p, int64_t rows, int64_t stride, int64_t heads, int64_t head, int64_t d, int64_t size = 2)
{
    return place(p, d * size, rows, stride * size, heads, head * size);
}
inline Place place_of_pages(const KvGeom &g, const void *d_pages)
{
    return place(d_pages, (int64_t)g.n_pages * g.n_kv_heads * g.blocks_per_page * (g.rec + (g.group ? 0 : (int64_t)sizeof(KvScales))));
}
inline bool apart_from_batch(const Place &x, const mf_kv4_batch *b)
{
    const int64_t n = b->n_seq;
    return apart(x, {place(b->d_q_start, (n + 1) * 4), place(b->d_kv_len, n * 4), place(b->table_cols > 0 ? b->d_page_table : nullptr, b->table_cols * 4ll, n, b->table_stride * 4)});
}
// Whether rows of results lie over their source itself: each element is read by those who write it, and before that.
inline bool itself(const void *in, int64_t stride, int64_t head, const void *out, int64_t out_stride, int64_t out_head, int64_t rows, int64_t heads)
{
    return in == out && (rows <= 1 || stride == out_stride) && (heads <= 1 || head == out_head);
}

// The arguments of an append to a cache of geometry a.g; none: there is nothing to do.
inline mf_status check_append(const void *d_pages, const mf_kv4_batch *batch, const mf_kv4_append_args *args, KvAppendArgs &a, bool &none)
{
    const mf_status st = check_batch(a.g.blocks_per_page * kKvBlock, d_pages, batch, true, a.b);
    if (st != MF_OK) return st;
    if (!args || !half_type(as_int(args->dtype))) return MF_EINVAL;
    const int64_t rows = batch->rows, d = a.g.head_dim;
    if ((args->d_cos == nullptr) != (args->d_sin == nullptr)) return MF_EINVAL;
    if (args->d_q && (!args->d_cos || !args->d_q_out || args->n_heads < 1)) return MF_EINVAL;
    if (args->n_heads < 0) return MF_EINVAL;
    if (args->n_heads > 4096) return MF_EUNSUPPORTED;
    if (args->d_cos) {
        if (args->rot_dim < 16 || args->rot_dim > d) return MF_EINVAL;
        if (args->rot_dim % 16 != 0) return MF_EUNSUPPORTED;
        if (args->n_pos < batch->max_kv || !aligned(args->d_cos, 4) || !aligned(args->d_sin, 4)) return MF_EINVAL;
    }
    none = rows == 0 || batch->n_seq == 0 || batch->max_new == 0;
    if (none) return MF_OK;
    if (!args->d_k || !args->d_v || !aligned(args->d_k, 2) || !aligned(args->d_v, 2) || !aligned(args->d_q, 2) || !aligned(args->d_q_out, 2))
        return MF_EINVAL;
    if (!strides_fit(rows, args->k_stride, a.g.n_kv_heads, args->k_head_stride, d, false) ||
        !strides_fit(rows, args->v_stride, a.g.n_kv_heads, args->v_head_stride, d, false))
        return MF_EINVAL;
    if (args->d_q && (!strides_fit(rows, args->q_stride, args->n_heads, args->q_head_stride, d, false) ||
                      !strides_fit(rows, args->qo_stride, args->n_heads, args->qo_head_stride, d, true)))
        return MF_EINVAL;
    const Place pages = place_of_pages(a.g, d_pages), k = place_of_rows(args->d_k, rows, args->k_stride, a.g.n_kv_heads, args->k_head_stride, d),
                v = place_of_rows(args->d_v, rows, args->v_stride, a.g.n_kv_heads, args->v_head_stride, d);
    const int64_t angles = args->d_cos ? (int64_t)args->n_pos * (args->rot_dim / 2) * 4 : 0;
    const Place cos = place(args->d_cos, angles), sin = place(args->d_sin, angles);
    if (!apart(pages, {k, v, cos, sin}) || !apart_from_batch(pages, batch)) return MF_EINVAL;
    if (args->d_q) {
        const Place q = place_of_rows(args->d_q, rows, args->q_stride, args->n_heads, args->q_head_stride, d),
                    out = place_of_rows(args->d_q_out, rows, args->qo_stride, args->n_heads, args->qo_head_stride, d);
        if (!apart(out, {pages, k, v, cos, sin}) || !apart_from_batch(out, batch) || !apart(pages, q)) return MF_EINVAL;
        if (!itself(args->d_q, args->q_stride, args->q_head_stride, args->d_q_out, args->qo_stride, args->qo_head_stride, rows, args->n_heads) && !apart(out, q))
            return MF_EINVAL;
    }
    a.k = args->d_k;
    a.v = args->d_v;
    a.q = args->d_q;
    a.q_out = args->d_q_out;
    a.cos = args->d_cos;
    a.sin = args->d_sin;
    a.k_stride = args->k_stride;
    a.k_head = args->k_head_stride;
    a.v_stride = args->v_stride;
    a.v_head = args->v_head_stride;
    a.q_stride = args->q_stride;
    a.q_head = args->q_head_stride;
    a.qo_stride = args->qo_stride;
    a.qo_head = args->qo_head_stride;
    a.rot = args->d_cos ? args->rot_dim : 0;
    a.interleaved = args->interleaved != 0;
    a.n_heads = args->d_q ? args->n_heads : 0;
    return MF_OK;
}

inline mf_status check_read(const void *d_pages, const mf_kv4_batch *batch, int ty, void *d_k, void *d_v, KvReadArgs &a, bool &none)
{
    const mf_status st = check_batch(a.g.blocks_per_page * kKvBlock, d_pages, batch, true, a.b);
    if (st != MF_OK) return st;
    if (ty != MF_F32 && !half_type(ty)) return MF_EINVAL;
    const size_t el = ty == MF_F32 ? 4 : 2;
    if (!aligned(d_k, el) || !aligned(d_v, el)) return MF_EINVAL;
    none = batch->rows == 0 || batch->n_seq == 0 || batch->max_new == 0 || (!d_k && !d_v);
    if (none) return MF_OK;
    const int64_t bytes = batch->rows * a.g.n_kv_heads * a.g.head_dim * (int64_t)el;
    const Place k = place(d_k, bytes), v = place(d_v, bytes), pages = place_of_pages(a.g, d_pages);
    if (!apart(k, {v, pages}) || !apart(v, {pages})) return MF_EINVAL;
    for (const Place &x : {k, v})
        if (x.at != 0 && !apart_from_batch(x, batch)) return MF_EINVAL;
    a.k = d_k;
    a.v = d_v;
    return MF_OK;
}

// The arguments of attention over a cache of geometry a.g; `plan` lays its work over the card.
template <class P>
mf_status check_attn(const void *d_pages, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, bool run, const P &plan, KvAttnArgs &a, KvPlan &p)
{
    const int page_size = a.g.blocks_per_page * kKvBlock;
    const mf_status st = check_batch(page_size, d_pages, batch, run, a.b);
    if (st != MF_OK) return st;
    if (!args || !half_type(as_int(args->dtype))) return MF_EINVAL;
    if (args->n_heads < 1 || args->n_heads % a.g.n_kv_heads != 0 || args->window < 0) return MF_EINVAL;
    if (args->n_heads > 4096) return MF_EUNSUPPORTED;
    if (!std::isfinite(args->scale) || args->scale <= 0.f) return MF_EINVAL;
    a.n_heads = args->n_heads;
    a.per_kv = args->n_heads / a.g.n_kv_heads;
    if (batch->rows * a.per_kv > INT32_MAX - 1024) return MF_EUNSUPPORTED;   // rows of a sequence and key head are an int
    a.window = args->window;
    a.scale_log2 = (float)((double)args->scale * 1.4426950408889634);
    p = plan(a.g, a.b, a.n_heads, a.window);
    // all sequences' units of one head are an int
    if ((((int64_t)batch->max_kv + kAttnUnit - 1) / kAttnUnit + 1) * batch->n_seq > INT32_MAX) return MF_EUNSUPPORTED;
    // a workgroup's number, and a row's of the join, are an int
    const int64_t items = p.row_tiles * batch->n_seq * a.g.n_kv_heads;
    if (p.workgroups > INT32_MAX || (p.slots > 0 && (items * p.slot_rows > INT32_MAX || p.slots > INT32_MAX))) return MF_EUNSUPPORTED;
    a.row_tiles = (int)p.row_tiles;
    a.splits = p.splits;
    a.chunk = p.chunk;
    a.workgroups = (int)p.workgroups;
    a.whole = p.whole;
    a.slots = (int)p.slots;
    a.slot_rows = p.slot_rows;
    return MF_OK;
}

// The operands and the workspace of attention, after check_attn; none: there is nothing to do.
inline mf_status check_attn_run(const mf_kv4_batch *batch, const mf_kv4_attn_args *args, void *d_ws, size_t ws_bytes, const KvPlan &p, KvAttnArgs &a,
                                bool &none)
{
    none = batch->rows == 0 || batch->n_seq == 0 || batch->max_new == 0;
    if (none) return MF_OK;
    if (!args->d_q || !args->d_out || !aligned(args->d_q, 2) || !aligned(args->d_out, 2) || !aligned(args->d_lse, 4)) return MF_EINVAL;
    const int64_t d = a.g.head_dim;
    if (!strides_fit(batch->rows, args->q_stride, args->n_heads, args->q_head_stride, d, false) ||
        !strides_fit(batch->rows, args->out_stride, args->n_heads, args->out_head_stride, d, true))
        return MF_EINVAL;
    const Place q = place_of_rows(args->d_q, batch->rows, args->q_stride, args->n_heads, args->q_head_stride, d),
                out = place_of_rows(args->d_out, batch->rows, args->out_stride, args->n_heads, args->out_head_stride, d),
                lse = place(args->d_lse, batch->rows * args->n_heads * 4), pages = place_of_pages(a.g, a.g.pages);
    if (!itself(args->d_q, args->q_stride, args->q_head_stride, args->d_out, args->out_stride, args->out_head_stride, batch->rows, args->n_heads) && !apart(out, q))
        return MF_EINVAL;
    if (!apart(out, {pages, lse}) || !apart(lse, {pages, q})) return MF_EINVAL;
    if (ws_bytes < p.ws_bytes || (p.ws_bytes > 0 && !d_ws)) return MF_ENOMEM;
    if (p.ws_bytes > 0 && (!aligned(d_ws, 256) || !apart(place(d_ws, (int64_t)p.ws_bytes), {q, out, lse, pages}))) return MF_EINVAL;
    if (!apart_from_batch(out, batch) || (args->d_lse && !apart_from_batch(lse, batch))) return MF_EINVAL;
    a.q = args->d_q;
    a.out = args->d_out;
    a.lse = args->d_lse;
    a.q_stride = args->q_stride;
    a.q_head = args->q_head_stride;
    a.out_stride = args->out_stride;
    a.out_head = args->out_head_stride;
    a.part = (float *)d_ws;
    return MF_OK;
}

}  // namespace mfs
