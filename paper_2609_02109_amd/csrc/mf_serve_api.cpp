// C entry points of the served steps' operators: argument checks, sizes, and
// the kernels' argument blocks.  Nothing here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

#include "mf_serve.h"

using namespace mfs;

namespace {

// A C caller may pass any int as an enum: read through its representation.
int as_int(const mf_dtype &d)
{
    int v;
    static_assert(sizeof v == sizeof d, "mf_dtype is int-sized");
    std::memcpy(&v, &d, sizeof v);
    return v;
}

bool half_type(int d) { return d == MF_BF16 || d == MF_F16; }
bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
mf_status of(hipError_t e) { return e == hipSuccess ? MF_OK : MF_EDEVICE; }

// Rows of `heads` times D elements at these strides: no two overlap, and the
// furthest element stays within 2^62 elements.
bool strides_fit(int64_t rows, int64_t stride, int64_t heads, int64_t head, int64_t d, bool out)
{
    const int64_t most = (int64_t)1 << 40;
    if (stride < 0 || head < 0 || stride > most || head > most) return false;
    if (!out) return true;
    // outputs: heads inside rows or rows inside heads
    if (heads > 1 && head < d) return false;
    if (rows > 1 && stride < d) return false;
    return heads <= 1 || rows <= 1 || stride >= (heads - 1) * head + d || head >= (rows - 1) * stride + d;
}

mf_status check_w4(const mf_w4_desc *d)
{
    if (!d) return MF_EINVAL;
    if (!half_type(as_int(d->dtype))) return MF_EINVAL;
    if (d->group != 32 && d->group != 64 && d->group != 128) return MF_EUNSUPPORTED;
    if (d->n_out < 1 || d->n_in < 1 || d->n_in % d->group != 0) return MF_EINVAL;
    if (d->n_out > kW4MostOut || d->n_in > (1 << 24)) return MF_EUNSUPPORTED;
    return MF_OK;
}

mf_status check_w4_rows(const mf_w4_args *a)
{
    const mf_status st = check_w4(&a->w);
    if (st != MF_OK) return st;
    if (a->rows < 0) return MF_EINVAL;
    // blocks of 32 rows are a grid's third dimension, rows times outputs a grid's first
    if (a->rows > (1 << 20) || a->rows * (a->w.n_out / 4 + 1) > INT32_MAX * (int64_t)256) return MF_EUNSUPPORTED;
    return MF_OK;
}

size_t w4_bytes(const mf_w4_desc &d)
{
    return (size_t)((d.n_out + kW4Tile - 1) / kW4Tile) * (size_t)((d.n_in + kW4Chunk - 1) / kW4Chunk) * w4_record(d.group);
}

mf_status check_cache(const mf_kv4_cache *c, KvGeom &g)
{
    if (!c) return MF_EINVAL;
    if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->group < 1) return MF_EINVAL;
    if (c->page_size % kKvBlock != 0 || c->page_size > 1024 || c->n_kv_heads > 1024) return MF_EUNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return MF_EUNSUPPORTED;
    if ((c->group != 32 && c->group != 64 && c->group != 128) || c->group > c->head_dim) return MF_EUNSUPPORTED;
    g.pages = (uint8_t *)c->d_pages;
    g.n_pages = c->n_pages;
    g.blocks_per_page = c->page_size / kKvBlock;
    g.n_kv_heads = c->n_kv_heads;
    g.head_dim = c->head_dim;
    g.group = c->group;
    g.rec = 16 * c->head_dim + 128 * (c->head_dim / c->group);
    g.magic = block_magic(g.blocks_per_page);
    return MF_OK;
}

// The batch of a call; `run`: its device arrays too.
mf_status check_batch(const mf_kv4_cache *c, const mf_kv4_batch *b, bool run, KvBatch &o)
{
    if (!b) return MF_EINVAL;
    if (b->n_seq < 0 || b->max_new < 0 || b->max_kv < 0 || b->rows < 0 || b->table_cols < 0) return MF_EINVAL;
    if (b->n_seq > (1 << 20) || b->rows > (1 << 30) || b->max_kv > (1 << 30)) return MF_EUNSUPPORTED;
    if ((int64_t)b->max_kv > (int64_t)b->table_cols * c->page_size) return MF_EINVAL;
    if (b->table_stride < 0 || b->table_stride > ((int64_t)1 << 40) || (b->n_seq > 1 && b->table_stride < b->table_cols)) return MF_EINVAL;
    if (run && b->n_seq > 0 && b->rows > 0) {
        if (!c->d_pages || !aligned(c->d_pages, 256)) return MF_EINVAL;
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

mf_status check_attn(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, bool run, KvAttnArgs &a, KvPlan &p)
{
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_batch(cache, batch, run, a.b);
    if (st != MF_OK) return st;
    if (!args || !half_type(as_int(args->dtype))) return MF_EINVAL;
    if (args->n_heads < 1 || args->n_heads % cache->n_kv_heads != 0 || args->window < 0) return MF_EINVAL;
    if (args->n_heads > 4096) return MF_EUNSUPPORTED;
    if (!std::isfinite(args->scale) || args->scale <= 0.f) return MF_EINVAL;
    a.n_heads = args->n_heads;
    a.per_kv = args->n_heads / cache->n_kv_heads;
    if (batch->rows * a.per_kv > INT32_MAX - 1024) return MF_EUNSUPPORTED;   // rows of a sequence and key head are an int
    a.window = args->window;
    a.scale_log2 = (float)((double)args->scale * 1.4426950408889634);
    p = kv4_plan(a.g, a.b, a.n_heads, a.window);
    // all sequences' units of one head are an int
    if ((((int64_t)batch->max_kv + kAttnUnit - 1) / kAttnUnit + 1) * batch->n_seq > INT32_MAX) return MF_EUNSUPPORTED;
    // a workgroup's number, and a row's of the join, are an int
    const int64_t items = p.row_tiles * batch->n_seq * cache->n_kv_heads;
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

}  // namespace

extern "C" {

mf_status mf_w4_pack_bytes(const mf_w4_desc *desc, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    const mf_status st = check_w4(desc);
    if (st == MF_OK) *bytes = w4_bytes(*desc);
    return st;
}

mf_status mf_w4_pack(const mf_w4_desc *desc, const uint8_t *d_codes, const void *d_scales, const uint8_t *d_zeros, void *d_packed,
                     size_t packed_bytes, void *stream)
{
    const mf_status st = check_w4(desc);
    if (st != MF_OK) return st;
    if (!d_codes || !d_scales || !d_packed || !aligned(d_scales, 2) || !aligned(d_packed, 256)) return MF_EINVAL;
    if (packed_bytes < w4_bytes(*desc)) return MF_ENOMEM;
    W4PackArgs a;
    a.codes = d_codes;
    a.zeros = d_zeros;
    a.scales = (const uint16_t *)d_scales;
    a.packed = (uint8_t *)d_packed;
    a.n_out = (int)desc->n_out;
    a.n_in = (int)desc->n_in;
    a.group = desc->group;
    a.f16 = as_int(desc->dtype) == MF_F16;
    return of(launch_w4_pack(a, (hipStream_t)stream));
}

mf_status mf_w4_workspace_size(const mf_w4_args *args, size_t *bytes)
{
    if (!args || !bytes) return MF_EINVAL;
    const mf_status st = check_w4_rows(args);
    if (st == MF_OK) *bytes = args->rows > 0 ? w4_plan((int)args->rows, (int)args->w.n_out, (int)args->w.n_in).ws_bytes : 0;
    return st;
}

mf_status mf_w4_matmul(const mf_w4_args *args, void *d_ws, size_t ws_bytes, void *stream)
{
    if (!args) return MF_EINVAL;
    const mf_status st = check_w4_rows(args);
    if (st != MF_OK) return st;
    const mf_w4_desc &w = args->w;
    if (args->rows == 0) return MF_OK;
    if (!args->d_packed || !aligned(args->d_packed, 256) || !args->d_x || !args->d_y || !aligned(args->d_x, 2) ||
        !aligned(args->d_y, 2) || !aligned(args->d_bias, 2))
        return MF_EINVAL;
    if (!strides_fit(args->rows, args->x_stride, 1, 0, w.n_in, false) || !strides_fit(args->rows, args->y_stride, 1, 0, w.n_out, true) ||
        (args->rows > 1 && args->x_stride < w.n_in))
        return MF_EINVAL;
    W4Args a;
    a.packed = (const uint8_t *)args->d_packed;
    a.x = args->d_x;
    a.bias = args->d_bias;
    a.y = args->d_y;
    a.x_stride = args->x_stride;
    a.y_stride = args->y_stride;
    a.rows = (int)args->rows;
    a.n_out = (int)w.n_out;
    a.n_in = (int)w.n_in;
    const W4Plan p = w4_plan(a.rows, a.n_out, a.n_in);
    if (p.ws_bytes > 0 && (ws_bytes < p.ws_bytes || !d_ws)) return MF_ENOMEM;
    if (p.ws_bytes > 0 && !aligned(d_ws, 256)) return MF_EINVAL;
    return of(launch_w4(a, p, w.group, as_int(w.dtype) == MF_F16, (float *)d_ws, (hipStream_t)stream));
}

mf_status mf_kv4_cache_bytes(const mf_kv4_cache *cache, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    KvGeom g;
    const mf_status st = check_cache(cache, g);
    if (st == MF_OK) *bytes = (size_t)g.n_pages * g.n_kv_heads * g.blocks_per_page * (size_t)g.rec;
    return st;
}

mf_status mf_kv4_append(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_append_args *args, void *stream)
{
    KvAppendArgs a;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_batch(cache, batch, true, a.b);
    if (st != MF_OK) return st;
    if (!args || !half_type(as_int(args->dtype))) return MF_EINVAL;
    const int64_t rows = batch->rows, d = cache->head_dim;
    if ((args->d_cos == nullptr) != (args->d_sin == nullptr)) return MF_EINVAL;
    if (args->d_q && (!args->d_cos || !args->d_q_out || args->n_heads < 1)) return MF_EINVAL;
    if (args->n_heads < 0) return MF_EINVAL;
    if (args->n_heads > 4096) return MF_EUNSUPPORTED;
    if (args->d_cos) {
        if (args->rot_dim < 16 || args->rot_dim > d) return MF_EINVAL;
        if (args->rot_dim % 16 != 0) return MF_EUNSUPPORTED;
        if (args->n_pos < batch->max_kv || !aligned(args->d_cos, 4) || !aligned(args->d_sin, 4)) return MF_EINVAL;
    }
    if (rows == 0 || batch->n_seq == 0 || batch->max_new == 0) return MF_OK;
    if (!args->d_k || !args->d_v || !aligned(args->d_k, 2) || !aligned(args->d_v, 2) || !aligned(args->d_q, 2) || !aligned(args->d_q_out, 2))
        return MF_EINVAL;
    if (!strides_fit(rows, args->k_stride, cache->n_kv_heads, args->k_head_stride, d, false) ||
        !strides_fit(rows, args->v_stride, cache->n_kv_heads, args->v_head_stride, d, false))
        return MF_EINVAL;
    if (args->d_q && (!strides_fit(rows, args->q_stride, args->n_heads, args->q_head_stride, d, false) ||
                      !strides_fit(rows, args->qo_stride, args->n_heads, args->qo_head_stride, d, true)))
        return MF_EINVAL;
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
    return of(launch_kv4_append(a, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_kv4_read(const mf_kv4_cache *cache, const mf_kv4_batch *batch, mf_dtype dtype, void *d_k, void *d_v, void *stream)
{
    KvReadArgs a;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_batch(cache, batch, true, a.b);
    if (st != MF_OK) return st;
    const int ty = as_int(dtype);
    if (ty != MF_F32 && !half_type(ty)) return MF_EINVAL;
    const size_t el = ty == MF_F32 ? 4 : 2;
    if (!aligned(d_k, el) || !aligned(d_v, el)) return MF_EINVAL;
    if (batch->rows == 0 || batch->n_seq == 0 || batch->max_new == 0 || (!d_k && !d_v)) return MF_OK;
    a.k = d_k;
    a.v = d_v;
    return of(launch_kv4_read(a, ty, (hipStream_t)stream));
}

mf_status mf_kv4_workspace_size(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    KvAttnArgs a;
    KvPlan p;
    const mf_status st = check_attn(cache, batch, args, false, a, p);
    if (st == MF_OK) *bytes = p.ws_bytes;
    return st;
}

mf_status mf_kv4_attention(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, void *d_ws,
                           size_t ws_bytes, void *stream)
{
    KvAttnArgs a;
    KvPlan p;
    const mf_status st = check_attn(cache, batch, args, true, a, p);
    if (st != MF_OK) return st;
    if (batch->rows == 0 || batch->n_seq == 0 || batch->max_new == 0) return MF_OK;
    if (!args->d_q || !args->d_out || !aligned(args->d_q, 2) || !aligned(args->d_out, 2) || !aligned(args->d_lse, 4)) return MF_EINVAL;
    const int64_t d = cache->head_dim;
    if (!strides_fit(batch->rows, args->q_stride, args->n_heads, args->q_head_stride, d, false) ||
        !strides_fit(batch->rows, args->out_stride, args->n_heads, args->out_head_stride, d, true))
        return MF_EINVAL;
    if (ws_bytes < p.ws_bytes || (p.ws_bytes > 0 && !d_ws)) return MF_ENOMEM;
    if (p.ws_bytes > 0 && !aligned(d_ws, 256)) return MF_EINVAL;
    a.q = args->d_q;
    a.out = args->d_out;
    a.lse = args->d_lse;
    a.q_stride = args->q_stride;
    a.q_head = args->q_head_stride;
    a.out_stride = args->out_stride;
    a.out_head = args->out_head_stride;
    a.part = (float *)d_ws;
    return of(launch_kv4_attn(a, p, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

}  // extern "C"
