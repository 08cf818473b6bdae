// C entry points of the served steps' operators: argument checks, sizes, and
// the kernels' argument blocks.  Nothing here allocates or synchronises.
#include "mf_serve_check.h"

using namespace mfs;

namespace {

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
    const int64_t groups = desc->n_out * (desc->n_in / desc->group);
    if (!apart(place(d_packed, (int64_t)w4_bytes(*desc)), {place(d_codes, desc->n_out * (desc->n_in / 2)), place(d_scales, groups * 2), place(d_zeros, groups)})) return MF_EINVAL;
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
    const Place x = place(args->d_x, w.n_in * 2, args->rows, args->x_stride * 2), y = place(args->d_y, w.n_out * 2, args->rows, args->y_stride * 2);
    const Place bias = place(args->d_bias, w.n_out * 2), packed = place(args->d_packed, (int64_t)w4_bytes(w));
    if (!apart(y, {x, bias, packed}) || (p.ws_bytes > 0 && !apart(place(d_ws, (int64_t)p.ws_bytes), {x, bias, packed, y}))) return MF_EINVAL;
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
    bool none = true;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_append(cache->d_pages, batch, args, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv4_append(a, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_kv4_read(const mf_kv4_cache *cache, const mf_kv4_batch *batch, mf_dtype dtype, void *d_k, void *d_v, void *stream)
{
    KvReadArgs a;
    bool none = true;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_read(cache->d_pages, batch, as_int(dtype), d_k, d_v, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv4_read(a, as_int(dtype), (hipStream_t)stream));
}

mf_status mf_kv4_workspace_size(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    KvAttnArgs a;
    KvPlan p;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_attn(cache->d_pages, batch, args, false, kv4_plan, a, p);
    if (st == MF_OK) *bytes = p.ws_bytes;
    return st;
}

mf_status mf_kv4_attention(const mf_kv4_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, void *d_ws,
                           size_t ws_bytes, void *stream)
{
    KvAttnArgs a;
    KvPlan p;
    bool none = true;
    mf_status st = check_cache(cache, a.g);
    if (st == MF_OK) st = check_attn(cache->d_pages, batch, args, true, kv4_plan, a, p);
    if (st == MF_OK) st = check_attn_run(batch, args, d_ws, ws_bytes, p, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv4_attn(a, p, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

}  // extern "C"
