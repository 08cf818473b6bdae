// C entry points of the operators of an 8-bit variant's step: argument checks,
// sizes, and the kernels' argument blocks.  Nothing here allocates or synchronises.
#include "mf_serve_check.h"

using namespace mfs;

namespace {

// Row strides of `n` elements each that a call's rows may have.
bool row_stride(int64_t rows, int64_t stride, int64_t n, bool out) { return strides_fit(rows, stride, 1, 0, n, out) && (rows <= 1 || stride >= n); }

// Rows of n values of `size` bytes.
Place rows_at(const void *p, int64_t rows, int64_t stride, int64_t n, int64_t size) { return place(p, n * size, rows, stride * size); }

// What every call over rows has.
mf_status check_rows8(const mf_rows8_args *r)
{
    if (!half_type(as_int(r->dtype)) || r->rows < 0 || r->n < 1) return MF_EINVAL;
    if (r->rows > (1 << 30) || r->n > kRows8Most) return MF_EUNSUPPORTED;
    if (r->rows == 0) return MF_OK;
    if (!r->d_x || !r->d_codes || !r->d_scales || !aligned(r->d_x, 2) || !aligned(r->d_scales, 4)) return MF_EINVAL;
    if (!row_stride(r->rows, r->x_stride, r->n, false) || !row_stride(r->rows, r->codes_stride, r->n, true)) return MF_EINVAL;
    return MF_OK;
}

// Whether the codes and the scales lie over none of the row's x and what else a call reads and writes, nor over one another.
bool rows8_apart(const mf_rows8_args &r, const Place &one = {}, const Place &two = {}, const Place &three = {})
{
    const Place x = rows_at(r.d_x, r.rows, r.x_stride, r.n, 2), codes = rows_at(r.d_codes, r.rows, r.codes_stride, r.n, 1), scales = place(r.d_scales, r.rows * 4);
    return apart(codes, {scales, x, one, two, three}) && apart(scales, {x, one, two, three});
}

Rows8Args rows8_of(const mf_rows8_args &r)
{
    Rows8Args a = {};
    a.x = r.d_x;
    a.codes = r.d_codes;
    a.scales = r.d_scales;
    a.rows = r.rows;
    a.n = (int)r.n;
    a.x_stride = r.x_stride;
    a.codes_stride = r.codes_stride;
    return a;
}

mf_status check_w8(const mf_w8_desc *d)
{
    if (!d) return MF_EINVAL;
    if (!half_type(as_int(d->dtype)) || d->n_out < 1 || d->n_in < 1) return MF_EINVAL;
    if (d->n_in % 16 != 0 || d->n_out > kW8MostOut || d->n_in > kW8MostIn) return MF_EUNSUPPORTED;
    return MF_OK;
}

mf_status check_w8_rows(const mf_w8_args *a)
{
    const mf_status st = check_w8(&a->w);
    if (st != MF_OK) return st;
    if (a->rows < 0) return MF_EINVAL;
    // blocks of 128 rows and 256 outputs are a grid's first dimension: 2^37 outputs are 2^22 of them, of 512 threads
    return a->rows > (1 << 20) || a->rows * a->w.n_out > (int64_t)1 << 37 ? MF_EUNSUPPORTED : MF_OK;
}

size_t w8_records(const mf_w8_desc &d) { return (size_t)((d.n_out + kW8Tile - 1) / kW8Tile) * (size_t)w8_chunks((int)d.n_in) * kW8Record; }
size_t w8_bytes(const mf_w8_desc &d) { return w8_records(d) + (size_t)((d.n_out + kW8Tile - 1) / kW8Tile) * kW8Tile * sizeof(float); }

mf_status check_cache8(const mf_kv8_cache *c, KvGeom &g)
{
    if (!c) return MF_EINVAL;
    if (c->n_pages < 1 || c->page_size < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return MF_EINVAL;
    if (c->page_size % kKvBlock != 0 || c->page_size > 1024 || c->n_kv_heads > 1024) return MF_EUNSUPPORTED;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return MF_EUNSUPPORTED;
    g.pages = (uint8_t *)c->d_pages;
    g.n_pages = c->n_pages;
    g.blocks_per_page = c->page_size / kKvBlock;
    g.n_kv_heads = c->n_kv_heads;
    g.head_dim = c->head_dim;
    g.group = 0;
    g.rec = 32 * c->head_dim;
    g.magic = block_magic(g.blocks_per_page);
    return MF_OK;
}

// The workspace: codes and scales of rows that come in 16 bits, where the product does not put them into 8 itself.
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t w8_ws(const mf_w8_args &a)
{
    if (a.rows == 0 || a.d_x_scales || w8_takes_16((int)a.rows, (int)a.w.n_in)) return 0;
    return up256((size_t)a.rows * (size_t)a.w.n_in) + (size_t)a.rows * sizeof(float);
}

}  // namespace

extern "C" {

mf_status mf_rows8(const mf_rows8_args *args, void *stream)
{
    if (!args) return MF_EINVAL;
    const mf_status st = check_rows8(args);
    if (st != MF_OK || args->rows == 0) return st;
    if (!rows8_apart(*args)) return MF_EINVAL;
    return of(launch_rows8(rows8_of(*args), kRowsPlain, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_norm8(const mf_norm8_args *args, void *stream)
{
    if (!args) return MF_EINVAL;
    const mf_rows8_args &r = args->row;
    const mf_status st = check_rows8(&r);
    if (st != MF_OK) return st;
    if (!std::isfinite(args->eps) || args->eps < 0.f) return MF_EINVAL;
    if (r.rows == 0) return MF_OK;
    if (!args->d_weight || !aligned(args->d_weight, 2)) return MF_EINVAL;
    Rows8Args a = rows8_of(r);
    const Place weight = place(args->d_weight, 2 * r.n);
    Place residual = {}, sum = {};
    if (args->d_residual) {
        if (!args->d_sum || !aligned(args->d_residual, 2) || !aligned(args->d_sum, 2)) return MF_EINVAL;
        if (!row_stride(r.rows, args->residual_stride, r.n, false) || !row_stride(r.rows, args->sum_stride, r.n, true)) return MF_EINVAL;
        residual = rows_at(args->d_residual, r.rows, args->residual_stride, r.n, 2);
        sum = rows_at(args->d_sum, r.rows, args->sum_stride, r.n, 2);
        // over a row itself, which has to lie as it does, or over none
        const auto itself_or_apart = [&](const void *x, int64_t stride) {
            return (x == args->d_sum && (r.rows == 1 || stride == args->sum_stride)) || apart(sum, rows_at(x, r.rows, stride, r.n, 2));
        };
        if (!itself_or_apart(r.d_x, r.x_stride) || !itself_or_apart(args->d_residual, args->residual_stride) || !apart(sum, weight)) return MF_EINVAL;
        a.y = args->d_residual;
        a.sum = args->d_sum;
        a.y_stride = args->residual_stride;
        a.sum_stride = args->sum_stride;
    }
    if (!rows8_apart(r, residual, sum, weight)) return MF_EINVAL;
    a.weight = args->d_weight;
    a.eps = args->eps;
    return of(launch_rows8(a, kRowsNorm, as_int(r.dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_gate8(const mf_gate8_args *args, void *stream)
{
    if (!args) return MF_EINVAL;
    const mf_rows8_args &r = args->row;
    const mf_status st = check_rows8(&r);
    if (st != MF_OK || r.rows == 0) return st;
    if (!args->d_up || !aligned(args->d_up, 2) || !row_stride(r.rows, args->up_stride, r.n, false)) return MF_EINVAL;
    if (!rows8_apart(r, rows_at(args->d_up, r.rows, args->up_stride, r.n, 2))) return MF_EINVAL;
    Rows8Args a = rows8_of(r);
    a.y = args->d_up;
    a.y_stride = args->up_stride;
    return of(launch_rows8(a, kRowsGate, as_int(r.dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_rows8_values(mf_dtype dtype, int64_t rows, int64_t n, const int8_t *d_codes, int64_t codes_stride, const float *d_scales,
                          void *d_out, int64_t out_stride, void *stream)
{
    const int ty = as_int(dtype);
    if ((ty != MF_F32 && !half_type(ty)) || rows < 0 || n < 1) return MF_EINVAL;
    if (rows > (1 << 30) || n > kRows8Most) return MF_EUNSUPPORTED;
    if (rows == 0) return MF_OK;
    if (!d_codes || !d_scales || !d_out || !aligned(d_scales, 4) || !aligned(d_out, ty == MF_F32 ? 4 : 2)) return MF_EINVAL;
    if (!row_stride(rows, codes_stride, n, false) || !row_stride(rows, out_stride, n, true)) return MF_EINVAL;
    if (!apart(rows_at(d_out, rows, out_stride, n, ty == MF_F32 ? 4 : 2), {rows_at(d_codes, rows, codes_stride, n, 1), place(d_scales, rows * 4)})) return MF_EINVAL;
    Values8Args a;
    a.codes = d_codes;
    a.scales = d_scales;
    a.out = d_out;
    a.rows = rows;
    a.codes_stride = codes_stride;
    a.out_stride = out_stride;
    a.n = (int)n;
    return of(launch_values8(a, ty, (hipStream_t)stream));
}

mf_status mf_w8_pack_bytes(const mf_w8_desc *desc, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    const mf_status st = check_w8(desc);
    if (st == MF_OK) *bytes = w8_bytes(*desc);
    return st;
}

mf_status mf_w8_pack(const mf_w8_desc *desc, const int8_t *d_codes, const float *d_scales, void *d_packed, size_t packed_bytes, void *stream)
{
    const mf_status st = check_w8(desc);
    if (st != MF_OK) return st;
    if (!d_codes || !d_scales || !d_packed || !aligned(d_scales, 4) || !aligned(d_packed, 256)) return MF_EINVAL;
    if (packed_bytes < w8_bytes(*desc)) return MF_ENOMEM;
    if (!apart(place(d_packed, (int64_t)w8_bytes(*desc)), {place(d_codes, desc->n_out * desc->n_in), place(d_scales, desc->n_out * 4)})) return MF_EINVAL;
    W8PackArgs a;
    a.codes = d_codes;
    a.scales = d_scales;
    a.packed = (uint8_t *)d_packed;
    a.n_out = (int)desc->n_out;
    a.n_in = (int)desc->n_in;
    return of(launch_w8_pack(a, (hipStream_t)stream));
}

mf_status mf_w8_workspace_size(const mf_w8_args *args, size_t *bytes)
{
    if (!args || !bytes) return MF_EINVAL;
    const mf_status st = check_w8_rows(args);
    if (st == MF_OK) *bytes = w8_ws(*args);
    return st;
}

mf_status mf_w8_matmul(const mf_w8_args *args, void *d_ws, size_t ws_bytes, void *stream)
{
    if (!args) return MF_EINVAL;
    const mf_status st = check_w8_rows(args);
    if (st != MF_OK) return st;
    const mf_w8_desc &w = args->w;
    if (args->rows == 0) return MF_OK;
    if (!args->d_packed || !aligned(args->d_packed, 256) || !args->d_x || !args->d_y || !aligned(args->d_x, args->d_x_scales ? 1 : 2) ||
        !aligned(args->d_x_scales, 4) || !aligned(args->d_y, 2) || !aligned(args->d_bias, 2))
        return MF_EINVAL;
    if (!row_stride(args->rows, args->x_stride, w.n_in, false) || !row_stride(args->rows, args->y_stride, w.n_out, true)) return MF_EINVAL;
    const int64_t size = args->d_x_scales ? 1 : 2;
    const Place x = rows_at(args->d_x, args->rows, args->x_stride, w.n_in, size), y = rows_at(args->d_y, args->rows, args->y_stride, w.n_out, 2);
    const Place scales = place(args->d_x_scales, args->rows * 4), bias = place(args->d_bias, w.n_out * 2), packed = place(args->d_packed, (int64_t)w8_bytes(w));
    if (!apart(y, {x, scales, bias, packed})) return MF_EINVAL;
    const size_t need = w8_ws(*args);
    if (need > 0 && (ws_bytes < need || !d_ws)) return MF_ENOMEM;
    if (need > 0 && (!aligned(d_ws, 256) || !apart(place(d_ws, (int64_t)need), {x, bias, packed, y}))) return MF_EINVAL;
    W8Args a;
    a.packed = (const uint8_t *)args->d_packed;
    a.w_scales = (const float *)(a.packed + w8_records(w));
    a.x = (const int8_t *)args->d_x;
    a.x16 = args->d_x;
    a.x_scales = args->d_x_scales;
    a.bias = args->d_bias;
    a.y = args->d_y;
    a.x_stride = args->x_stride;
    a.y_stride = args->y_stride;
    a.rows = (int)args->rows;
    a.n_out = (int)w.n_out;
    a.n_in = (int)w.n_in;
    const bool f16 = as_int(w.dtype) == MF_F16;
    if (need > 0) {
        Rows8Args r = {};
        r.x = args->d_x;
        r.x_stride = args->x_stride;
        r.rows = a.rows;
        r.n = a.n_in;
        r.codes = (int8_t *)d_ws;
        r.codes_stride = a.n_in;
        r.scales = (float *)(r.codes + up256((size_t)a.rows * a.n_in));
        const hipError_t e = launch_rows8(r, kRowsPlain, f16, (hipStream_t)stream);
        if (e != hipSuccess) return of(e);
        a.x = r.codes;
        a.x_stride = r.codes_stride;
        a.x_scales = r.scales;
    }
    return of(launch_w8(a, f16, (hipStream_t)stream));
}

mf_status mf_kv8_cache_bytes(const mf_kv8_cache *cache, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    KvGeom g;
    const mf_status st = check_cache8(cache, g);
    if (st == MF_OK) *bytes = (size_t)g.n_pages * g.n_kv_heads * g.blocks_per_page * ((size_t)g.rec + sizeof(KvScales));
    return st;
}

mf_status mf_kv8_append(const mf_kv8_cache *cache, const mf_kv4_batch *batch, const mf_kv4_append_args *args, void *stream)
{
    KvAppendArgs a;
    bool none = true;
    mf_status st = check_cache8(cache, a.g);
    if (st == MF_OK) st = check_append(cache->d_pages, batch, args, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv8_append(a, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

mf_status mf_kv8_read(const mf_kv8_cache *cache, const mf_kv4_batch *batch, mf_dtype dtype, void *d_k, void *d_v, void *stream)
{
    KvReadArgs a;
    bool none = true;
    mf_status st = check_cache8(cache, a.g);
    if (st == MF_OK) st = check_read(cache->d_pages, batch, as_int(dtype), d_k, d_v, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv8_read(a, as_int(dtype), (hipStream_t)stream));
}

mf_status mf_kv8_workspace_size(const mf_kv8_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, size_t *bytes)
{
    if (!bytes) return MF_EINVAL;
    KvAttnArgs a;
    KvPlan p;
    mf_status st = check_cache8(cache, a.g);
    if (st == MF_OK) st = check_attn(cache->d_pages, batch, args, false, kv8_plan, a, p);
    if (st == MF_OK) *bytes = p.ws_bytes;
    return st;
}

mf_status mf_kv8_attention(const mf_kv8_cache *cache, const mf_kv4_batch *batch, const mf_kv4_attn_args *args, void *d_ws,
                           size_t ws_bytes, void *stream)
{
    KvAttnArgs a;
    KvPlan p;
    bool none = true;
    mf_status st = check_cache8(cache, a.g);
    if (st == MF_OK) st = check_attn(cache->d_pages, batch, args, true, kv8_plan, a, p);
    if (st == MF_OK) st = check_attn_run(batch, args, d_ws, ws_bytes, p, a, none);
    if (st != MF_OK || none) return st;
    return of(launch_kv8_attn(a, p, as_int(args->dtype) == MF_F16, (hipStream_t)stream));
}

}  // extern "C"
