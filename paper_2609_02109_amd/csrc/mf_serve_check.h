// What the served steps' C entries (mf_serve_api.cpp, mf_serve8_api.cpp) check arguments with.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <cstring>

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

}  // namespace mfs
