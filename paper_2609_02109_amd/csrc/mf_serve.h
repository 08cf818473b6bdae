// Shared by the operators of the served steps (mf_w4.hip, mf_kv4.hip,
// mf_kv4_attn*.hip, mf_serve_api.cpp): the layouts of the packed weights and of
// the 4-bit cache, kernel argument blocks, launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mf.h"

namespace mfs {

// A launch has fewer than 2^32 threads in a dimension of its grid: the most
// workgroups.  Larger grids are launched in parts.
constexpr long long most_workgroups(int threads) { return ((1ll << 32) - 1) / threads; }

// ---------------------------------------------------------------- codes
// Eight codes of a row, k = 8 q + j, share a dword: code j sits at bits
// 16 (j % 2) + 4 (j / 2), so that a mask takes a pair (2 s, 2 s + 1) to the same
// place in both halves: the two make one register of a matrix operand.

// ------------------------------------------------------- packed 4-bit weights
// [N / 16][K / 128] records: 1024 bytes of codes, then 128 / G x 16 dwords of
// (scale, 16 + zero) in the weights' 16-bit type.  Lane l of a wave holds 16
// bytes of a record: dword i is the codes k = 32 i + 8 (l / 16) .. + 7 of output
// l % 16, the A operand of v_mfma_f32_16x16x32 number i.  Outputs past N and
// inputs past K have code 0 and scale 0.
constexpr int kW4Tile = 16, kW4Chunk = 128, kW4Codes = 1024;
// a workgroup of 512 threads a tile at most (1024 only where there are few tiles), in one launch
constexpr long long kW4MostOut = most_workgroups(512) * kW4Tile;
static_assert(kW4MostOut == (1ll << 27) - 16, "as include/mf.h has it");
__host__ __device__ constexpr int w4_record(int group) { return kW4Codes + (kW4Chunk / group) * 64; }

struct W4Args {
    const uint8_t *packed;
    const void *x, *bias;
    void *y;
    long long x_stride, y_stride;
    int rows, n_out, n_in;
};
struct W4PackArgs {
    const uint8_t *codes, *zeros;
    const uint16_t *scales;
    uint8_t *packed;
    int n_out, n_in, group;
    bool f16;
};
hipError_t launch_w4_pack(const W4PackArgs &a, hipStream_t s);
enum W4Form {
    kW4One16, kW4One8, kW4Four4,        // up to 16 rows: tiles of outputs, waves of a workgroup
    kW4Two8,                            // up to 32 rows, one tile of outputs, 8 waves
    kW4Rows32, kW4Rows64, kW4Rows64x2   // by rows: 32 or 64 of them, one or two tiles of outputs a wave
};
// How the work is laid over the card: a function of the sizes alone.
struct W4Plan {
    W4Form form;
    int splits;       // by rows: parts of the inputs that different workgroups take
    size_t ws_bytes;  // their sums
};
W4Plan w4_plan(int rows, int n_out, int n_in);
hipError_t launch_w4(const W4Args &a, const W4Plan &p, int group, bool f16, float *part, hipStream_t s);

// ------------------------------------------------------------- 4-bit cache
// A page holds, per head and per block of 16 tokens, one record (rec bytes):
//   keys    8 D bytes: lane l's D / 8 bytes at l D / 8; dword i is the codes
//           d = 32 i + 8 (l / 16) .. + 7 of token l % 16 (an A operand)
//   values  8 D bytes: lane l's D / 8 bytes at l D / 8; dword i is dims
//           d = 32 i + l % 16 (pairs s = 0, 2) and 32 i + 16 + l % 16 (s = 1, 3)
//           of tokens 4 (l / 16) .. + 3, pair s / 2 = tokens (2 (s / 2), 2 (s / 2) + 1)
//   binary16 tables: scales [token / 4][keys, values][group][token % 4], key
//   offsets [token][group], value offsets [group][token]
// The values' order makes the matrix product's own result rows (tokens
// 4 (l / 16) + r) the next product's contraction index, so the softmax weights
// never cross lanes.
constexpr int kKvBlock = 16;
// A group with a NaN has a NaN scale and offset 0: offsets are finite.
struct KvGeom {
    uint8_t *pages;
    int n_pages, blocks_per_page, n_kv_heads, head_dim, group;
    int rec;                 // bytes of a record
    unsigned long long magic;   // ceil(2^32 / blocks_per_page): b / blocks_per_page = b magic >> 32 for b < 2^27
};
struct KvBatch {
    int n_seq, max_new, max_kv, rows;
    const int *q_start, *kv_len, *table;
    long long table_stride;
};

__host__ __device__ inline unsigned long long block_magic(int bpp)
{
    return ((1ull << 32) + (unsigned)bpp - 1) / (unsigned)bpp;
}

#ifdef __HIPCC__
__device__ __forceinline__ int page_of_block(const KvGeom &g, int b) { return (int)(((unsigned long long)(unsigned)b * g.magic) >> 32); }

// The record of block b of sequence s for head h; null where the page number
// is not one of the cache's.
__device__ __forceinline__ uint8_t *kv_record(const KvGeom &g, const KvBatch &b, int s, int h, int blk)
{
    const int col = page_of_block(g, blk);
    const int page = b.table[(long long)s * b.table_stride + col];
    if ((unsigned)page >= (unsigned)g.n_pages) return nullptr;
    return g.pages + (((long long)page * g.n_kv_heads + h) * g.blocks_per_page + (blk - col * g.blocks_per_page)) * (long long)g.rec;
}
#endif

struct KvAppendArgs {
    KvGeom g;
    KvBatch b;
    const void *k, *v, *q;
    void *q_out;
    const float *cos, *sin;
    long long k_stride, k_head, v_stride, v_head, q_stride, q_head, qo_stride, qo_head;
    int rot, interleaved, n_heads;
    int first_seq;           // of this launch
};
struct KvReadArgs {
    KvGeom g;
    KvBatch b;
    void *k, *v;
    int first_seq;
};
constexpr int kAttnWaves = 4;
constexpr int kAttnStep = 32;   // tokens a wave takes at a time
constexpr int kAttnUnit = kAttnStep * kAttnWaves;

// Rows a workgroup covers.
__host__ __device__ constexpr int attn_rows(int rt, bool rows_by_wave) { return rt * 16 * (rows_by_wave ? kAttnWaves : 1); }
struct KvAttnArgs {
    KvGeom g;
    KvBatch b;
    const void *q;
    void *out;
    float *lse;
    long long q_stride, q_head, out_stride, out_head;
    float scale_log2;        // softmax scale times log2 e
    int window, n_heads, per_kv;   // per_kv = n_heads / n_kv_heads
    // from the plan (kv4_plan)
    int row_tiles;           // by rows: tiles of rows that a sequence and head can have
    int splits, chunk;       // by rows: parts of the tokens, tokens of a part
    int workgroups, whole;   // by tokens
    int slots, slot_rows;    // room for parts that the join adds up
    int first;               // workgroup of this launch, where they are more than one launch's
    float *part;             // [slot][row][D] sums, then [slot][row] (base, sum of weights)
};
// How the work is laid over the card: a function of the sizes alone.
struct KvPlan {
    int rt;                  // 16-row tiles a wave holds
    bool rows_by_wave;       // the waves of a workgroup take different rows (else: different tokens)
    bool whole;              // by tokens: a workgroup per sequence and head
    int waves;               // by tokens: waves of a workgroup
    long long row_tiles, workgroups, slots;
    int splits, chunk, slot_rows;
    size_t ws_bytes;
};
KvPlan kv4_plan(const KvGeom &g, const KvBatch &b, int n_heads, int window);
hipError_t launch_kv4_append(const KvAppendArgs &a, bool f16, hipStream_t s);
hipError_t launch_kv4_read(const KvReadArgs &a, int dtype, hipStream_t s);
hipError_t launch_kv4_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

}  // namespace mfs
