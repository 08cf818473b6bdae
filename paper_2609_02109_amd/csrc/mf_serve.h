// Shared by the operators of the served steps (mf_w4.hip, mf_kv4.hip,
// mf_kv4_attn*.hip, mf_rows8.hip, mf_w8.hip, mf_kv8.hip, mf_kv8_attn*,
// mf_serve_api.cpp, mf_serve8_api.cpp): the layouts of the packed weights and of
// the caches, kernel argument blocks, launchers.
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
struct KvScales {   // of a record of the 8-bit cache
    float k, v;
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
// Its number among all records of the 8-bit cache, -1 where there is none, and all records' scales.
__device__ __forceinline__ long long kv8_record(const KvGeom &g, const KvBatch &b, int s, int h, int blk)
{
    const int col = page_of_block(g, blk);
    const int page = b.table[(long long)s * b.table_stride + col];
    if ((unsigned)page >= (unsigned)g.n_pages) return -1;
    return ((long long)page * g.n_kv_heads + h) * g.blocks_per_page + (blk - col * g.blocks_per_page);
}
__device__ __forceinline__ KvScales *kv8_scales(const KvGeom &g)
{
    return (KvScales *)(g.pages + (long long)g.n_pages * g.n_kv_heads * g.blocks_per_page * (long long)g.rec);
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
// Adds up the parts that a launch left (either cache's).
hipError_t launch_kv_join(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);
hipError_t launch_kv4_append(const KvAppendArgs &a, bool f16, hipStream_t s);
hipError_t launch_kv4_read(const KvReadArgs &a, int dtype, hipStream_t s);
hipError_t launch_kv4_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

// ------------------------------------------------------------- 8-bit cache
// As the 4-bit cache, with 32 D bytes a record; a byte is a code + 128:
//   keys    64 dims in 1 KB: lane l's 16 bytes at 16 l are dims 64 j + 16 (l / 16)
//           .. + 15 of token l % 16 (two A operands of v_mfma_f32_16x16x32)
//   values  64 dims in 1 KB: lane l's dword i at 16 l + 4 i is dim 64 j + 16 i +
//           l % 16 of tokens 4 (l / 16) .. + 3
// After all records two fp32 numbers for each, in the records' order: the scales
// of its keys and of its values.
// Scales are 2^-40 up to 65504 / 127, or NaN.
constexpr float kKv8LeastScale = 0x1p-40f, kKv8MostScale = 0x1p10f;
hipError_t launch_kv8_append(const KvAppendArgs &a, bool f16, hipStream_t s);
hipError_t launch_kv8_read(const KvReadArgs &a, int dtype, hipStream_t s);
KvPlan kv8_plan(const KvGeom &g, const KvBatch &b, int n_heads, int window);
hipError_t launch_kv8_attn(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s);

// ------------------------------------------------------------ rows in 8 bits
enum Rows8Op { kRowsPlain, kRowsNorm, kRowsGate };
constexpr int kRows8Most = 1 << 17;   // values of a row: 1024 threads of 128
struct Rows8Args {
    const void *x, *y;       // y: the residual (may be null) or the gate's factors
    const void *weight;      // norm
    void *sum;               // norm with a residual: x + y
    int8_t *codes;
    float *scales;
    long long rows, x_stride, y_stride, sum_stride, codes_stride;
    int n;
    float eps;
};
hipError_t launch_rows8(const Rows8Args &a, Rows8Op op, bool f16, hipStream_t s);
struct Values8Args {
    const int8_t *codes;
    const float *scales;
    void *out;
    long long rows, codes_stride, out_stride;
    int n;
};
hipError_t launch_values8(const Values8Args &a, int dtype, hipStream_t s);

// ------------------------------------------------------- packed 8-bit weights
// [N / 16][K / 64] records of 1024 bytes, an even number of them a tile: lane l of a
// wave holds 16 of them, the inputs k = 16 (l / 16) .. + 15 of output l % 16, the A operand of
// v_mfma_i32_16x16x64_i8.  Outputs past N and inputs past K have code 0.  After
// the records the scales of all tiles' outputs, 0 past N.
constexpr int kW8Tile = 16, kW8Chunk = 64, kW8Record = kW8Tile * kW8Chunk;
constexpr long long kW8MostOut = most_workgroups(512) * kW8Tile;   // as kW4MostOut
constexpr int kW8MostIn = 131056;   // 2^14 K < 2^31: products of codes down to -128, in 32 bits
__host__ __device__ constexpr long long w8_chunks(int n_in) { return (n_in + 2 * kW8Chunk - 1) / (2 * kW8Chunk) * 2; }
struct W8Args {
    const uint8_t *packed;
    const float *w_scales;
    const int8_t *x;
    const float *x_scales;   // null: x16, rows of the type, are put into 8 bits by the product itself
    const void *x16;
    const void *bias;
    void *y;
    long long x_stride, y_stride;
    int rows, n_out, n_in;
};
struct W8PackArgs {
    const int8_t *codes;
    const float *scales;
    uint8_t *packed;
    int n_out, n_in;
};
hipError_t launch_w8_pack(const W8PackArgs &a, hipStream_t s);
enum W8Form {
    kW8Few16, kW8Few8x2,                                    // up to 16 rows: waves of a workgroup (x tiles of outputs)
    kW8Rows32x1, kW8Rows32, kW8Rows32x4,                    // up to 32
    kW8Block32, kW8Block64, kW8Block64x4, kW8Block128x4,    // rows of a block (x tiles of outputs, else two)
    kW8Tiles128, kW8Tiles256                                // by 256 outputs
};
// How the work is laid over the card, and whether rows in 16 bits are put into 8 in the product's own kernel: functions of
// the sizes alone.
W8Form w8_form(int rows, int n_out, int n_in);
bool w8_takes_16(int rows, int n_in);
hipError_t launch_w8(const W8Args &a, bool f16, hipStream_t s);

}  // namespace mfs
