// Device helpers of the served steps' operators: 16-bit types, codes to matrix
// operands, loads that need no more than their elements' alignment.
#pragma once

#include <string.h>

#include "mf_serve.h"

namespace mfs {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

template <typename To, typename From>
__device__ __forceinline__ To bits(const From &v)
{
    static_assert(sizeof(To) == sizeof(From), "same size");
    To r;
    __builtin_memcpy(&r, &v, sizeof r);
    return r;
}

// 16 bytes from an address aligned to 2.
__device__ __forceinline__ u32x4 load16(const void *p)
{
    u32x4 v;
    __builtin_memcpy(&v, __builtin_assume_aligned(p, 2), 16);
    return v;
}

// N dwords from an address aligned to 8, to 16 from four on.
template <int N>
struct Words {
    uint32_t w[N];
};
template <int N>
__device__ __forceinline__ Words<N> load_words(const uint8_t *p)
{
    Words<N> r;
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; i++) {
            const u32x4 v = ((const u32x4 *)p)[i];
#pragma unroll
            for (int j = 0; j < 4; j++) r.w[4 * i + j] = v[j];
        }
    } else {
        static_assert(N == 2, "8 bytes");
        const u32x2 v = *(const u32x2 *)p;
        r.w[0] = v[0];
        r.w[1] = v[1];
    }
    return r;
}

template <bool F16>
__device__ __forceinline__ float to_float(uint16_t h)
{
    if (F16) return (float)bits<_Float16>(h);
    return __uint_as_float((uint32_t)h << 16);
}
template <bool F16>
__device__ __forceinline__ uint16_t from_float(float x)
{
    if (F16) return bits<uint16_t>((_Float16)x);
    return bits<uint16_t>((__bf16)x);
}
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if (F16) {
        const f16x2 v = __builtin_convertvector((f32x2){a, b}, f16x2);
        return bits<uint32_t>(v);
    }
    const bf16x2 v = __builtin_convertvector((f32x2){a, b}, bf16x2);
    return bits<uint32_t>(v);
}

// Codes 2 s, 2 s + 1 of a dword as two values 16 + c of the 16-bit type.  The two
// constants are kept in registers (one scalar, one vector): as literals they
// would make an and and an or of one v_and_or_b32.
struct CodeBits {
    uint32_t mask, sixteen;
};
template <bool F16>
__device__ __forceinline__ CodeBits code_bits()
{
    CodeBits b = {F16 ? 0x03c003c0u : 0x00780078u, F16 ? 0x4c004c00u : 0x41804180u};
    asm("" : "+s"(b.mask));
    asm("" : "+v"(b.sixteen));
    return b;
}
template <bool F16, int S>
__device__ __forceinline__ uint32_t codes2(uint32_t w, const CodeBits &b)
{
    constexpr int left = (F16 ? 6 : 3) - 4 * S;   // to bits 6.. or 3.. of each half
    const uint32_t v = left >= 0 ? w << (left & 31) : w >> (-left & 31);
    return (v & b.mask) | b.sixteen;
}
template <bool F16>
__device__ __forceinline__ u32x4 codes8(uint32_t w, const CodeBits &b)
{
    return (u32x4){codes2<F16, 0>(w, b), codes2<F16, 1>(w, b), codes2<F16, 2>(w, b), codes2<F16, 3>(w, b)};
}

// A row of y in 8 bits: what its largest magnitude (as bits, for infinities and NaN are above all others) makes of it.
struct Row8 {
    float scale, inv;
    bool bad;   // an infinity or a NaN: the scale is a NaN, the codes are 0
};
__device__ __forceinline__ Row8 row8_of(uint32_t top)
{
    Row8 r;
    r.bad = top >= 0x7f800000u;
    const float scale = __uint_as_float(top) * (float)(1.0 / 127.0);
    r.scale = r.bad ? __uint_as_float(0x7fc00000u) : scale < 0x1p-126f ? 0.f : scale;   // below that 1 / scale may leave fp32
    r.inv = r.scale > 0.f ? 1.f / scale : 0.f;
    return r;
}
__device__ __forceinline__ uint32_t code8(const Row8 &r, float y)
{
    return r.bad ? 0u : (uint32_t)(int)fminf(fmaxf(rintf(y * r.inv), -127.f), 127.f) & 255u;
}

// D += A B, 16 x 16 x 32: lane l holds A[l % 16][8 (l / 16) ..+8], B[8 (l / 16) ..+8][l % 16], D[4 (l / 16) + r][l % 16].
template <bool F16>
__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(bits<f16x8>(a), bits<f16x8>(b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(bits<bf16x8>(a), bits<bf16x8>(b), c, 0, 0, 0);
}
// A matrix of ones as an A operand.
template <bool F16>
__device__ __forceinline__ u32x4 ones8()
{
    const uint32_t o = F16 ? 0x3c003c00u : 0x3f803f80u;
    return (u32x4){o, o, o, o};
}

__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// A barrier for what went through LDS.  __syncthreads() also waits for every load
// from memory that is on its way, which is the end of fetching ahead.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48 (the contraction index of an operand).
__device__ __forceinline__ float quarters_max(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quarters_min(float x) { return -quarters_max(-x); }
__device__ __forceinline__ float quarters_sum(float x)
{
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// f over all lanes of a wave, in each of them (f: of 32 bits, in any order).  No trip through LDS, which a __shfl is.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_bits(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <class X, class F>
__device__ __forceinline__ X over_wave(X v, const F &f)
{
    static_assert(sizeof(X) == 4, "32 bits");
    v = f(v, bits<X>(dpp_bits<0xb1>(bits<uint32_t>(v))));    // the neighbour, the other pair of four, the other four of eight, the other eight of sixteen
    v = f(v, bits<X>(dpp_bits<0x4e>(bits<uint32_t>(v))));
    v = f(v, bits<X>(dpp_bits<0x141>(bits<uint32_t>(v))));
    v = f(v, bits<X>(dpp_bits<0x140>(bits<uint32_t>(v))));
    auto r = __builtin_amdgcn_permlane16_swap(bits<uint32_t>(v), bits<uint32_t>(v), false, false);
    v = f(bits<X>((uint32_t)r[0]), bits<X>((uint32_t)r[1]));
    r = __builtin_amdgcn_permlane32_swap(bits<uint32_t>(v), bits<uint32_t>(v), false, false);
    return f(bits<X>((uint32_t)r[0]), bits<X>((uint32_t)r[1]));
}

}  // namespace mfs
