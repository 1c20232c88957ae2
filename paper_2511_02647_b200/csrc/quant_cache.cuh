// The 4-bit cache.  A row of one head is head_dim / 32 groups of 32 channels.  A group holds 32 nibbles, the even channel in
// the low half of its byte, and one scale byte b; channel c is (nibble - 8) * scale(b), scale(b) = (8 + (b & 7)) * 2^((b >> 3) - 21),
// 2^-18 to 15360 in eight steps per power of two.  nibble - 8 and scale have four significant bits each, so every value that the
// cache can hold is exact in bf16, and so are the steps of the conversion below.
//   codes  [caches][Hkv][cap][head_dim / 2] bytes, scales [caches][Hkv][cap][head_dim / 32] bytes; cap a multiple of 16, so that 16 rows
//   of either are whole 16-byte pieces.
#pragma once

#include "common.cuh"

namespace fedattn {

constexpr int kQuantGroup = 32;

// two scale bytes -> a bf16 pair: a byte is the exponent's lower bits and three of the mantissa.  (Multiplications and additions: the
// pipe for shifts and selections is the one that the conversion fills.)
__device__ __forceinline__ uint32_t scale_pair(uint32_t lo, uint32_t hi) { return hi * 0x00100000u + (lo * 0x10u + 0x36803680u); }
__device__ __forceinline__ uint32_t scale_pair(uint32_t both) { return both * 0x00100010u + 0x36803680u; }
__device__ __forceinline__ float scale_float(uint32_t byte) { return __uint_as_float(((byte << 4) + 0x3680u) << 16); }

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// -136 * scale, what the conversion adds: (128 + nibble) * scale - 136 * scale.  136 = 17 * 8 and scale = m * 2^e, 8 <= m <= 15:
// 17 m has eight bits, exact.
__device__ __forceinline__ uint32_t offset_pair(uint32_t scale)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(scale), "r"(0xc308c308u));
    return r;
}
// The nibbles at bits 4 kAt .. of either half of x as bf16 values: 128 + nibble is 0x4300 | nibble.
template <int kAt> __device__ __forceinline__ uint32_t nibble_pair(uint32_t x, uint32_t scale, uint32_t offset)
{
    // (one selection: written as two operations it was compiled to two.  Shifts as upper halves of products, which other units take:
    // slower, one of three 10.2 -> 11.1 us, all three 12.5, decode of 8 x 4096 rows.)
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x >> (4 * kAt)), "r"(0x000f000fu), "r"(0x43004300u));      // (a & b) | c
    return fma_bf16x2(y, scale, offset);
}

// eight channels: as they lie in memory, then as fp32
template <typename T> struct Eight;
template <> struct Eight<float> {
    float4 a, b;
    __device__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ void load(const float *p) { a = reinterpret_cast<const float4 *>(p)[0]; b = reinterpret_cast<const float4 *>(p)[1]; }
    __device__ void get(float (&x)[8]) const
    {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint4 v;
    __device__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ void get(float (&x)[8]) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};

}  // namespace fedattn
