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

// scale bytes in the low byte of either half -> a bf16 pair: the byte is the exponent's lower bits and three of the mantissa
__device__ __forceinline__ uint32_t scale_pair(uint32_t bytes) { return (bytes << 4) + 0x36803680u; }
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
    return fma_bf16x2(((x >> (4 * kAt)) & 0x000f000fu) | 0x43004300u, scale, offset);
}

}  // namespace fedattn
