// Rows of keys and values into the 4-bit cache and back (quant_cache.cuh has the format).  Bound by memory: 4.25 bits per element
// on one side, the storage type on the other.
//
// Scale of a group: the least of the 256 whose sevenfold reaches the group's largest magnitude.  Code: x / scale to the nearest
// integer, ties to the even one, -7 .. 7.  Both are exact decisions: 7 * scale and code * scale are exact in fp32 (7 and 8
// significant bits), so comparisons with them carry no rounding, and what an approximate quotient gets wrong is put right.
//
// A warp takes one row of one of the two tensors; a lane 8 channels at a time, four lanes a group.
#include "quant_cache.cuh"

namespace fedattn {

namespace {

constexpr int kThreads = 256;

// the least scale byte with 7 * scale >= amax (255 when none has)
__device__ __forceinline__ uint32_t scale_byte(float amax)
{
    // 1/7 rounded: the guess is off by one step at most, and the comparisons decide
    const int bits = __float_as_int(amax * 0.14285715f);
    int b = (bits >> 20) - ((127 - 18) << 3);                   // exponent and three mantissa bits, rounded down
    b = max(0, min(255, b));
    if (7.f * scale_float(b) < amax && b < 255) ++b;
    if (7.f * scale_float(b) < amax && b < 255) ++b;
    if (b > 0 && 7.f * scale_float(b - 1) >= amax) --b;
    return (uint32_t)b;
}

// x / scale, to nearest, ties to even, within -7 .. 7; offset by 8
__device__ __forceinline__ uint32_t code_of(float x, float scale, float inv)
{
    const float ax = fabsf(x);
    float n = rintf(fminf(ax * inv, 8.f));
    const float rest = fmaf(-n, scale, ax), half = 0.5f * scale;
    const bool odd = ((int)n & 1) != 0;
    if (rest > half || (rest == half && odd)) n += 1.f;
    else if (rest < -half || (rest == -half && odd)) n -= 1.f;
    n = fminf(n, 7.f);
    return (uint32_t)(8 + (int)copysignf(n, x));
}

template <typename T> __device__ __forceinline__ void load8(const T *p, float (&x)[8]);
template <> __device__ __forceinline__ void load8<float>(const float *p, float (&x)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16 *p, float (&x)[8])
{
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}

// the row of the cache that row i stands for, or -1 where there is none (skipped, or out of range: status)
__device__ __forceinline__ int64_t cache_row(const QuantRows &p, int64_t i)
{
    const int64_t at = p.at ? (int64_t)ld_int(p.at + i) : i;
    if (at >= p.n_caches * p.cap) {
        if ((threadIdx.x & 31) == 0) atomicMax(p.status, (int32_t)FEDATTN_ERR_INDEX);
        return -1;
    }
    return at;
}

template <typename T, int kD>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const __grid_constant__ QuantRows p)
{
    constexpr int kVecs = kD / 8;                               // lanes of a head
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    grid_wait();                                                // nothing is read or written before
    if (unit >= 2 * p.n_rows) return;
    const int64_t row = unit >> 1;
    const bool is_v = unit & 1;
    const int64_t at = cache_row(p, row);
    if (at < 0) return;
    const int64_t cache = at / p.cap, within = at - cache * p.cap;
    const T *src = static_cast<const T *>(is_v ? p.v : p.k) + row * (is_v ? p.v_stride : p.k_stride);
    uint8_t *codes = is_v ? p.v_codes : p.k_codes, *scales = is_v ? p.v_scales : p.k_scales;
    const int n = p.hkv * kVecs;
#pragma unroll 4
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane, h = i / kVecs, c = (i - h * kVecs) * 8;
        float x[8], amax = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (i < n) load8(src + (int64_t)h * kD + c, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const uint32_t b = scale_byte(amax);
        const float scale = scale_float(b), inv = 1.f / scale;
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= code_of(x[e], scale, inv) << (4 * e);
        if (i < n) {
            const int64_t r = (cache * p.hkv + h) * p.cap + within;
            *reinterpret_cast<uint32_t *>(codes + r * (kD / 2) + c / 2) = w;
            if ((i & 3) == 0) scales[r * (kD / kQuantGroup) + c / kQuantGroup] = (uint8_t)b;
        }
    }
}

template <typename T> __device__ __forceinline__ void store8(T *p, const uint32_t (&pair)[4]);       // pair[i]: channels i, i + 4
template <> __device__ __forceinline__ void store8<float>(float *p, const uint32_t (&pair)[4])
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(pair[i] << 16); x[i + 4] = __uint_as_float(pair[i] & 0xffff0000u); }
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16 *p, const uint32_t (&pair)[4])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(__byte_perm(pair[0], pair[1], 0x5410), __byte_perm(pair[2], pair[3], 0x5410),
                                               __byte_perm(pair[0], pair[1], 0x7632), __byte_perm(pair[2], pair[3], 0x7632));
}

template <typename T, int kD>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const __grid_constant__ QuantRows p)
{
    constexpr int kVecs = kD / 8;
    const int lane = threadIdx.x & 31;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    grid_wait();                                                // nothing is read or written before
    if (unit >= 2 * p.n_rows) return;
    const int64_t row = unit >> 1;
    const bool is_v = unit & 1;
    const int64_t at = cache_row(p, row);
    if (at < 0) return;
    const int64_t cache = at / p.cap, within = at - cache * p.cap;
    T *dst = static_cast<T *>(is_v ? p.v_out : p.k_out) + row * p.hkv * kD;
    const uint8_t *codes = is_v ? p.v_codes : p.k_codes, *scales = is_v ? p.v_scales : p.k_scales;
    const int n = p.hkv * kVecs;
#pragma unroll 4
    for (int i = lane; i < n; i += 32) {
        const int h = i / kVecs, c = (i - h * kVecs) * 8;
        const int64_t r = (cache * p.hkv + h) * p.cap + within;
        const uint32_t w = *reinterpret_cast<const uint32_t *>(codes + r * (kD / 2) + c / 2);
        const uint32_t s = scale_pair(scales[r * (kD / kQuantGroup) + c / kQuantGroup] * 0x10001u), off = offset_pair(s);
        const uint32_t pair[4] = {nibble_pair<0>(w, s, off), nibble_pair<1>(w, s, off), nibble_pair<2>(w, s, off), nibble_pair<3>(w, s, off)};
        store8(dst + (int64_t)h * kD + c, pair);
    }
}

template <typename T>
void (*rows_kernel(int d, bool back))(const QuantRows)
{
    switch (d) {
    case 32: return back ? dequantize_kernel<T, 32> : quantize_kernel<T, 32>;
    case 64: return back ? dequantize_kernel<T, 64> : quantize_kernel<T, 64>;
    case 96: return back ? dequantize_kernel<T, 96> : quantize_kernel<T, 96>;
    default: return back ? dequantize_kernel<T, 128> : quantize_kernel<T, 128>;
    }
}

}  // namespace

cudaError_t launch_quant_rows(const QuantRows &p, bool back, int dtype, int d, cudaStream_t s, int64_t *launches)
{
    const int64_t blocks = (2 * p.n_rows + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    WaitFirstLaunch l(dim3((unsigned)blocks), dim3(kThreads), 0, s);
    const cudaError_t e = cudaLaunchKernelEx(&l.cfg, dtype == FEDATTN_BF16 ? rows_kernel<__nv_bfloat16>(d, back) : rows_kernel<float>(d, back), p);
    ++*launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace fedattn
