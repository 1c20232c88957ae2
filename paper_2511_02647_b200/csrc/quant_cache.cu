// Rows of keys and values into the 4-bit cache and back (quant_cache.cuh has the format).  Bound by memory: 4.25 bits per element
// on one side, the storage type on the other.
//
// Scale of a group: the least of the 256 whose sevenfold reaches the group's largest magnitude.  Code: x / scale to the nearest
// integer, ties to the even one, -7 .. 7.  Both are exact decisions, although the quotients are not.  scale = m * 2^e with 8 <= m <= 15.
//   bf16: x is at most 255 times a power of two, so x / scale lies on a tie or at least 1 / 960 away from it (twice the quotient is a
//   fraction over m * 2^5 at the most where it is near an odd number), and amax / 7 on a scale or 2^-9 of itself away.  Rounding the
//   product with 1 / scale to a multiple of 2^-13 first puts it on the tie when it belongs there.
//   fp32: comparisons put right what the approximate quotient gets wrong: 7 * scale and code * scale are exact in fp32 (7 and 8
//   significant bits), and so is x minus the latter near a tie.
//
// A warp takes the same head of neighbouring rows at a time (2 of 128 channels), so that what it writes to the cache is one run of 128
// bytes when the rows are neighbours there; a lane has 8 channels, four lanes a group.
#include "quant_cache.cuh"

namespace fedattn {

namespace {

constexpr int kThreads = 256;
// Heads of a warp, whose loads are in flight together.  (8192 rows of 8 heads of 128 channels in and out, two launches: 1 28.7 us, 2 21.4, 4 19.5,
// 8 20.7; 85 MB, 13 us at the copy rate.)
constexpr int kBatch = 4;

// the least scale byte with 7 * scale >= amax (255 when none has)
template <typename T> __device__ __forceinline__ uint32_t scale_byte(float amax)
{
    // 1/7 rounded down, so that a product that should be a scale does not pass it; then up to four significant bits
    const int bits = __float_as_int(amax * __int_as_float(0x3e124924));
    int b = ((bits + 0xfffff) >> 20) - ((127 - 18) << 3);
    b = max(0, min(255, b));
    if (sizeof(T) == 4 && 7.f * scale_float(b) < amax && b < 255) ++b;
    return (uint32_t)b;
}

// eight codes, offset by 8, as nibbles
template <typename T> __device__ __forceinline__ uint32_t codes_of(float (&x)[8], float scale, bool saturated);
template <> __device__ __forceinline__ uint32_t codes_of<__nv_bfloat16>(float (&x)[8], float scale, bool saturated)
{
    if (saturated)
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fminf(fmaxf(x[e], -7.f * scale), 7.f * scale);
    // (1 / scale to 2 units of the last place: t is off by 4e-6 at the most, far less than half a step of the first rounding)
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale));
    uint64_t t[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // to a multiple of 2^-13, then to an integer, plus 8, in the low bits of the sum
        asm("{\n\t.reg .b64 x, c;\n\t"
            "mov.b64 x, {%1, %2};\n\tmov.b64 c, {%3, %3};\n\tmul.rn.f32x2 x, x, c;\n\t"
            "mov.b64 c, {%4, %4};\n\tadd.rn.f32x2 x, x, c;\n\tmov.b64 c, {%5, %5};\n\tadd.rn.f32x2 x, x, c;\n\t"
            "mov.b64 c, {%6, %6};\n\tadd.rn.f32x2 %0, x, c;\n\t}"
            : "=l"(t[i]) : "f"(x[2 * i]), "f"(x[2 * i + 1]), "f"(inv), "f"(1536.f), "f"(-1536.f), "f"(12582920.f));
    }
    // every sum's bits are 0x4b400000 + 8 + code: shifted and added without a mask, what the constants make is taken off at the end
    uint32_t w = 0;
#pragma unroll
    for (int i = 3; i >= 0; --i) w = (w * 16 + (uint32_t)(t[i] >> 32)) * 16 + (uint32_t)t[i];
    return w - 0x4b400000u * 0x11111111u;
}
template <> __device__ __forceinline__ uint32_t codes_of<float>(float (&x)[8], float scale, bool)
{
    const float inv = 1.f / scale, half = 0.5f * scale;
    uint32_t w = 0;
#pragma unroll
    for (int e = 7; e >= 0; --e) {
        const float ax = fabsf(x[e]);
        float n = rintf(fminf(ax * inv, 8.f));
        const float rest = fmaf(-n, scale, ax);
        const bool odd = ((int)n & 1) != 0;
        if (rest > half || (rest == half && odd)) n += 1.f;
        else if (rest < -half || (rest == -half && odd)) n -= 1.f;
        n = fminf(n, 7.f);
        w = w * 16 + (uint32_t)(8 + (int)copysignf(n, x[e]));
    }
    return w;
}

// the row of the caches that row i stands for, or -1 where there is none (skipped, or out of range: status).  (There are fewer than 2^31.)
__device__ __forceinline__ int cache_row(const QuantRows &p, int i)
{
    const int at = p.at ? ld_int(p.at + i) : i;
    if (at >= p.n_caches * p.cap) {
        atomicMax(p.status, (int32_t)FEDATTN_ERR_INDEX);
        return -1;
    }
    return at;
}

// What a lane works on: a row, and 8 channels of each of kBatch heads of K (even blockIdx.y) or V.
template <int kD> struct LaneWork {
    static constexpr int kVecs = kD / 8, kRows = 32 / kVecs;    // lanes of a head, rows of a warp
    int row, c, head0, vec;
    bool is_v, mine;
    __device__ explicit LaneWork(const QuantRows &p)
    {
        const int lane = threadIdx.x & 31, r = lane / kVecs;
        const int64_t first = ((int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5)) * kRows;
        vec = lane - r * kVecs;
        c = vec * 8;
        head0 = (int)(blockIdx.y >> 1) * kBatch;
        is_v = blockIdx.y & 1;
        mine = r < kRows && first + r < p.n_rows;
        row = mine ? (int)first + r : 0;
    }
    // flat row of head0 in the codes and scales
    __device__ int64_t place(const QuantRows &p, int at) const
    {
        const int cap = (int)p.cap, cache = at / cap;
        return ((int64_t)cache * p.hkv + head0) * cap + (at - cache * cap);
    }
};

template <typename T, int kD>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const __grid_constant__ QuantRows p)
{
    grid_wait();                                                // nothing is read or written before
    const LaneWork<kD> w(p);
    const int at = w.mine ? cache_row(p, w.row) : -1;
    const T *src = static_cast<const T *>(w.is_v ? p.v : p.k) + w.row * (w.is_v ? p.v_stride : p.k_stride) + (int64_t)w.head0 * kD + w.c;
    uint8_t *codes = w.is_v ? p.v_codes : p.k_codes, *scales = w.is_v ? p.v_scales : p.k_scales;
    Eight<T> raw[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        raw[u].zero();
        if (w.mine && w.head0 + u < p.hkv) raw[u].load(src + u * kD);
    }
    const int64_t r0 = at >= 0 ? w.place(p, at) : 0;
    codes += r0 * (kD / 2) + w.c / 2;
    scales += r0 * (kD / kQuantGroup) + w.c / kQuantGroup;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        float x[8], amax = 0.f;
        raw[u].get(x);
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        const uint32_t b = scale_byte<T>(amax);
        const uint32_t word = codes_of<T>(x, scale_float(b), b == 255);
        if (at >= 0 && w.head0 + u < p.hkv) {
            *reinterpret_cast<uint32_t *>(codes + u * p.cap * (kD / 2)) = word;
            if ((w.vec & 3) == 0) scales[u * p.cap * (kD / kQuantGroup)] = (uint8_t)b;
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
    grid_wait();                                                // nothing is read or written before
    const LaneWork<kD> w(p);
    const int at = w.mine ? cache_row(p, w.row) : -1;
    if (at < 0) return;
    T *dst = static_cast<T *>(w.is_v ? p.v_out : p.k_out) + ((int64_t)w.row * p.hkv + w.head0) * kD + w.c;
    const int64_t r0 = w.place(p, at);
    const uint8_t *codes = (w.is_v ? p.v_codes : p.k_codes) + r0 * (kD / 2) + w.c / 2;
    const uint8_t *scales = (w.is_v ? p.v_scales : p.k_scales) + r0 * (kD / kQuantGroup) + w.c / kQuantGroup;
    uint32_t word[kBatch], byte[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        word[u] = byte[u] = 0;
        if (w.head0 + u < p.hkv) {
            word[u] = *reinterpret_cast<const uint32_t *>(codes + u * p.cap * (kD / 2));
            byte[u] = scales[u * p.cap * (kD / kQuantGroup)];
        }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
        const uint32_t s = scale_pair(byte[u]), off = offset_pair(s);
        const uint32_t pair[4] = {nibble_pair<0>(word[u], s, off), nibble_pair<1>(word[u], s, off), nibble_pair<2>(word[u], s, off),
                                  nibble_pair<3>(word[u], s, off)};
        if (w.head0 + u < p.hkv) store8(dst + u * kD, pair);
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
    const int rows = 32 / (d / 8) * (kThreads / 32);            // of a CTA
    const int64_t blocks = (p.n_rows + rows - 1) / rows, pieces = 2 * (((int64_t)p.hkv + kBatch - 1) / kBatch);
    if (pieces > 65535) return cudaErrorInvalidValue;           // grid
    WaitFirstLaunch l(dim3((unsigned)blocks, (unsigned)pieces), dim3(kThreads), 0, s);
    const cudaError_t e = cudaLaunchKernelEx(&l.cfg, dtype == FEDATTN_BF16 ? rows_kernel<__nv_bfloat16>(d, back) : rows_kernel<float>(d, back), p);
    ++*launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace fedattn
