// Queries and keys as the attention calls take them: every head's RMS norm and the rotation by the token's position.
//     y_c = x_c w_c / sqrt(mean_c x_c^2 + eps);   channels (i, i + r/2) or (2 i, 2 i + 1) turned by pos * f_i, i < r/2.
// Bound by memory: a row is read once and written once, 8 flop per element.  A head is held by 16 lanes (8 up to 64 channels),
// four channels of either half of the rotation per lane: both members of a pair are in one lane, and the sum of squares takes
// 3 or 4 shuffles.  A warp takes several heads of one row, because the sines and cosines depend on the row only.
//
// The angle.  pos * f would lose in fp32 what matters (position 10^6 leaves 0.06 rad).  f is a fixed-point fraction of a turn with
// 64 bits instead; pos times that, modulo 2^64, is the fraction of a turn exactly, for any int32 position, and only what is
// left of an eighth of a turn becomes a float: 2^-28 turns at most.
#include "common.cuh"

namespace fedattn {

namespace {

// four channels
template <typename T> struct Vec4;
template <> struct Vec4<float> {
    float4 v;
    __device__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ void load(const float *p) { v = *reinterpret_cast<const float4 *>(p); }
    __device__ void get(float (&x)[4]) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    static __device__ void store(float *p, const float (&x)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
template <> struct Vec4<__nv_bfloat16> {
    uint2 v;
    __device__ void zero() { v = make_uint2(0, 0); }
    __device__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint2 *>(p); }
    __device__ void get(float (&x)[4]) const
    {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    static __device__ void store(__nv_bfloat16 *p, const float (&x)[4])
    {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(x[0], x[1]), hi = __floats2bfloat162_rn(x[2], x[3]);
        *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
    }
};

// sine and cosine of a fraction of a turn with 64 bits
__device__ __forceinline__ void turn_sincos(uint64_t turn, float &sn, float &cs)
{
    const uint64_t near = turn + (1ull << 61);                  // quarter turns, rounded
    const int quarter = (int)(near >> 62);
    const int64_t rest = (int64_t)(near & ((1ull << 62) - 1)) - (int64_t)(1ull << 61);
    float s, c;
    sincospif((float)rest * 0x1p-63f, &s, &c);                  // half turns
    const float a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
    sn = quarter & 2 ? -a : a;
    cs = (quarter + 1) & 2 ? -b : b;
}

constexpr int kThreads = 128;
constexpr int kBatch = 4;                                       // heads per lane group whose loads are in flight together

// A unit is a row and `per` of its heads (queries first, then keys), taken by one warp.
template <typename T, int kLanes>
__global__ void __launch_bounds__(kThreads)
qk_norm_rope_kernel(const __grid_constant__ RopeParams p, int per, int n_chunks, int64_t n_units)
{
    constexpr int kGroups = 32 / kLanes;                        // heads a warp holds at a time
    const int lane = threadIdx.x & 31, s = lane & (kLanes - 1), grp = lane / kLanes;
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    grid_wait();                                                // nothing is read or written before
    if (unit >= n_units) return;
    const int64_t row = n_chunks == 1 ? unit : unit / n_chunks;
    const int h_lo = (int)(unit - row * n_chunks) * per, n_heads = p.hq + p.hkv, h_hi = min(h_lo + per, n_heads);

    // This lane's channels: a pair of units of four.  Half-split rotation: s and s + r/8; interleaved, and behind the
    // rotated channels, two neighbouring units.
    const int d = p.d, half_units = p.rot >> 3;
    const bool turned = s < half_units, mine = s < (d >> 3);
    const bool split = turned && !p.interleaved;
    const int c0 = split ? 4 * s : 8 * s, c1 = split ? 4 * s + 4 * half_units : 8 * s + 4;
    float wq[8], wk[8], sn[4], cs[4];
#pragma unroll
    for (int i = 0; i < 8; ++i) wq[i] = wk[i] = 1.f;
    auto load_w = [&](const void *w, float (&x)[8]) {
        if (!w || !mine) return;
        Vec4<T> a, b;
        a.load(static_cast<const T *>(w) + c0);
        b.load(static_cast<const T *>(w) + c1);
        float t[4];
        a.get(t);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = t[i];
        b.get(t);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 + i] = t[i];
    };
    load_w(p.wq, wq);
    load_w(p.wk, wk);
    // Frequencies 4 s .. 4 s + 3: the lane groups hold the same channels of different heads and share the work.
    {
        const int64_t pos = p.pos ? (int64_t)ld_int(p.pos + row) : row;
        float sv[4 / kGroups], cv[4 / kGroups];
#pragma unroll
        for (int i = 0; i < 4 / kGroups; ++i) turn_sincos((uint64_t)pos * p.freq[turned ? 4 * s + i * kGroups + grp : 0], sv[i], cv[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int from = (i & (kGroups - 1)) * kLanes + s;
            sn[i] = __shfl_sync(0xffffffffu, sv[i / kGroups], from);
            cs[i] = __shfl_sync(0xffffffffu, cv[i / kGroups], from);
            if (!turned) { sn[i] = 0.f; cs[i] = 1.f; }
        }
    }
    const T *q = static_cast<const T *>(p.q) + row * p.q_stride, *k = static_cast<const T *>(p.k) + row * p.k_stride;
    T *qo = static_cast<T *>(p.qo) + row * p.hq * d, *ko = static_cast<T *>(p.ko) + row * p.hkv * d;
    const float inv_d = 1.f / (float)d;
#pragma unroll 1
    for (int h0 = h_lo; h0 < h_hi; h0 += kBatch * kGroups) {
        Vec4<T> a[kBatch], b[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int h = h0 + u * kGroups + grp;
            a[u].zero();
            b[u].zero();
            if (h < h_hi && mine) {
                const T *x = h < p.hq ? q + h * d : k + (h - p.hq) * d;
                a[u].load(x + c0);
                b[u].load(x + c1);
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int h = h0 + u * kGroups + grp;
            float x[4], y[4], ss = 0.f;
            a[u].get(x);
            b[u].get(y);
#pragma unroll
            for (int i = 0; i < 4; ++i) ss = fmaf(x[i], x[i], fmaf(y[i], y[i], ss));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float r = 1.f / sqrtf(fmaf(ss, inv_d, p.eps));
            const bool is_q = h < p.hq;
            float xo[4], yo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] *= r * (is_q ? wq[i] : wk[i]);
                y[i] *= r * (is_q ? wq[4 + i] : wk[4 + i]);
            }
            if (!p.interleaved) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    xo[i] = x[i] * cs[i] - y[i] * sn[i];
                    yo[i] = y[i] * cs[i] + x[i] * sn[i];
                }
            } else {                                            // pairs 4 s .. 4 s + 3: two in either unit
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    xo[2 * i] = x[2 * i] * cs[i] - x[2 * i + 1] * sn[i];
                    xo[2 * i + 1] = x[2 * i + 1] * cs[i] + x[2 * i] * sn[i];
                    yo[2 * i] = y[2 * i] * cs[2 + i] - y[2 * i + 1] * sn[2 + i];
                    yo[2 * i + 1] = y[2 * i + 1] * cs[2 + i] + y[2 * i] * sn[2 + i];
                }
            }
            if (h < h_hi && mine) {
                T *dst = is_q ? qo + h * d : ko + (h - p.hq) * d;
                Vec4<T>::store(dst + c0, xo);
                Vec4<T>::store(dst + c1, yo);
            }
        }
    }
}

template <typename T, int kLanes>
cudaError_t launch(const RopeParams &p, int sm_count, cudaStream_t s)
{
    constexpr int kGroups = 32 / kLanes, kStep = kBatch * kGroups;
    const int n_heads = p.hq + p.hkv;
    // A warp takes all heads of a row when the rows alone fill the GPU, fewer (one lane group's each at the least) when not.
    int per = (n_heads + kStep - 1) / kStep * kStep;
    while (per > kGroups && p.n_rows * ((n_heads + per - 1) / per) < (int64_t)sm_count * 16) per = (per / 2 + kGroups - 1) / kGroups * kGroups;
    const int n_chunks = (n_heads + per - 1) / per;
    const int64_t units = p.n_rows * n_chunks, blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    WaitFirstLaunch l(dim3((unsigned)blocks), dim3(kThreads), 0, s);
    return cudaLaunchKernelEx(&l.cfg, qk_norm_rope_kernel<T, kLanes>, p, per, n_chunks, units);
}

}  // namespace

cudaError_t launch_qk_norm_rope(const RopeParams &p, int dtype, int sm_count, cudaStream_t s, int64_t *launches)
{
    typedef __nv_bfloat16 bf;
    cudaError_t e;
    if (p.d <= 64) e = dtype == FEDATTN_BF16 ? launch<bf, 8>(p, sm_count, s) : launch<float, 8>(p, sm_count, s);
    else e = dtype == FEDATTN_BF16 ? launch<bf, 16>(p, sm_count, s) : launch<float, 16>(p, sm_count, s);
    ++*launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace fedattn
