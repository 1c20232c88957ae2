// Queries and keys as the attention calls take them: every head's RMS norm and the rotation by the token's position.
//     y_c = x_c w_c / sqrt(mean_c x_c^2 + eps);   channels (i, i + r/2) or (2 i, 2 i + 1) turned by pos * f_i, i < r/2.
// Bound by memory: a row is read once and written once, 8 flop per element.  A lane holds both members of its pairs: two units of 16
// bytes (8 bf16 or 4 fp32 channels), one from either half of the rotated channels, or neighbours where pairs are neighbours; so a
// head of 128 bf16 channels is 8 lanes, the sum of squares three shuffles, and nothing else is exchanged.  (Units of 4 bf16 channels serve
// the sizes that 8 do not divide.)  A warp takes several heads of one row: the sines and cosines depend on the row only, are computed by
// all lanes together and are multiplied by the weights once per row: per element two FMAs and the factor of its head are left.
//
// The angle.  pos * f would lose in fp32 what matters (position 10^6 leaves 0.06 rad).  f is a fixed-point fraction of a turn with
// 64 bits instead; pos times that, modulo 2^64, is the fraction of a turn exactly, for any int32 position, and only what is
// left of an eighth of a turn becomes a float: 2^-28 turns at most.
#include "common.cuh"

namespace fedattn {

namespace {

// kUnit channels as they lie in memory
template <typename T, int kUnit> struct Unit;
template <> struct Unit<float, 4> {
    float4 v;
    __device__ void zero() { v = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ void load(const float *p) { v = *reinterpret_cast<const float4 *>(p); }
    __device__ void get(float *x) const { x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    static __device__ void store(float *p, const float *x) { *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]); }
};
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <> struct Unit<__nv_bfloat16, 4> {
    uint2 v;
    __device__ void zero() { v = make_uint2(0, 0); }
    __device__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint2 *>(p); }
    __device__ void get(float *x) const
    {
        x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
        x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    static __device__ void store(__nv_bfloat16 *p, const float *x)
    {
        *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    }
};
template <> struct Unit<__nv_bfloat16, 8> {
    uint4 v;
    __device__ void zero() { v = make_uint4(0, 0, 0, 0); }
    __device__ void load(const __nv_bfloat16 *p) { v = *reinterpret_cast<const uint4 *>(p); }
    __device__ void get(float *x) const
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ void store(__nv_bfloat16 *p, const float *x)
    {
        *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
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

__device__ __forceinline__ uint64_t pack2(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// One lane's share of a head.  kLanes: lanes of a head.
template <typename T, int kUnit, int kLanes, bool kInterleaved> struct Lane {
    static constexpr int kGroups = 32 / kLanes;                 // heads a warp holds at a time
    typedef Unit<T, kUnit> U;
    int s, grp, c0, c1;
    bool turned, mine;
    float inv_d, eps;
    // The lane groups hold the same channels of different heads and share the work on sines and cosines.
    static constexpr int kMine = kUnit > kGroups ? kUnit / kGroups : 1, kSharers = kUnit / kMine;
    uint64_t freq[kMine];
    float sn[kUnit], cs[kUnit];
    // pairs (i, i + 1) of x' = x xx + y xy, y' = y yy + x yx, times the head's factor
    uint64_t xx[kUnit / 2], xy[kUnit / 2], yy[kUnit / 2], yx[kUnit / 2];

    // Units at c0 and c1.  Behind the rotated channels they are neighbours, turned by nothing.
    __device__ explicit Lane(const RopeParams &p)
    {
        const int lane = threadIdx.x & 31;
        s = lane & (kLanes - 1);
        grp = lane / kLanes;
        turned = 2 * kUnit * s < p.rot;
        mine = 2 * kUnit * s < p.d;
        const bool split = turned && !kInterleaved;
        c0 = split ? kUnit * s : 2 * kUnit * s;
        c1 = split ? c0 + (p.rot >> 1) : c0 + kUnit;
        inv_d = 1.f / (float)p.d;
        eps = p.eps;
#pragma unroll
        for (int i = 0; i < kMine; ++i) freq[i] = p.freq[turned ? kUnit * s + i * kSharers + grp % kSharers : 0];
    }
    // Pair i of the lane is (x[i], y[i]).
    __device__ void pairs(const U &a, const U &b, float (&x)[kUnit], float (&y)[kUnit]) const
    {
        float t[2 * kUnit];
        a.get(t);
        b.get(t + kUnit);
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            x[i] = kInterleaved ? t[2 * i] : t[i];
            y[i] = kInterleaved ? t[2 * i + 1] : t[kUnit + i];
        }
    }
    // sines and cosines of a row
    __device__ void turn_to(int64_t pos)
    {
        float sv[kMine], cv[kMine];
#pragma unroll
        for (int i = 0; i < kMine; ++i) turn_sincos((uint64_t)pos * freq[i], sv[i], cv[i]);
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            const int from = (i % kSharers) * kLanes + s;
            sn[i] = __shfl_sync(0xffffffffu, sv[i / kSharers], from);
            cs[i] = __shfl_sync(0xffffffffu, cv[i / kSharers], from);
            if (!turned) { sn[i] = 0.f; cs[i] = 1.f; }
        }
    }
    __device__ void load_weights(const void *w, U &a, U &b) const
    {
        a.zero();
        b.zero();
        if (w && mine) {
            a.load(static_cast<const T *>(w) + c0);
            b.load(static_cast<const T *>(w) + c1);
        }
    }
    __device__ void weigh(const void *w, const U &a, const U &b)
    {
        float wx[kUnit], wy[kUnit];
        pairs(a, b, wx, wy);
#pragma unroll
        for (int i = 0; i < kUnit; ++i)
            if (!w) wx[i] = wy[i] = 1.f;
#pragma unroll
        for (int i = 0; i < kUnit; i += 2) {
            xx[i / 2] = pack2(wx[i] * cs[i], wx[i + 1] * cs[i + 1]);
            xy[i / 2] = pack2(-wy[i] * sn[i], -wy[i + 1] * sn[i + 1]);
            yy[i / 2] = pack2(wy[i] * cs[i], wy[i + 1] * cs[i + 1]);
            yx[i / 2] = pack2(wx[i] * sn[i], wx[i + 1] * sn[i + 1]);
        }
    }
    // one head per lane group (every lane of the warp calls it)
    __device__ void head(const U &a, const U &b, T *dst, bool store) const
    {
        float x[kUnit], y[kUnit];
        pairs(a, b, x, y);
        uint64_t x2[kUnit / 2], y2[kUnit / 2], sum = 0;
#pragma unroll
        for (int i = 0; i < kUnit / 2; ++i) {
            x2[i] = pack2(x[2 * i], x[2 * i + 1]);
            y2[i] = pack2(y[2 * i], y[2 * i + 1]);
            sum = fma2(y2[i], y2[i], fma2(x2[i], x2[i], sum));
        }
        const float2 part = unpack2(sum);
        float ss = part.x + part.y;
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        // 1 / sqrt with a Newton step behind the approximation
        const float v = fmaf(ss, inv_d, eps), r0 = rsqrtf(v), r = r0 * fmaf(-0.5f * v * r0, r0, 1.5f);
        const uint64_t r2 = pack2(r, r);
        float o[2 * kUnit];
#pragma unroll
        for (int i = 0; i < kUnit / 2; ++i) {
            const float2 xo = unpack2(mul2(fma2(x2[i], xx[i], mul2(y2[i], xy[i])), r2));
            const float2 yo = unpack2(mul2(fma2(y2[i], yy[i], mul2(x2[i], yx[i])), r2));
            o[kInterleaved ? 4 * i : 2 * i] = xo.x;
            o[kInterleaved ? 4 * i + 2 : 2 * i + 1] = xo.y;
            o[kInterleaved ? 4 * i + 1 : kUnit + 2 * i] = yo.x;
            o[kInterleaved ? 4 * i + 3 : kUnit + 2 * i + 1] = yo.y;
        }
        if (store) {
            U::store(dst + c0, o);
            U::store(dst + c1, o + kUnit);
        }
    }
};

constexpr int kThreads = 128;

// Few rows: a unit of work is a row and `per` of its heads (queries first, then keys), taken by one warp.
template <typename T, int kUnit, int kLanes, bool kInterleaved>
__global__ void __launch_bounds__(kThreads)
qk_norm_rope_kernel(const __grid_constant__ RopeParams p, int per, int n_chunks, int64_t n_units)
{
    typedef Lane<T, kUnit, kLanes, kInterleaved> L;
    typedef typename L::U U;
    constexpr int kBatch = 16 / kUnit;                          // heads of a lane group whose loads are in flight together
    const int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    grid_wait();                                                // nothing is read or written before
    if (unit >= n_units) return;
    const int64_t row = n_chunks == 1 ? unit : unit / n_chunks;
    const int h_lo = (int)(unit - row * n_chunks) * per, h_hi = min(h_lo + per, p.hq + p.hkv), d = p.d;
    L me(p);
    me.turn_to(p.pos ? (int64_t)ld_int(p.pos + row) : row);
#pragma unroll 1
    for (int is_k = 0; is_k < 2; ++is_k) {
        const int lo = is_k ? max(0, h_lo - p.hq) : h_lo, hi = is_k ? h_hi - p.hq : min(h_hi, p.hq);
        if (lo >= hi) continue;
        const T *src = is_k ? static_cast<const T *>(p.k) + row * p.k_stride : static_cast<const T *>(p.q) + row * p.q_stride;
        T *dst = is_k ? static_cast<T *>(p.ko) + row * p.hkv * d : static_cast<T *>(p.qo) + row * p.hq * d;
        U wa, wb;
        me.load_weights(is_k ? p.wk : p.wq, wa, wb);
        me.weigh(is_k ? p.wk : p.wq, wa, wb);
#pragma unroll 1
        for (int h0 = lo; h0 < hi; h0 += kBatch * L::kGroups) {
            U a[kBatch], b[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int h = h0 + u * L::kGroups + me.grp;
                a[u].zero();
                b[u].zero();
                if (h < hi && me.mine) {
                    a[u].load(src + h * d + me.c0);
                    b[u].load(src + h * d + me.c1);
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int h = h0 + u * L::kGroups + me.grp;
                me.head(a[u], b[u], dst + h * d, h < hi && me.mine);
            }
        }
    }
}

// Many rows: a warp walks rows and keeps the next ones on their way into a ring of its own in shared memory (asynchronous copies), so
// that what is in flight does not depend on registers: 16 warps of an SM held 32 KB in registers, 8 hold 80 KB here.  A CTA is one warp: as
// many as the rings leave room for.  (13 633 rows of 32 + 8 heads of 128 channels, 279 MB, 42.7 us at the copy rate: loads to registers 58.7 us;
// rings in CTAs of four warps 51.7, of two 50.8, of one 49.3 = 5.66 TB/s, with three stages 56.8.)
constexpr int kRingThreads = 32;
constexpr int kRingStages = 2;
template <typename T, int kUnit, int kLanes, bool kInterleaved>
__global__ void __launch_bounds__(kRingThreads)
qk_norm_rope_ring_kernel(const __grid_constant__ RopeParams p, int stage_bytes)
{
    typedef Lane<T, kUnit, kLanes, kInterleaved> L;
    typedef typename L::U U;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, d = p.d;
    const int64_t first = (int64_t)blockIdx.x * (kRingThreads / 32) + warp, step = (int64_t)gridDim.x * (kRingThreads / 32);
    uint8_t *ring = smem + (size_t)warp * kRingStages * stage_bytes;
    const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    const int q_bytes = p.hq * d * (int)sizeof(T);
    grid_wait();                                                // nothing is read or written before
    auto load_row = [&](int64_t row, int stage) {
        if (row < p.n_rows) {
            const uint8_t *q = reinterpret_cast<const uint8_t *>(static_cast<const T *>(p.q) + row * p.q_stride);
            const uint8_t *k = reinterpret_cast<const uint8_t *>(static_cast<const T *>(p.k) + row * p.k_stride) - q_bytes;
            const uint32_t dst = ring_s + stage * stage_bytes;
#pragma unroll 4
            for (int i = lane * 16; i < stage_bytes; i += 512)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + i - lane * 16), "l"((i < q_bytes ? q : k) + i) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kRingStages; ++i) load_row(first + i * step, i);
    L me(p);
    U w[4];
    me.load_weights(p.wq, w[0], w[1]);
    me.load_weights(p.wk, w[2], w[3]);
    int stage = 0;
    auto pos_of = [&](int64_t row) -> int64_t { return p.pos && row < p.n_rows ? (int64_t)ld_int(p.pos + row) : row; };
    int64_t next_pos = pos_of(first);
#pragma unroll 1
    for (int64_t row = first; row < p.n_rows; row += step) {
        const int64_t pos = next_pos;
        next_pos = pos_of(row + step);
        me.turn_to(pos);
        asm volatile("cp.async.wait_group %0;" ::"n"(kRingStages - 1) : "memory");
        __syncwarp();
        const T *src = reinterpret_cast<const T *>(ring + stage * stage_bytes);
#pragma unroll 1
        for (int is_k = 0; is_k < 2; ++is_k) {
            const int n = is_k ? p.hkv : p.hq;
            T *dst = is_k ? static_cast<T *>(p.ko) + row * p.hkv * d : static_cast<T *>(p.qo) + row * p.hq * d;
            if (is_k) me.weigh(p.wk, w[2], w[3]);
            else me.weigh(p.wq, w[0], w[1]);
#pragma unroll 2
            for (int h0 = 0; h0 < n; h0 += L::kGroups) {
                const int h = h0 + me.grp;
                const bool have = h < n && me.mine;
                U a, b;
                a.zero();
                b.zero();
                if (have) {
                    a.load(src + h * d + me.c0);
                    b.load(src + h * d + me.c1);
                }
                me.head(a, b, dst + h * d, have);
            }
            src += p.hq * d;
        }
        __syncwarp();                                           // every lane has read the stage
        load_row(row + kRingStages * step, stage);
        stage = stage + 1 == kRingStages ? 0 : stage + 1;
    }
}

typedef void (*Kernel)(const RopeParams, int, int, int64_t);
typedef void (*RingKernel)(const RopeParams, int);
struct Form {
    Kernel few;
    RingKernel many;
    int groups;                                                 // heads a warp holds at a time
};
template <typename T, int kUnit, int kLanes> Form form_of(bool interleaved)
{
    return interleaved ? Form{qk_norm_rope_kernel<T, kUnit, kLanes, true>, qk_norm_rope_ring_kernel<T, kUnit, kLanes, true>, 32 / kLanes}
                       : Form{qk_norm_rope_kernel<T, kUnit, kLanes, false>, qk_norm_rope_ring_kernel<T, kUnit, kLanes, false>, 32 / kLanes};
}

constexpr int kRingMost = 24 * 1024;                            // bytes of a row in a ring: an SM holds the rings of four warps

}  // namespace

cudaError_t launch_qk_norm_rope(const RopeParams &p, int dtype, int device, int sm_count, cudaStream_t s, int64_t *launches)
{
    typedef __nv_bfloat16 bf;
    const bool il = p.interleaved != 0, wide = p.d % 16 == 0 && p.rot % 16 == 0;
    const int type = dtype != FEDATTN_BF16 ? 0 : (wide ? 2 : 1), which = 2 * type + (p.d > 64);
    static Form (*const forms[6])(bool) = {form_of<float, 4, 8>, form_of<float, 4, 16>, form_of<bf, 4, 8>, form_of<bf, 4, 16>, form_of<bf, 8, 4>, form_of<bf, 8, 8>};
    const Form f = forms[which](il);
    const int n_heads = p.hq + p.hkv;
    const int64_t row_bytes = (int64_t)n_heads * p.d * (dtype == FEDATTN_BF16 ? 2 : 4);
    // The rings, when every warp that they leave room for gets two rows.
    const int64_t ring_bytes = row_bytes * kRingStages * (kRingThreads / 32);
    const int most = 16 * 32 / kRingThreads, fit = ring_bytes > 0 ? (int)(225 * 1024 / (ring_bytes + 1024)) : 0, ctas = fit < most ? fit : most;
    if (row_bytes <= kRingMost && ctas >= 1 && p.n_rows >= (int64_t)sm_count * ctas * (kRingThreads / 32) * 2) {
        static bool attr_set[64][6][2] = {};
        bool &set = attr_set[device & 63][which][il];
        if (!set) {
            const cudaError_t e = cudaFuncSetAttribute(f.many, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingMost * kRingStages * (kRingThreads / 32));
            if (e != cudaSuccess) return e;
            set = true;
        }
        WaitFirstLaunch l(dim3((unsigned)(sm_count * ctas)), dim3(kRingThreads), (size_t)ring_bytes, s);
        const cudaError_t e = cudaLaunchKernelEx(&l.cfg, f.many, p, (int)row_bytes);
        ++*launches;
        return e != cudaSuccess ? e : cudaGetLastError();
    }
    // A warp takes fewer heads of a row (what it holds at a time at the least) while the warps do not fill the GPU.
    int per = (n_heads + f.groups - 1) / f.groups * f.groups;
    while (per > f.groups && p.n_rows * ((n_heads + per - 1) / per) < (int64_t)sm_count * 16) per = (per / 2 + f.groups - 1) / f.groups * f.groups;
    const int n_chunks = (n_heads + per - 1) / per;
    const int64_t units = p.n_rows * n_chunks, blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    WaitFirstLaunch l(dim3((unsigned)blocks), dim3(kThreads), 0, s);
    const cudaError_t e = cudaLaunchKernelEx(&l.cfg, f.few, p, per, n_chunks, units);
    ++*launches;
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace fedattn
