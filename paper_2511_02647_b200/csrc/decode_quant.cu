// Decode over a cache held in 4 bits (quant_cache.cuh): one new query token per participant, local or shared caches, all
// keys or the first n_sink and the last `window`.  A key and value of 128 channels is 136 bytes.
//
// Bound by issue slots rather than by memory alone: at the copy rate an SM gets 46 elements per clock, and every eight of them take 11
// instructions to become bf16 (three shifts, four bit selections, four fma: quant_cache.cuh; nothing is rounded).  So everything else
// is kept off that path:
//   * Both products stand on their side, S^T = K Q^T and O^T = V^T P^T.  Keys and channels are the 16 rows of an mma.sync.m16n8k16, the
//     query rows that share a KV head its 8 columns: a group of 4 heads wastes half a tile, not three quarters, and takes half the
//     products and accumulators.
//   * The nibbles come out of a word in pairs (i, i + 4); which channel, or key, stands at which place of a sum is free, so Q and the keys
//     are placed to fit.  K: a lane's quarter of the row is one vector load, its nibbles are operand A as they come.  V: the halves of two keys'
//     words side by side (one byte permutation for eight elements) make the pairs that run along the keys.
//   * A warp has tiles of 32 keys of its own and its own ring of asynchronous copies: no barrier between warps during the walk.  Head-major
//     rows make every copy a run of consecutive bytes.
// The exponent reference of a row moves when its maximum has grown by more than 2^8 (one vote per tile).  fp32 queries go in as three bf16
// parts, and so do their weights (24 bits): six products for two.  bf16 calls round a weight to one bf16 behind its sum, at every head_dim: by 2^-8
// of it at most, like the output's own rounding, where the other bf16 calls below 128 channels keep 17 or 24 bits; a second part would take
// half as many products again in a kernel that issue slots bound.
//
// Up to 8 splits of a (cache, KV head) are one cluster and one launch; more are merged by a second kernel out of the workspace.
#include <cooperative_groups.h>
#include <string.h>

#include "quant_cache.cuh"

namespace fedattn {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kTileKeys = 32;
constexpr int kMaxSlots = 64;                                   // partials per output row in the workspace
constexpr int kMaxCluster = 8;
constexpr float kRescale = 8.f;                                 // log2 units

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// transposes an 8 x 8 matrix of 16-bit values that the warp holds, a pair per lane
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// the leading 8 bits of two values as a bf16 pair; what is left stays in them
__device__ __forceinline__ uint32_t take_part(float &lo, float &hi)
{
    const uint32_t a = __float_as_uint(lo), b = __float_as_uint(hi);
    lo -= __uint_as_float(a & 0xffff0000u);
    hi -= __uint_as_float(b & 0xffff0000u);
    return __byte_perm(a, b, 0x7632);
}
// partials, past L1 (volatile: behind the wait for the kernel that wrote them)
__device__ __forceinline__ float2 ld_partial2(const float *p)
{
    float2 v;
    asm volatile("ld.global.cg.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ float4 ld_partial4(const float *p)
{
    float4 v;
    asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v)
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

// T: type of q and o; kD: channels; kNT: column tiles of 8 query rows; kOneLaunch: the splits are a cluster.
template <typename T, int kD, int kNT> struct Layout {
    static constexpr int kParts = sizeof(T) == 4 ? 3 : 1;       // bf16 parts of queries and weights
    static constexpr int kW = kD / 32;                          // words of a lane's quarter of a key: 8 channels each
    static constexpr int kCodeRow = kD / 2, kScaleRow = kD / kQuantGroup;                 // bytes
    static constexpr int kCodeBytes = kTileKeys * kCodeRow, kScaleBytes = kTileKeys * kScaleRow;
    static constexpr int kStageBytes = 2 * (kCodeBytes + kScaleBytes);
    // (8 caches of 4096 rows, 32 / 8 heads: 9.4 us, 10.0 with four and 10.2 with two: what the ring leaves free seats the next call's CTAs)
    static constexpr int kStages = 3;
    static constexpr int kRing = kStages * kStageBytes;         // of a warp
    static constexpr int kQBytes = kParts * kNT * 8 * kD * 2;
    static constexpr int kPartialRow = kD + 4;                  // m, l, 2 pad, o
    static constexpr int kPartialBytes = kWarps * kNT * 8 * kPartialRow * 4;
    static constexpr int kRingBytes = kWarps * kRing > kPartialBytes ? kWarps * kRing : kPartialBytes;
    static constexpr int kBytes = kQBytes + kRingBytes;
    static constexpr bool kQInRegs = kNT * kParts <= 2;
};

// Registers: with two (three) CTAs per SM a CTA of the merge kernel still finds its 6144.  It has to: the next call's stream kernel is
// launched when all of those have started.  (243 registers, what 32 rows take without the limit: 8 participants over 32 768 rows 27.1 us, with
// 224 and 60 bytes spilled 19.9, 208 21.0.)
template <typename T, int kD, int kNT, bool kOneLaunch>
__global__ void __maxnreg__((kNT == 4 || sizeof(T) == 4 ? 224 : 152))
decode_quant_kernel(const __grid_constant__ QuantDecodeParams p, int n_splits, int n_chunks)
{
    using L = Layout<T, kD, kNT>;
    constexpr int kW = L::kW, kParts = L::kParts, kRows = 8 * kNT, kMt = kD / 16, kStages = L::kStages;
    extern __shared__ __align__(16) uint8_t smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = lane >> 2, t = lane & 3;
    // Inputs are read before the preceding grid of the stream is known to be complete unless they may be its outputs.
    if (!p.early) grid_wait();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int split = blockIdx.x, kvh = blockIdx.y;
    const int cache = blockIdx.z / n_chunks, chunk = blockIdx.z - cache * n_chunks;
    const int g = p.hq / p.hkv;
    const int rows_total = p.sync ? p.n_part * g : g;           // query rows that share this cache and KV head
    const int rows_here = min(kRows, rows_total - chunk * kRows);
    auto out_row = [&](int srow) -> int64_t {                   // stacked row -> row of q and o
        const int part = p.sync ? srow / g : cache, sub = p.sync ? srow - part * g : srow;
        return (int64_t)part * p.hq + kvh * g + sub;
    };

    // the rows of Q on their way while the length is: word x of row i / (kD / 8), i = tid + kThreads j
    constexpr int kQWords = kRows * (kD / 8), kQEach = (kQWords + kThreads - 1) / kThreads;
    Eight<T> raw[kQEach];
#pragma unroll
    for (int j = 0; j < kQEach; ++j) {
        const int i = tid + kThreads * j, row = i / (kD / 8);
        raw[j].zero();
        if (i < kQWords && row < rows_here) raw[j].load(static_cast<const T *>(p.q) + out_row(chunk * kRows + row) * kD + 8 * (i - row * (kD / 8)));
    }
    const CacheWalk<kTileKeys> walk(min(ld_int(p.kv_len + (p.sync ? 0 : cache)), p.max_kv_len), p.window, p.n_sink);
    const int per = (walk.n_tiles + n_splits - 1) / n_splits;
    const int tile_lo = min(split * per, walk.n_tiles), tile_hi = min(tile_lo + per, walk.n_tiles);
    const int64_t row0 = ((int64_t)cache * p.hkv + kvh) * p.cap;
    const uint8_t *kc = p.k_codes + row0 * L::kCodeRow, *ks = p.k_scales + row0 * L::kScaleRow;
    const uint8_t *vc = p.v_codes + row0 * L::kCodeRow, *vs = p.v_scales + row0 * L::kScaleRow;

    uint8_t *ring = smem + L::kQBytes + warp * L::kRing;
    // Pieces of 16 bytes.  Rows are copied up to the length, rounded up to 16 rows (the cache has them); what lies behind that in a tile is
    // whatever was there: finite, and masked.  128 channels: the pieces of rows 2, 3, 6, 7, .. of V change places in pairs, which
    // spreads the reads of rows t over the banks (row i / 4 of piece i: its bit 1 flips bit 1 of the piece).
    const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring) + lane * 16;
    const int v_shift = kD == 128 ? ((lane ^ ((lane >> 2) & 2)) - lane) * 16 : 0;
    const uint8_t *k_lane = kc + lane * 16, *v_lane = vc + lane * 16, *s_lane = (lane < 16 ? ks : vs) + (lane & 15) * 16;
    auto load_tile = [&](int tile, int stage) {
        const int key0 = walk.key0(tile), rows = (walk.len - key0 + 15) & ~15;
        const uint32_t dst = ring_s + stage * L::kStageBytes;
        const uint8_t *k_src = k_lane + (int64_t)key0 * L::kCodeRow, *v_src = v_lane + (int64_t)key0 * L::kCodeRow;
        constexpr int kPieces = L::kCodeBytes / 16, kRowPieces = L::kCodeRow / 16, kScalePieces = L::kScaleBytes / 16;
        const bool whole = rows >= kTileKeys;
#pragma unroll
        for (int i0 = 0; i0 < kPieces; i0 += 32)
            if (whole ? kPieces % 32 == 0 || i0 + lane < kPieces : i0 + lane < rows * kRowPieces) {
                cp_async16(dst + i0 * 16, k_src + i0 * 16);
                cp_async16(dst + L::kCodeBytes + i0 * 16 + v_shift, v_src + i0 * 16);
            }
        if ((lane & 15) < (whole ? kScalePieces : rows * L::kScaleRow / 16))
            cp_async16(dst + 2 * L::kCodeBytes + (lane >> 4) * (L::kScaleBytes - 256), s_lane + (int64_t)key0 * L::kScaleRow);
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
        if (tile_lo + warp + s * kWarps < tile_hi) load_tile(tile_lo + warp + s * kWarps, s);
        cp_async_commit();
    }

    // ---- Q as operand B: [part][column tile][step][lane] pairs of pairs ----
    // Step 2 w + h of a lane: word w of its quarter of the channels, nibble pairs 2 h and 2 h + 1 (nibbles i and i + 4).
    // (Both steps of a word lie side by side.)
    uint4 *sq = reinterpret_cast<uint4 *>(smem);
#pragma unroll
    for (int j = 0; j < kQEach; ++j) {
        const int i = tid + kThreads * j, row = i / (kD / 8), x = i - row * (kD / 8), qt = x / kW, w = x - qt * kW;
        if (i >= kQWords) break;
        float v[8];
        raw[j].get(v);
#pragma unroll
        for (int part = 0; part < kParts; ++part) {
            uint32_t pr[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) pr[e] = take_part(v[e], v[e + 4]);
            sq[((part * kNT + (row >> 3)) * kW + w) * 32 + (row & 7) * 4 + qt] = make_uint4(pr[0], pr[1], pr[2], pr[3]);
        }
    }
    __syncthreads();
    uint4 qf[L::kQInRegs ? kNT * kParts : 1][kW];
    if (L::kQInRegs) {
#pragma unroll
        for (int n = 0; n < kNT * kParts; ++n)
#pragma unroll
            for (int w = 0; w < kW; ++w) qf[n][w] = sq[(n * kW + w) * 32 + lane];
    }

    const float sl2 = p.scale * 1.4426950408889634f;
    float m[kNT][2], l[kNT][2];                                 // query rows 2 t, 2 t + 1 of a column tile
    float acc[kNT][kMt][4];                                     // O^T: channels (kD / 8) r + 2 i, + 1 by rows 2 t, 2 t + 1
#pragma unroll
    for (int n = 0; n < kNT; ++n) {
        m[n][0] = m[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
#pragma unroll
        for (int i = 0; i < kMt; ++i) acc[n][i][0] = acc[n][i][1] = acc[n][i][2] = acc[n][i][3] = 0.f;
    }
    // Key of row i of a 16-row operand: i = 2 t + e (+ 8) stands for key t + 4 e (+ 8).
    const int my_key = (r >> 1) + 4 * (r & 1);
    int stage = 0;
#pragma unroll 1
    for (int tile = tile_lo + warp; tile < tile_hi; tile += kWarps) {
        cp_async_wait<kStages - 2>();
        __syncwarp();
        {
            const int next = tile + (kStages - 1) * kWarps, st = stage == 0 ? kStages - 1 : stage - 1;
            if (next < tile_hi) load_tile(next, st);
            cp_async_commit();
        }
        const uint8_t *sK = ring + stage * L::kStageBytes, *sV = sK + L::kCodeBytes;
        const uint8_t *sKs = sV + L::kCodeBytes, *sVs = sKs + L::kScaleBytes;
        stage = stage + 1 == kStages ? 0 : stage + 1;

        // ---- S^T = K Q^T: two row tiles of 16 keys ----
        float s[2][kNT][4];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[mt][n][c] = 0.f;
        uint32_t code[2][2][kW];                                // keys 16 mt + 8 e + my_key
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint8_t *src = sK + (16 * mt + 8 * e + my_key) * L::kCodeRow + t * (kD / 8);
                if (kW == 4) {
                    const uint4 x = *reinterpret_cast<const uint4 *>(src);
                    code[mt][e][0] = x.x; code[mt][e][1] = x.y; code[mt][e][2 % kW] = x.z; code[mt][e][3 % kW] = x.w;
                } else if (kW == 2) {
                    const uint2 x = *reinterpret_cast<const uint2 *>(src);
                    code[mt][e][0] = x.x; code[mt][e][1 % kW] = x.y;
                } else {
#pragma unroll
                    for (int w = 0; w < kW; ++w) code[mt][e][w] = reinterpret_cast<const uint32_t *>(src)[w];
                }
            }
        uint32_t sc[2][2], of[2][2];
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            uint32_t a[2][2][4];                                // [half of the word][row tile]
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (w == 0 || kW == 3) {                    // the group of this word; 96 channels: a quarter may touch two
                        sc[mt][e] = scale_pair(sKs[(16 * mt + 8 * e + my_key) * L::kScaleRow + ((t * kW + w) >> 2)]);
                        of[mt][e] = offset_pair(sc[mt][e]);
                    }
                    const uint32_t x = code[mt][e][w];
                    a[0][mt][e] = nibble_pair<0>(x, sc[mt][e], of[mt][e]);
                    a[0][mt][2 + e] = nibble_pair<1>(x, sc[mt][e], of[mt][e]);
                    a[1][mt][e] = nibble_pair<2>(x, sc[mt][e], of[mt][e]);
                    a[1][mt][2 + e] = nibble_pair<3>(x, sc[mt][e], of[mt][e]);
                }
            // products on one sum stand as far apart as they can
#pragma unroll
            for (int part = 0; part < kParts; ++part) {
                uint4 b[kNT];
#pragma unroll
                for (int n = 0; n < kNT; ++n) b[n] = L::kQInRegs ? qf[part * kNT + n][w] : sq[((part * kNT + n) * kW + w) * 32 + lane];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int n = 0; n < kNT; ++n)
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt) mma_bf16(s[mt][n], a[h][mt], h ? b[n].z : b[n].x, h ? b[n].w : b[n].y);
            }
        }
        // ---- mask, online softmax: a row's 32 keys are 4 values in each of the 8 lanes with the same t ----
        const int key0 = walk.key0(tile);
        if (!walk.sees_all(key0)) {                                         // (-inf stays -inf under a positive factor)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (!walk.sees(key0 + 16 * mt + 8 * e + my_key))
#pragma unroll
                        for (int n = 0; n < kNT; ++n) s[mt][n][2 * e] = s[mt][n][2 * e + 1] = -INFINITY;
        }
        // The reference of a row moves when one of its lanes has seen a logit more than 2^8 above it: one vote per tile for all rows,
        // and the shuffles only then.
        float mx[kNT][2];
        bool above = false;
#pragma unroll
        for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                mx[n][e] = fmaxf(fmaxf(s[0][n][e], s[0][n][2 + e]), fmaxf(s[1][n][e], s[1][n][2 + e])) * sl2;
                above = above || mx[n][e] > m[n][e] + kRescale;
            }
        if (__any_sync(0xffffffffu, above)) {
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) mx[n][e] = fmaxf(mx[n][e], __shfl_xor_sync(0xffffffffu, mx[n][e], o));
                    const float mn = fmaxf(m[n][e], mx[n][e]), al = mn == -INFINITY ? 1.f : ex2(m[n][e] - mn);
                    m[n][e] = mn;
                    l[n][e] *= al;
#pragma unroll
                    for (int i = 0; i < kMt; ++i) { acc[n][i][e] *= al; acc[n][i][2 + e] *= al; }
                }
        }
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
            const float ref[2] = {m[n][0] == -INFINITY ? 0.f : m[n][0], m[n][1] == -INFINITY ? 0.f : m[n][1]};
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    s[mt][n][c] = ex2(fmaf(s[mt][n][c], sl2, -ref[c & 1]));
                    l[n][c & 1] += s[mt][n][c];
                }
        }
        uint32_t pf[kParts][kNT][2][2];                         // P^T as operand B: [row tile of keys][half]
#pragma unroll
        for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int n = 0; n < kNT; ++n)
#pragma unroll
                for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        pf[part][n][mt][e] = transpose8(kParts > 1 ? take_part(s[mt][n][2 * e], s[mt][n][2 * e + 1])
                                                                   : pack_bf16(s[mt][n][2 * e], s[mt][n][2 * e + 1]));
        // ---- O^T += V^T P^T ----
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
            // keys 16 mt + 8 e + t + 4 f: half e of the step, member f of the pair
            uint32_t code[2][2][kW > 1 ? (kW + 1) / 2 : 1];     // this lane's kD / 8 channels: kW half-words
            uint32_t sc[2], of[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const int key = 16 * mt + 8 * e + 4 * f + t;
                    const uint8_t *src = sV + key * L::kCodeRow;
                    if (kW == 4) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(src + (((r >> 1) ^ (t & 2)) << 4) + 8 * (r & 1));
                        code[e][f][0] = x.x; code[e][f][kW > 2 ? 1 : 0] = x.y;
                    } else if (kW == 2) {
                        code[e][f][0] = *reinterpret_cast<const uint32_t *>(src + 4 * r);
                    } else {
                        const uint16_t *h = reinterpret_cast<const uint16_t *>(src + 2 * kW * r);
                        code[e][f][0] = h[0];
                        if (kW == 3) { code[e][f][0] |= (uint32_t)h[1 % kW] << 16; code[e][f][kW > 2 ? 1 : 0] = h[2 % kW]; }
                    }
                }
#pragma unroll
            for (int u = 0; u < kW; ++u) {                      // half-words: channels (kD / 8) r + 4 u .. + 3
                if (u == 0 || kW == 3) {
                    const int grp = ((kD / 8) * r + 4 * u) / kQuantGroup;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint8_t *src = sVs + (16 * mt + 8 * e + t) * L::kScaleRow + grp;
                        sc[e] = scale_pair(src[0], src[4 * L::kScaleRow]);
                        of[e] = offset_pair(sc[e]);
                    }
                }
                uint32_t v[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = __byte_perm(code[e][0][u >> 1], code[e][1][u >> 1], u & 1 ? 0x7632 : 0x5410);
                    v[e][0] = nibble_pair<0>(x, sc[e], of[e]);
                    v[e][1] = nibble_pair<1>(x, sc[e], of[e]);
                    v[e][2] = nibble_pair<2>(x, sc[e], of[e]);
                    v[e][3] = nibble_pair<3>(x, sc[e], of[e]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t a[4] = {v[0][2 * i], v[0][2 * i + 1], v[1][2 * i], v[1][2 * i + 1]};
#pragma unroll
                    for (int part = 0; part < kParts; ++part)
#pragma unroll
                        for (int n = 0; n < kNT; ++n) mma_bf16(acc[n][2 * u + i], a, pf[part][n][mt][0], pf[part][n][mt][1]);
                }
            }
        }
        __syncwarp();                                           // every lane is done with the stage that the next copies overwrite
    }
    cp_async_wait<0>();

    // ---- partials of the warps, where the rings were ----
    __syncthreads();
    float *part = reinterpret_cast<float *>(smem + L::kQBytes); // [warp][row][kPartialRow]
#pragma unroll
    for (int n = 0; n < kNT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float z = l[n][e];
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
            float *dst = part + (warp * kRows + 8 * n + 2 * t + e) * L::kPartialRow;
            if (r == 0) *reinterpret_cast<float2 *>(dst) = make_float2(m[n][e], z);
            dst += 4 + (kD / 8) * r;
#pragma unroll
            for (int i = 0; i < kMt; i += 2)
                *reinterpret_cast<float4 *>(dst + 2 * i) = make_float4(acc[n][i][e], acc[n][i][2 + e], acc[n][i + 1][e], acc[n][i + 1][2 + e]);
        }
    __syncthreads();
    // The workspace may still be read by the merge of the previous call; outputs and this grid's end come behind the wait too.
    if (!kOneLaunch) grid_wait();
    // ---- fold the warps: a warp per row, four channels per lane; into the first warp's row, or the workspace ----
    constexpr int kEach = kRows / kWarps, kFold = kEach < 4 ? kEach : 4;     // rows of a warp, and how many at a time
#pragma unroll 1
    for (int r0 = 0; r0 < kEach; r0 += kFold) {
        float2 ml[kFold][kWarps];
        float4 v[kFold][kWarps];
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const float *src = part + (warp + kWarps * (r0 + i)) * L::kPartialRow;
#pragma unroll
            for (int q = 0; q < kWarps; ++q) {
                ml[i][q] = *reinterpret_cast<const float2 *>(src + q * kRows * L::kPartialRow);
                v[i][q] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (4 * lane < kD) v[i][q] = *reinterpret_cast<const float4 *>(src + q * kRows * L::kPartialRow + 4 + 4 * lane);
            }
        }
        __syncwarp();                                           // every lane has read the maxima and sums
#pragma unroll
        for (int i = 0; i < kFold; ++i) {
            const int row = warp + kWarps * (r0 + i);
            const float mx = fmaxf(fmaxf(ml[i][0].x, ml[i][1].x), fmaxf(ml[i][2].x, ml[i][3].x)), ref = mx == -INFINITY ? 0.f : mx;
            float z = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < kWarps; ++q) {
                const float f = ex2(ml[i][q].x - ref);
                z += ml[i][q].y * f;
                o.x += v[i][q].x * f; o.y += v[i][q].y * f; o.z += v[i][q].z * f; o.w += v[i][q].w * f;
            }
            if (row >= rows_here) break;
            float *dst = kOneLaunch ? part + row * L::kPartialRow : p.partial + (out_row(chunk * kRows + row) * n_splits + split) * L::kPartialRow;
            if (lane == 0) *reinterpret_cast<float2 *>(dst) = make_float2(mx, z);
            if (4 * lane < kD) *reinterpret_cast<float4 *>(dst + 4 + 4 * lane) = o;
        }
    }
    if (!kOneLaunch) return;
    // ---- fold the CTAs of the cluster: rank q finishes rows q, q + n_splits, ... ----
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    if (n_splits > 1) cluster.sync(); else __syncthreads();
    grid_wait();                                                // before the first write
    for (int row = split + n_splits * warp; row < rows_here; row += n_splits * kWarps) {
        float2 ml[kMaxCluster];
        float4 v[kMaxCluster];
        float mx = -INFINITY;
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) {
            ml[q] = make_float2(-INFINITY, 0.f);
            v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (q < n_splits) {
                const float *src = (n_splits > 1 ? cluster.map_shared_rank(part, q) : part) + row * L::kPartialRow;
                ml[q] = *reinterpret_cast<const float2 *>(src);
                if (4 * lane < kD) v[q] = *reinterpret_cast<const float4 *>(src + 4 + 4 * lane);
            }
        }
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) mx = fmaxf(mx, ml[q].x);
        const float ref = mx == -INFINITY ? 0.f : mx;
        float z = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int q = 0; q < kMaxCluster; ++q) {
            const float f = ex2(ml[q].x - ref);
            z += ml[q].y * f;
            o.x += v[q].x * f; o.y += v[q].y * f; o.z += v[q].z * f; o.w += v[q].w * f;
        }
        const float inv = z > 0.f ? 1.f / z : 0.f;
        const int64_t orow = out_row(chunk * kRows + row);
        if (4 * lane < kD) store4(static_cast<T *>(p.o) + orow * kD + 4 * lane, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
        if (lane == 0 && p.lse) p.lse[orow] = z > 0.f ? lse_exact(mx, z) : -INFINITY;
    }
    if (n_splits > 1) cluster.sync();                           // peers may still be reading this CTA's partials
}

// A CTA takes output rows blockIdx.x, blockIdx.x + gridDim.x, ...: four groups of slots by 32 lanes of four channels.  At most one CTA
// per SM, and small: the next call's stream kernel is launched when every CTA of this grid has started.
constexpr int kMergeGroups = 4;
template <typename T>
__global__ void __launch_bounds__(32 * kMergeGroups)
decode_quant_merge_kernel(const float *partial, T *out, float *lse, int d, int n_slots, int n_rows)
{
    __shared__ float4 s_o[kMergeGroups][32];
    __shared__ float2 s_ml[kMergeGroups];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    grid_wait();                                                // the partials of this call
    const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
    const bool mine = 4 * lane < d;
    for (int64_t orow = blockIdx.x; orow < n_rows; orow += gridDim.x) {
        const float *src = partial + orow * n_slots * (d + 4);
        float mm = -INFINITY, ll = 0.f;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = grp; k0 < n_slots; k0 += 4 * kMergeGroups) {
            float2 ml[4];
            float4 v[4];
            float mn = mm;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int slot = k0 + k * kMergeGroups;
                ml[k] = make_float2(-INFINITY, 0.f);
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (slot < n_slots) {
                    ml[k] = ld_partial2(src + slot * (d + 4));
                    if (mine) v[k] = ld_partial4(src + slot * (d + 4) + 4 + 4 * lane);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) mn = fmaxf(mn, ml[k].x);
            const float ref = mn == -INFINITY ? 0.f : mn, f0 = ex2(mm - ref);
            ll *= f0; a.x *= f0; a.y *= f0; a.z *= f0; a.w *= f0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float f = ex2(ml[k].x - ref);             // 0 for an empty partial
                ll += ml[k].y * f;
                a.x += v[k].x * f; a.y += v[k].y * f; a.z += v[k].z * f; a.w += v[k].w * f;
            }
            mm = mn;
        }
        s_o[grp][lane] = a;
        if (lane == 0) s_ml[grp] = make_float2(mm, ll);
        __syncthreads();
        if (grp == 0) {
            float mx = -INFINITY, z = 0.f;
#pragma unroll
            for (int q = 0; q < kMergeGroups; ++q) mx = fmaxf(mx, s_ml[q].x);
            const float ref = mx == -INFINITY ? 0.f : mx;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int q = 0; q < kMergeGroups; ++q) {
                const float f = ex2(s_ml[q].x - ref);
                const float4 v = s_o[q][lane];
                z += s_ml[q].y * f;
                o.x += v.x * f; o.y += v.y * f; o.z += v.z * f; o.w += v.w * f;
            }
            const float inv = z > 0.f ? 1.f / z : 0.f;
            if (mine) store4(out + orow * d + 4 * lane, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
            if (lane == 0 && lse) lse[orow] = z > 0.f ? lse_exact(mx, z) : -INFINITY;
        }
        __syncthreads();                                        // the group buffers are reused by the next row
    }
}

typedef void (*Kernel)(const QuantDecodeParams, int, int);
struct Variant {
    Kernel kernel;
    int smem;
};
template <typename T, int kD, bool kOneLaunch> Variant variant_of(int nt)
{
    if (nt == 1) return {decode_quant_kernel<T, kD, 1, kOneLaunch>, Layout<T, kD, 1>::kBytes};
    if (nt == 2 || sizeof(T) == 4) return {decode_quant_kernel<T, kD, 2, kOneLaunch>, Layout<T, kD, 2>::kBytes};
    return {decode_quant_kernel<T, kD, sizeof(T) == 4 ? 2 : 4, kOneLaunch>, Layout<T, kD, sizeof(T) == 4 ? 2 : 4>::kBytes};
}
template <typename T, bool kOneLaunch> Variant variant_of(int d, int nt)
{
    switch (d) {
    case 32: return variant_of<T, 32, kOneLaunch>(nt);
    case 64: return variant_of<T, 64, kOneLaunch>(nt);
    case 96: return variant_of<T, 96, kOneLaunch>(nt);
    default: return variant_of<T, 128, kOneLaunch>(nt);
    }
}

}  // namespace

size_t decode_quant_scratch_bytes(int n_part, int hq, int d)
{
    return d % kQuantGroup == 0 ? (size_t)n_part * hq * kMaxSlots * (d + 4) * sizeof(float) : 0;
}

cudaError_t launch_decode_quant(const QuantDecodeParams &p_in, int dtype, int device, int sm_count, cudaStream_t s, int64_t *launches)
{
    QuantDecodeParams p = p_in;
    const int g = p.hq / p.hkv, rows_total = p.sync ? p.n_part * g : g, caches = p.sync ? 1 : p.n_part;
    const bool f32 = dtype == FEDATTN_F32;
    const int nt = rows_total <= 8 ? 1 : (rows_total <= 16 || f32 ? 2 : 4);
    const int n_chunks = (rows_total + 8 * nt - 1) / (8 * nt);
    const int64_t sources = (int64_t)caches * p.hkv * n_chunks;
    if ((int64_t)caches * n_chunks > 65535 || p.hkv > 65535) return cudaErrorInvalidValue;        // grid
    // keys that a walk goes over, at most
    int64_t keys = p.max_kv_len;
    if (p.window > 0 && (int64_t)p.window + p.n_sink + 2 * kTileKeys < keys) keys = (int64_t)p.window + p.n_sink + 2 * kTileKeys;
    const int tiles = (int)((keys + kTileKeys - 1) / kTileKeys);
    const int per_sm = nt == 4 || f32 ? 2 : 3;                  // CTAs of an SM: one wave
    int64_t n_splits = (int64_t)per_sm * sm_count / sources;
    if (n_splits > tiles / kWarps) n_splits = tiles / kWarps;   // a tile per warp at the least
    if (n_splits > kMaxSlots) n_splits = kMaxSlots;
    if (n_splits < 1) n_splits = 1;
    bool one_launch = n_splits <= kMaxCluster;
    if (!one_launch && (size_t)p.n_part * p.hq * n_splits * (p.d + 4) * sizeof(float) > p.partial_bytes) return cudaErrorInvalidValue;
    typedef __nv_bfloat16 bf;
    const Variant v = one_launch ? (f32 ? variant_of<float, true>(p.d, nt) : variant_of<bf, true>(p.d, nt))
                                 : (f32 ? variant_of<float, false>(p.d, nt) : variant_of<bf, false>(p.d, nt));
    static bool attr_set[64][2][2][4][3] = {};                  // the attribute is per device
    bool &set = attr_set[device & 63][f32][one_launch][p.d / 32 - 1][nt >> 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, v.smem);
        if (e != cudaSuccess) return e;
        set = true;
    }
    // may the stream kernel read its inputs before the preceding grid of the stream is complete?
    const size_t rows = (size_t)caches * p.hkv * p.cap, code_bytes = rows * (p.d / 2), scale_bytes = rows * (p.d / kQuantGroup);
    const size_t qo_bytes = (size_t)p.n_part * p.hq * p.d * (f32 ? 4 : 2);
    const MemRange in[6] = {{p.q, qo_bytes}, {p.k_codes, code_bytes}, {p.k_scales, scale_bytes}, {p.v_codes, code_bytes},
                            {p.v_scales, scale_bytes}, {p.kv_len, caches * sizeof(int32_t)}};
    const MemRange out[2] = {{p.o, qo_bytes}, {p.lse, p.lse ? (size_t)p.n_part * p.hq * sizeof(float) : 0}};
    // (The record costs a short call 0.5 us of the host, 4.5 -> 5.0 us in a loop of 4 x 700 keys of 64 channels; replayed from a graph
    // the early start takes it from 4.2 to 1.5.)
    const EarlyStart es = early_start(device, s, in, 6, out, 2);
    p.early = es.early ? 1 : 0;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)n_splits; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3((unsigned)n_splits, (unsigned)p.hkv, (unsigned)(caches * n_chunks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = v.smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = one_launch ? 2 : 1;
    cudaError_t e = cudaLaunchKernelEx(&cfg, v.kernel, p, (int)n_splits, n_chunks);
    ++*launches;
    if (e != cudaSuccess || one_launch) return early_start_end(es, e != cudaSuccess ? e : cudaGetLastError());
    const int n_rows = p.n_part * p.hq, per_cta = (n_rows + sm_count - 1) / sm_count;
    cfg.gridDim = dim3((unsigned)((n_rows + per_cta - 1) / per_cta));
    cfg.blockDim = dim3(32 * kMergeGroups);
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    const float *partial = p.partial;
    e = f32 ? cudaLaunchKernelEx(&cfg, decode_quant_merge_kernel<float>, partial, static_cast<float *>(p.o), p.lse, (int)p.d, (int)n_splits, n_rows)
            : cudaLaunchKernelEx(&cfg, decode_quant_merge_kernel<bf>, partial, static_cast<bf *>(p.o), p.lse, (int)p.d, (int)n_splits, n_rows);
    ++*launches;
    return early_start_end(es, e != cudaSuccess ? e : cudaGetLastError());
}

}  // namespace fedattn
