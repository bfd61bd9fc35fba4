// Gradient of a layer's weights from the 8-bit checkpoint of its input:  dw[n][k] = sum_t dy[t][n] x^[t][k].
//
// A bf16 (fp16) product on the tensor cores whose one operand is decoded on the way: x^ = q 2^E has 7 significant bits,
// so it is exact in either type, and the gradient carries no error beside the checkpoint's own and the fp32 sums'.
// Both operands lie in memory with the summed index (tokens) outermost, which the tensor cores take as it is (MN-major).
//
// x^ is the M operand (128 values of k a tile), dy the N operand (up to 256 channels): a decoded value then meets 256
// others, and a warp's 32 accumulator lanes are neighbours in a row of dw.  Per stage of 64 tokens the TMA fetches 8 KB of
// codes and 32 KB of dy; eight warps (two groups of them, in turn) turn the codes into 16 KB of operand (one block of 32 values a thread: a
// byte permutation, a subtraction and a multiplication for every two); one thread issues the four instructions of the
// stage; four warps write the previous tile out meanwhile (two accumulators of 256 columns fill tensor memory).
// (2047 x 2592 x 256 14.4 us; 8192 x 4096 x 4096 into fp32 388 us this way, by the pairs below 256 to 273.)
//
// Where the tiles do not cover the chip the tokens are split over a cluster, whose CTAs add their parts through
// distributed shared memory in a fixed order.  db is a tile of its own whose decoded operand is all ones.
#include <cooperative_groups.h>

#include <algorithm>

#include "learn.cuh"
#include "tc_image.cuh"

namespace accerl {

namespace {

__device__ int g_status;  // of this file's bounded waits

constexpr int kTileK = 128, kTokens = 64;        // values of k a tile, tokens a stage
constexpr int kRaw = 4, kDec = 3, kDy = 4;       // stages of the three rings
constexpr int kRawBytes = kTokens * kTileK, kDecBytes = 2 * kRawBytes;
constexpr int kAhead = 6;                        // stages whose exponents are on their way
constexpr int kMaxShare = 8;                     // CTAs of a cluster
constexpr int kConvWarps = 8, kGroups = 2;        // warps that decode a stage; groups of them that take stages in turn
constexpr int kFirstOut = 4 + kGroups * kConvWarps, kThreads = 32 * (kFirstOut + 4);

struct GradArgs {
    const uint8_t *e;
    void *dw, *db;
    long long ld_e, ld_dw;
    int tokens, n, k, out_dtype, accumulate;
    int n_tile, n_tiles, k_tiles, tiles;  // tiles: those of db included
    int cols32;
};

__device__ __forceinline__ void mma_f16(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// 64 columns of the M or N index (128 bytes) by rows of tokens, 128-byte swizzle: groups of 8 tokens lie 1024 bytes
// apart, blocks of 64 columns a whole block of kTokens rows
__device__ __forceinline__ uint64_t mn_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (uint64_t)((kTokens * 128) >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// two bytes of `w` (selected) as two bf16 integers: with 0x43 above them the low seven bits read 128 + value, the sign
// bit alone 128 or 256
template <typename T>
struct Decode;
template <>
struct Decode<__nv_bfloat16> {
    __nv_bfloat162 s;
    __device__ __forceinline__ explicit Decode(int e)
    {
        const uint32_t b = (uint32_t)e << 7;  // 2^(e - 127); 255: infinity, times the block's zeros NaN
        const uint32_t two = b | b << 16;
        s = *reinterpret_cast<const __nv_bfloat162 *>(&two);
    }
    __device__ __forceinline__ uint32_t pair(uint32_t w, uint32_t sel) const
    {
        const uint32_t t = __byte_perm(w, 0x43434343u, sel), a = t & 0xff7fff7fu, c = t & 0xff80ff80u;
        const __nv_bfloat162 q = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&c));
        const __nv_bfloat162 v = __hmul2(q, s);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static constexpr uint32_t kOnes = 0x3f803f80u;
};
template <>
struct Decode<__half> {
    __half2 s1, s2;  // 2^E in two factors, each a half (E goes beyond its range on both sides)
    __device__ __forceinline__ explicit Decode(int e)
    {
        const int E = e - 127, a = min(max(E, -14), 15), b = max(min(E - a, 1), -24);
        const float f1 = e == 255 ? NAN : __uint_as_float((uint32_t)(a + 127) << 23), f2 = __uint_as_float((uint32_t)(b + 127) << 23);
        s1 = __float2half2_rn(f1);
        s2 = __float2half2_rn(f2);
    }
    __device__ __forceinline__ uint32_t pair(uint32_t w, uint32_t sel) const
    {
        const uint32_t t = __byte_perm(w ^ 0x80808080u, 0x64646464u, sel);  // 1024 + 128 + value
        const __half2 q = __hsub2(*reinterpret_cast<const __half2 *>(&t), __float2half2_rn(1152.f));
        const __half2 v = __hmul2(__hmul2(q, s1), s2);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static constexpr uint32_t kOnes = 0x3c003c00u;
};

// A thread's share of a stage: 32 values of one token (block b of the row, t the token of the stage) from the TMA's
// swizzled codes to the operand's rows of 64 values, swizzled alike.  Lanes are tokens: no two of eight meet in a bank.
template <typename T>
__device__ __forceinline__ void load_codes(uint32_t raw, int b, int t, uint32_t (&q)[8])
{
    const uint32_t row = raw + t * 128;
    const uint4 lo = lds16(row + (((2 * b) ^ (t & 7)) << 4)), hi = lds16(row + (((2 * b + 1) ^ (t & 7)) << 4));
    q[0] = lo.x, q[1] = lo.y, q[2] = lo.z, q[3] = lo.w, q[4] = hi.x, q[5] = hi.y, q[6] = hi.z, q[7] = hi.w;
}
template <typename T>
__device__ __forceinline__ void put_values(uint32_t dec, int b, int t, const uint32_t (&q)[8], int e, bool ones)
{
    const uint32_t out = dec + (b >> 1) * (kTokens * 128) + t * 128;
    const Decode<T> d(e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint4 v;
        if (!ones) {
            v.x = d.pair(q[2 * i], 0x4140);
            v.y = d.pair(q[2 * i], 0x4342);
            v.z = d.pair(q[2 * i + 1], 0x4140);
            v.w = d.pair(q[2 * i + 1], 0x4342);
        } else {
            v.x = v.y = v.z = v.w = Decode<T>::kOnes;
        }
        sts16(out + ((((b & 1) * 4 + i) ^ (t & 7)) << 4), v);
    }
}

// fp32 results: the tensor cores cut a sum off at every addition, which over 8192 tokens costs 4.5e-6 of the result's
// norm (4e-7 with an fp32 product's rounding).  So an accumulator covers at most kChunk stages, and its parts are
// added in fp32 by the warps that write: 5e-7.  The sum lies in the other half of tensor memory (adding in memory instead
// cost 634 us with loads and 379 with reductions, for 8192 x 4096 x 4096), and the tensor cores wait while a part is
// added, some 5 % of a part's time.  Results of one part have two accumulators in turn instead.  16-bit results are in one
// part up to kChunk16 stages (8192 tokens), whose loss is far below their rounding; without an end to it the sums of 2^22 tokens
// of one sign would lose more than half a step of fp16.
constexpr int kChunk = 24, kChunk16 = 128;
__host__ __device__ __forceinline__ int chunks_of(int out_dtype, int stages)
{
    const int most = out_dtype == ACCERL_F32 ? kChunk : kChunk16;
    return (stages + most - 1) / most;
}

// the accumulators in turn: two, or always the first
struct Acc {
    int slot = 0;
    uint32_t phase = 0;
    bool one;
    __device__ __forceinline__ explicit Acc(bool single) : one(single) {}
    __device__ __forceinline__ void next()
    {
        if (one || ++slot == 2) {
            slot = 0;
            phase ^= 1;
        }
    }
};

// Adds a part to the sum in a warp's quarter of tensor memory (columns 256 behind it), or begins it.
__device__ __forceinline__ void add_part(uint32_t quarter, int j0, int j1, bool begin)
{
    for (int j = j0; j < j1; j += 16) {
        int part[16], sum[16];
        tmem_ld16(quarter + j, part);
        if (!begin) tmem_ld16(quarter + 256 + j, sum);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] = begin ? part[i] : __float_as_int(__int_as_float(sum[i]) + __int_as_float(part[i]));
        tmem_st16(quarter + 256 + j, sum);
    }
    tmem_wait_st();
}

struct __align__(8) GradBars {
    uint64_t raw_full[kRaw], raw_empty[kRaw], dec_full[kDec], dec_empty[kDec], dy_full[kDy], dy_empty[kDy], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
};

// position in a ring and its phase
template <int N>
struct Ring {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next()
    {
        if (++slot == N) {
            slot = 0;
            phase ^= 1;
        }
    }
};

__device__ __forceinline__ float load_out(const GradArgs &p, const void *base, long long at)
{
    return p.out_dtype == ACCERL_F32 ? static_cast<const float *>(base)[at] : 0.f;
}
__device__ __forceinline__ void store_out(const GradArgs &p, void *base, long long at, float v)
{
    if (p.out_dtype == ACCERL_F32) static_cast<float *>(base)[at] = v;
    else if (p.out_dtype == ACCERL_BF16) static_cast<__nv_bfloat16 *>(base)[at] = __float2bfloat16_rn(v);
    else static_cast<__half *>(base)[at] = __float2half_rn(v);
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 1)
weight_grad_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_dy,
                   const __grid_constant__ GradArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ GradBars bars;
    namespace cg = cooperative_groups;
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const int dy_bytes = p.n_tile * 2 * kTokens;
    const uint32_t raw0 = smem_u32(smem), dec0 = raw0 + kRaw * kRawBytes, dy0 = dec0 + kDec * kDecBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int share = (int)cg::this_cluster().num_blocks(), rank = (int)cg::this_cluster().block_rank();
    const int stages_all = (p.tokens + kTokens - 1) / kTokens;
    const int g0 = (int)((long long)stages_all * rank / share), g1 = (int)((long long)stages_all * (rank + 1) / share);
    const int first = (int)(blockIdx.x / (unsigned)share), stride = (int)(gridDim.x / (unsigned)share);
    const int chunks = chunks_of(p.out_dtype, g1 - g0);
    volatile int *abort_flag = &bars.abort_flag;
    auto bar = [](uint64_t &b) { return smem_u32(&b); };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kRaw; ++i) {
            mbar_init(bar(bars.raw_full[i]), 1);
            mbar_init(bar(bars.raw_empty[i]), kConvWarps);
        }
        for (int i = 0; i < kDec; ++i) {
            mbar_init(bar(bars.dec_full[i]), kConvWarps);
            mbar_init(bar(bars.dec_empty[i]), 1);
        }
        for (int i = 0; i < kDy; ++i) {
            mbar_init(bar(bars.dy_full[i]), 1);
            mbar_init(bar(bars.dy_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(bars.acc_full[i]), 1);
            mbar_init(bar(bars.acc_empty[i]), 4);
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = bars.tmem;
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------------------------ loads of codes
        // (apart from those of dy, which would hold them up: a stage of dy is free only when the tensor cores are done with it)
        Ring<kRaw> r;
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles;
            for (int g = g0; g < g1 && ok && kt < p.k_tiles; ++g) {
                ok = mbar_wait(bar(bars.raw_empty[r.slot]), r.phase ^ 1, abort_flag, &g_status, 1);
                if (ok && elect_one()) {
                    mbar_expect_tx(bar(bars.raw_full[r.slot]), kRawBytes);
                    tma_load_2d(raw0 + r.slot * kRawBytes, &map_q, kt * kTileK, g * kTokens, bar(bars.raw_full[r.slot]));
                }
                __syncwarp();
                r.next();
            }
        }
    } else if (warp == 2) {
        // --------------------------------------------------------------------------------- loads of dy
        Ring<kDy> d;
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int n0 = u % p.n_tiles * p.n_tile;
            for (int g = g0; g < g1 && ok; ++g) {
                ok = mbar_wait(bar(bars.dy_empty[d.slot]), d.phase ^ 1, abort_flag, &g_status, 2);
                if (ok && elect_one()) {
                    mbar_expect_tx(bar(bars.dy_full[d.slot]), (uint32_t)dy_bytes);
                    for (int b = 0; b < p.n_tile / 64; ++b)
                        tma_load_2d(dy0 + d.slot * dy_bytes + b * kTokens * 128, &map_dy, (n0 + 64 * b) * 2, g * kTokens, bar(bars.dy_full[d.slot]));
                }
                __syncwarp();
                d.next();
            }
        }
    } else if (warp == 1) {
        // ------------------------------------------------------------------------------ tensor core
        constexpr uint32_t kType = std::is_same<T, __half>::value ? 0u : 1u;
        const uint32_t idesc = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(p.n_tile >> 3) << 17) |
                               ((uint32_t)(kTileK >> 4) << 24);
        Ring<kDec> c;
        Ring<kDy> d;
        Acc a(chunks > 1);
        for (int u = first; u < p.tiles && ok; u += stride)
            for (int ch = 0; ch < chunks && ok; ++ch) {
                const int h0 = g0 + (int)((long long)(g1 - g0) * ch / chunks), h1 = g0 + (int)((long long)(g1 - g0) * (ch + 1) / chunks);
                ok = mbar_wait(bar(bars.acc_empty[a.slot]), a.phase ^ 1, abort_flag, &g_status, 4);
                fence_after();
                for (int g = h0; g < h1 && ok; ++g) {
                    ok = mbar_wait(bar(bars.dec_full[c.slot]), c.phase, abort_flag, &g_status, 8);
                    if (ok) ok = mbar_wait(bar(bars.dy_full[d.slot]), d.phase, abort_flag, &g_status, 8);
                    fence_after();
                    if (ok && elect_one()) {
                        const uint64_t ad = mn_desc(dec0 + c.slot * kDecBytes), bd = mn_desc(dy0 + d.slot * dy_bytes);
#pragma unroll
                        for (int ks = 0; ks < kTokens / 16; ++ks)
                            mma_f16(tmem + 256 * a.slot, ad + ks * (2048 >> 4), bd + ks * (2048 >> 4), idesc, (uint32_t)((g - h0) | ks));
                        mma_commit(bar(bars.dec_empty[c.slot]));
                        mma_commit(bar(bars.dy_empty[d.slot]));
                        if (g == h1 - 1) mma_commit(bar(bars.acc_full[a.slot]));
                    }
                    __syncwarp();
                    c.next();
                    d.next();
                }
                a.next();
            }
    } else if (warp >= 4 && warp < kFirstOut) {
        // ------------------------------------------------------------------------------------ decoding
        const int group = (warp - 4) / kConvWarps, w = (warp - 4) % kConvWarps;
        const int b = w & 3, t = (w >> 2) * 32 + lane;  // block of 32 values, token of the stage
        int seq = 0, raws = 0;                          // stages so far, of the CTA; those with codes
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles;
            const bool codes = kt < p.k_tiles;
            const int col = kt * kTileK + 32 * b;
            const bool in = codes && col < p.cols32;
            const uint8_t *e_at = p.e + col / 32 + (long long)t * p.ld_e;
            const long long e_step = (long long)kTokens * p.ld_e;
            const int g_first = g0 + (group - seq % kGroups + kGroups) % kGroups;  // this group's stages of the tile
            auto exponent = [&](int g) { return in && g < g1 && g * kTokens + t < p.tokens ? (int)__ldg(e_at + g * e_step) : 127; };
            int ahead[kAhead / kGroups];  // a load takes as long as some stages
#pragma unroll
            for (int i = 0; i < kAhead / kGroups; ++i) ahead[i] = exponent(g_first + kGroups * i);
            for (int g = g_first; g < g1 && ok;) {
#pragma unroll
                for (int i = 0; i < kAhead / kGroups; ++i) {  // (unrolled: a value on its way is not to be moved)
                    if (g >= g1 || !ok) break;
                    const int e = ahead[i];
                    ahead[i] = exponent(g + kAhead);
                    const int n = seq + g - g0, rn = raws + g - g0, rs = rn % kRaw, ds = n % kDec;
                    uint32_t q[8] = {};
                    if (codes) {
                        ok = mbar_wait(bar(bars.raw_full[rs]), (uint32_t)(rn / kRaw & 1), abort_flag, &g_status, 16);
                        load_codes<T>(raw0 + rs * kRawBytes, b, t, q);
                    }
                    if (ok) ok = mbar_wait(bar(bars.dec_empty[ds]), (uint32_t)(n / kDec & 1) ^ 1, abort_flag, &g_status, 32);
                    ok = __all_sync(0xffffffffu, ok);
                    put_values<T>(dec0 + ds * kDecBytes, b, t, q, e, !codes);
                    fence_async();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(bar(bars.dec_full[ds]));
                        // (only now: the codes have arrived in registers, not merely been asked for)
                        if (codes) mbar_arrive(bar(bars.raw_empty[rs]));
                    }
                    g += kGroups;
                }
            }
            seq += g1 - g0;
            if (codes) raws += g1 - g0;
        }
    } else if (warp >= kFirstOut) {
        // ---------------------------------------------------------------------------------------- out
        const int q = warp & 3;
        const int kl = 32 * q + lane;
        const uint32_t quarter = tmem + ((uint32_t)(q * 32) << 16);
        Acc a(chunks > 1);
        auto release = [&] {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(bars.acc_empty[a.slot]));
            a.next();
        };
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles, n0 = (u - kt * p.n_tiles) * p.n_tile;
            for (int ch = 0; ch < chunks && ok; ++ch) {
                ok = mbar_wait(bar(bars.acc_full[a.slot]), a.phase, abort_flag, &g_status, 64);
                fence_after();
                if (chunks == 1) break;
                add_part(quarter, 0, p.n_tile, ch == 0);
                release();
            }
            const uint32_t from = chunks > 1 ? quarter + 256 : quarter + 256 * a.slot;
            const bool sums = kt == p.k_tiles;  // db: every row of the accumulator is the same
            const int k = kt * kTileK + kl;
            const int n_end = min(p.n_tile, p.n - n0);
            float *part = reinterpret_cast<float *>(smem);  // [n_tile][128] of this CTA (share > 1: the rings are done with)
            for (int j = 0; j < p.n_tile; j += 32) {
                int raw[32];
                tmem_ld32(from + j, raw);
                tmem_wait_ld();
                if (share > 1) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) part[(j + i) * 128 + kl] = __int_as_float(raw[i]);
                } else if (sums ? kl == 0 : k < p.k) {
                    void *base = sums ? p.db : p.dw;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (j + i >= n_end) break;
                        const long long at = sums ? n0 + j + i : (long long)(n0 + j + i) * p.ld_dw + k;
                        float v = __int_as_float(raw[i]);
                        if (p.accumulate) v += load_out(p, base, at);
                        store_out(p, base, at, v);
                    }
                }
            }
            if (chunks == 1) release();
        }
    }
    if (share > 1) {  // one tile a cluster: every CTA adds up its share of the columns, four values a thread and a part's
                      // loads all in flight (distributed shared memory answers in about a microsecond)
        cg::this_cluster().sync();
        if (first < p.tiles) {
            const int kt = first / p.n_tiles, n0 = (first - kt * p.n_tiles) * p.n_tile;
            const bool sums = kt == p.k_tiles;
            const int n_end = min(p.n_tile, p.n - n0), k_end = sums ? 1 : min(kTileK, p.k - kt * kTileK);
            void *base = sums ? p.db : p.dw;
            float4 *part = reinterpret_cast<float4 *>(smem);
            for (int i = rank * kThreads + (int)threadIdx.x; i < n_end * (kTileK / 4); i += share * kThreads) {
                const int j = i / (kTileK / 4), kl = i % (kTileK / 4) * 4;
                if (kl >= k_end) continue;
                float4 x[kMaxShare];
#pragma unroll
                for (int c = 0; c < kMaxShare; ++c)
                    if (c < share) x[c] = *cg::this_cluster().map_shared_rank(&part[i], c);
                float v[4] = {};
#pragma unroll
                for (int c = 0; c < kMaxShare; ++c)
                    if (c < share) {
                        v[0] += x[c].x;
                        v[1] += x[c].y;
                        v[2] += x[c].z;
                        v[3] += x[c].w;
                    }
#pragma unroll
                for (int l = 0; l < 4; ++l)
                    if (kl + l < k_end) {
                        const long long at = sums ? n0 + j : (long long)(n0 + j) * p.ld_dw + kt * kTileK + kl + l;
                        store_out(p, base, at, p.accumulate ? v[l] + load_out(p, base, at) : v[l]);
                    }
            }
        }
        cg::this_cluster().sync();
    }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
    fence_before();
    __syncthreads();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// Many tiles: pairs of CTAs on tiles of 256 values of k x 256 channels.  A CTA decodes its 128 values of k and loads 128
// channels of dy; an instruction of the pair takes both CTAs' halves of dy, so that a CTA moves 40 KB a stage through its
// shared memory instead of 56, and 24 KB instead of 40 from L2.  Decoding is a chain of some 700 cycles a stage (wait,
// load, about 100 instructions, store, fence): two groups of eight warps take stages in turn.
constexpr int kPairTile = 256;
constexpr int kPairRaw = 4, kPairDec = 5, kPairDy = 5, kPairDyBytes = 2 * 128 * kTokens;
constexpr int kPairOut = 8, kPairThreads = 32 * (4 + kGroups * kConvWarps + kPairOut);
constexpr size_t kPairSmem = 1024 + kPairRaw * kRawBytes + kPairDec * kDecBytes + kPairDy * kPairDyBytes;

// The writing role of a pair's CTA (kPairOut warps, `warp` among them): parts are added up, tiles written.
template <typename T>
__device__ __forceinline__ void write_pair_tiles(const GradArgs &p, uint64_t *acc_full, uint64_t *acc_empty, uint32_t tmem, int warp, int lane,
                                                 int rank, int first, int stride, int chunks, volatile int *abort_flag)
{
    bool ok = true;
    auto bar = [](uint64_t &b) { return smem_u32(&b); };
    const int q = warp & 3, j0 = warp / 4 * (kPairTile / 2), j1 = j0 + kPairTile / 2;  // a quarter of tensor memory, a half of the columns
    const uint32_t quarter = tmem + ((uint32_t)(q * 32) << 16), total = quarter + 256;
    Acc a(chunks > 1);
    for (int u = first; u < p.tiles && ok; u += stride) {
        const int kt = u / p.n_tiles, n0 = (u - kt * p.n_tiles) * kPairTile;
        const bool sums = kt == p.k_tiles;  // db: every row of the accumulator is the same
        const int k = kt * kPairTile + 128 * rank + 32 * q + lane;
        const bool mine = sums ? rank == 0 && q == 0 && lane == 0 : k < p.k;
        const int n_end = min(kPairTile, p.n - n0);
        void *base = sums ? p.db : p.dw;
        const long long at0 = sums ? n0 : (long long)n0 * p.ld_dw + k, step = sums ? 1 : p.ld_dw;
        auto release = [&] {
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_pair(peer_addr(bar(acc_empty[a.slot]), 0));
            a.next();
        };
        for (int ch = 0; ch < chunks && ok; ++ch) {
            ok = mbar_wait(bar(acc_full[a.slot]), a.phase, abort_flag, &g_status, 64);
            fence_after();
            if (chunks == 1) break;
            add_part(quarter, j0, j1, ch == 0);
            release();
        }
        const uint32_t from = chunks > 1 ? total : quarter + 256 * a.slot;
        for (int j = j0; j < j1; j += 16) {
            int raw[16];
            tmem_ld16(from + j, raw);
            tmem_wait_ld();
            const int rows = mine ? n_end - j : 0;
            if (p.out_dtype == ACCERL_F32) {
                float *at = static_cast<float *>(base) + at0 + j * step;
                if (p.accumulate) {
                    float old[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) old[i] = i < rows ? at[i * step] : 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) raw[i] = __float_as_int(__int_as_float(raw[i]) + old[i]);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i < rows) *at = __int_as_float(raw[i]);
                    at += step;
                }
            } else {
                T *at = static_cast<T *>(base) + at0 + j * step;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    if (i < rows) *at = from_float<T>(__int_as_float(raw[i]));
                    at += step;
                }
            }
        }
        if (chunks == 1) release();
    }
}

struct __align__(8) PairBars {
    uint64_t raw_full[kPairRaw], raw_empty[kPairRaw], dec_full[kPairDec], dec_empty[kPairDec], dy_full[kPairDy], dy_empty[kPairDy],
        acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort_flag;
};

template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1)
weight_grad_pair_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_dy,
                        const __grid_constant__ GradArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ PairBars bars;
    namespace cg = cooperative_groups;
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t raw0 = smem_u32(smem), dec0 = raw0 + kPairRaw * kRawBytes, dy0 = dec0 + kPairDec * kDecBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cg::this_cluster().block_rank();
    const int stages = (p.tokens + kTokens - 1) / kTokens;
    const int chunks = chunks_of(p.out_dtype, stages);
    const int first = (int)blockIdx.x >> 1, stride = (int)gridDim.x >> 1;
    volatile int *abort_flag = &bars.abort_flag;
    auto bar = [](uint64_t &b) { return smem_u32(&b); };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPairRaw; ++i) {
            mbar_init(bar(bars.raw_full[i]), 1);
            mbar_init(bar(bars.raw_empty[i]), kConvWarps);
        }
        for (int i = 0; i < kPairDec; ++i) {
            mbar_init(bar(bars.dec_full[i]), 2 * kConvWarps);  // the first CTA's: the warps of both
            mbar_init(bar(bars.dec_empty[i]), 1);
        }
        for (int i = 0; i < kPairDy; ++i) {
            mbar_init(bar(bars.dy_full[i]), 1);  // the first CTA's: the loads of both
            mbar_init(bar(bars.dy_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(bars.acc_full[i]), 1);
            mbar_init(bar(bars.acc_empty[i]), 2 * kPairOut);  // the first CTA's: the writing warps of both
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();
    fence_after();
    const uint32_t tmem = bars.tmem;
    bool ok = true;

    if (warp == 0) {
        // ------------------------------------------------------------------------------ loads of codes
        Ring<kPairRaw> r;
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles;
            for (int g = 0; g < stages && ok && kt < p.k_tiles; ++g) {
                ok = mbar_wait(bar(bars.raw_empty[r.slot]), r.phase ^ 1, abort_flag, &g_status, 1);
                if (ok && elect_one()) {
                    mbar_expect_tx(bar(bars.raw_full[r.slot]), kRawBytes);
                    tma_load_2d(raw0 + r.slot * kRawBytes, &map_q, kt * kPairTile + 128 * rank, g * kTokens, bar(bars.raw_full[r.slot]));
                }
                __syncwarp();
                r.next();
            }
        }
    } else if (warp == 2) {
        // --------------------------------------------------------------------------------- loads of dy
        Ring<kPairDy> d;
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int n0 = u % p.n_tiles * kPairTile + 128 * rank;
            for (int g = 0; g < stages && ok; ++g) {
                ok = mbar_wait(bar(bars.dy_empty[d.slot]), d.phase ^ 1, abort_flag, &g_status, 2);
                if (ok && elect_one()) {
                    const uint32_t full = peer_addr(bar(bars.dy_full[d.slot]), 0);
                    if (rank == 0) mbar_expect_tx(bar(bars.dy_full[d.slot]), 2 * kPairDyBytes);
#pragma unroll
                    for (int b = 0; b < 2; ++b)
                        tma_load_2d_pair(dy0 + d.slot * kPairDyBytes + b * kTokens * 128, &map_dy, (n0 + 64 * b) * 2, g * kTokens, full);
                }
                __syncwarp();
                d.next();
            }
        }
    } else if (warp == 1 && rank == 0) {
        // ------------------------------------------------------------------------------ tensor core
        constexpr uint32_t kType = std::is_same<T, __half>::value ? 0u : 1u;
        constexpr uint32_t idesc = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 15) | (1u << 16) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
        Ring<kPairDec> c;
        Ring<kPairDy> d;
        Acc a(chunks > 1);
        for (int u = first; u < p.tiles && ok; u += stride) {
            for (int ch = 0; ch < chunks && ok; ++ch) {
                const int g0 = (int)((long long)stages * ch / chunks), g1 = (int)((long long)stages * (ch + 1) / chunks);
                ok = mbar_wait(bar(bars.acc_empty[a.slot]), a.phase ^ 1, abort_flag, &g_status, 4);
                fence_after();
                for (int g = g0; g < g1 && ok; ++g) {
                    ok = mbar_wait(bar(bars.dec_full[c.slot]), c.phase, abort_flag, &g_status, 8);
                    if (ok) ok = mbar_wait(bar(bars.dy_full[d.slot]), d.phase, abort_flag, &g_status, 8);
                    fence_after();
                    if (ok && elect_one()) {
                        const uint64_t ad = mn_desc(dec0 + c.slot * kDecBytes), bd = mn_desc(dy0 + d.slot * kPairDyBytes);
#pragma unroll
                        for (int ks = 0; ks < kTokens / 16; ++ks)
                            mma_f16_pair(tmem + 256 * a.slot, ad + ks * (2048 >> 4), bd + ks * (2048 >> 4), idesc, (uint32_t)((g - g0) | ks));
                        mma_commit_pair(bar(bars.dec_empty[c.slot]));
                        mma_commit_pair(bar(bars.dy_empty[d.slot]));
                        if (g == g1 - 1) mma_commit_pair(bar(bars.acc_full[a.slot]));
                    }
                    __syncwarp();
                    c.next();
                    d.next();
                }
                a.next();
            }
        }
    } else if (warp >= 4 && warp < 4 + kGroups * kConvWarps) {
        // ------------------------------------------------------------------------------------ decoding
        const int group = (warp - 4) / kConvWarps, w = (warp - 4) % kConvWarps;
        const int b = w & 3, t = (w >> 2) * 32 + lane;  // block of 32 values, token of the stage
        int seq = 0, raws = 0;                          // stages so far, of the CTA; those with codes
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles;
            const bool codes = kt < p.k_tiles;
            const int col = kt * kPairTile + 128 * rank + 32 * b;
            const bool in = codes && col < p.cols32;
            const uint8_t *e_at = p.e + col / 32 + (long long)t * p.ld_e;
            const long long e_step = (long long)kTokens * p.ld_e;
            // this group's stages of the tile
            const int g_first = (group - seq % kGroups + kGroups) % kGroups;
            auto exponent = [&](int g) { return in && g < stages && g * kTokens + t < p.tokens ? (int)__ldg(e_at + g * e_step) : 127; };
            int ahead[kAhead / kGroups];  // a load takes as long as some stages
#pragma unroll
            for (int i = 0; i < kAhead / kGroups; ++i) ahead[i] = exponent(g_first + kGroups * i);
            for (int g = g_first; g < stages && ok;) {
#pragma unroll
                for (int i = 0; i < kAhead / kGroups; ++i) {  // (unrolled: a value on its way is not to be moved)
                    if (g >= stages || !ok) break;
                    const int e = ahead[i];
                    ahead[i] = exponent(g + kAhead);
                    const int n = seq + g, rs = (raws + g) % kPairRaw, ds = n % kPairDec;
                    uint32_t q[8] = {};
                    if (codes) {
                        ok = mbar_wait(bar(bars.raw_full[rs]), (uint32_t)((raws + g) / kPairRaw & 1), abort_flag, &g_status, 16);
                        load_codes<T>(raw0 + rs * kRawBytes, b, t, q);
                    }
                    if (ok) ok = mbar_wait(bar(bars.dec_empty[ds]), (uint32_t)(n / kPairDec & 1) ^ 1, abort_flag, &g_status, 32);
                    ok = __all_sync(0xffffffffu, ok);
                    put_values<T>(dec0 + ds * kDecBytes, b, t, q, e, !codes);
                    fence_async();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive_pair(peer_addr(bar(bars.dec_full[ds]), 0));
                        // (only now: the codes have arrived in registers, not merely been asked for)
                        if (codes) mbar_arrive(bar(bars.raw_empty[rs]));
                    }
                    g += kGroups;
                }
            }
            seq += stages;
            if (codes) raws += stages;
        }
    } else if (warp >= 4 + kGroups * kConvWarps) {
        // ---------------------------------------------------------------------------------------- out
        write_pair_tiles<T>(p, bars.acc_full, bars.acc_empty, tmem, warp - (4 + kGroups * kConvWarps), lane, rank, first, stride, chunks, abort_flag);
    }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
    __syncwarp();
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();  // no barrier of a CTA is signalled once it has gone
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// The same from a checkpoint that has been read back (ckpt_load) into 16-bit rows: both operands come by TMA.  Every tile
// column of channels decodes a checkpoint anew, and decoding, not the tensor cores, bounds the kernel above (303 us for
// 8192 x 4096 x 4096, of which the tensor cores need 190); reading it back once costs 3 bytes a value, about what a
// 256-wide tile column takes on the tensor cores.  So from five tile columns on it is read back first.
constexpr int kPlainStages = 6, kPlainStage = kDecBytes + kPairDyBytes, kPlainThreads = 32 * (kPairOut + 4);
constexpr size_t kPlainSmem = 1024 + kDecBytes + kPlainStages * kPlainStage;

template <typename T>
__global__ void __launch_bounds__(kPlainThreads, 1)
weight_grad_plain_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_dy,
                         const __grid_constant__ GradArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ struct {
        uint64_t full[kPlainStages], empty[kPlainStages], acc_full[2], acc_empty[2];
        uint32_t tmem;
        int abort_flag;
    } bars;
    namespace cg = cooperative_groups;
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t ones = smem_u32(smem), ring = ones + kDecBytes;  // the operand of db; the stages
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cg::this_cluster().block_rank();
    const int stages = (p.tokens + kTokens - 1) / kTokens;
    const int chunks = chunks_of(p.out_dtype, stages);
    const int first = (int)blockIdx.x >> 1, stride = (int)gridDim.x >> 1;
    volatile int *abort_flag = &bars.abort_flag;
    auto bar = [](uint64_t &b) { return smem_u32(&b); };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPlainStages; ++i) {
            mbar_init(bar(bars.full[i]), 1);  // the first CTA's: the loads of both
            mbar_init(bar(bars.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(bars.acc_full[i]), 1);
            mbar_init(bar(bars.acc_empty[i]), 2 * kPairOut);  // the first CTA's: the writing warps of both
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = threadIdx.x; i < kDecBytes / 16; i += kPlainThreads)
        sts16(ones + 16 * i, make_uint4(Decode<T>::kOnes, Decode<T>::kOnes, Decode<T>::kOnes, Decode<T>::kOnes));
    fence_async();
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();
    fence_after();
    const uint32_t tmem = bars.tmem;
    bool ok = true;
    if (warp == 0) {
        Ring<kPlainStages> r;
        for (int u = first; u < p.tiles && ok; u += stride) {
            const int kt = u / p.n_tiles, n0 = (u - kt * p.n_tiles) * kPairTile + 128 * rank;
            const bool codes = kt < p.k_tiles;
            for (int g = 0; g < stages && ok; ++g) {
                ok = mbar_wait(bar(bars.empty[r.slot]), r.phase ^ 1, abort_flag, &g_status, 1);
                if (ok && elect_one()) {
                    const uint32_t full = peer_addr(bar(bars.full[r.slot]), 0), at = ring + r.slot * kPlainStage;
                    if (rank == 0) mbar_expect_tx(bar(bars.full[r.slot]), codes ? 2 * kPlainStage : 2 * kPairDyBytes);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (codes) tma_load_2d_pair(at + b * kTokens * 128, &map_x, (kt * kPairTile + 128 * rank + 64 * b) * 2, g * kTokens, full);
                        tma_load_2d_pair(at + kDecBytes + b * kTokens * 128, &map_dy, (n0 + 64 * b) * 2, g * kTokens, full);
                    }
                }
                __syncwarp();
                r.next();
            }
        }
    } else if (warp == 1 && rank == 0) {
        constexpr uint32_t kType = std::is_same<T, __half>::value ? 0u : 1u;
        constexpr uint32_t idesc = (1u << 4) | (kType << 7) | (kType << 10) | (1u << 15) | (1u << 16) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
        Ring<kPlainStages> r;
        Acc a(chunks > 1);
        for (int u = first; u < p.tiles && ok; u += stride) {
            const bool codes = u / p.n_tiles < p.k_tiles;
            for (int ch = 0; ch < chunks && ok; ++ch) {
                const int g0 = (int)((long long)stages * ch / chunks), g1 = (int)((long long)stages * (ch + 1) / chunks);
                ok = mbar_wait(bar(bars.acc_empty[a.slot]), a.phase ^ 1, abort_flag, &g_status, 4);
                fence_after();
                for (int g = g0; g < g1 && ok; ++g) {
                    ok = mbar_wait(bar(bars.full[r.slot]), r.phase, abort_flag, &g_status, 8);
                    fence_after();
                    if (ok && elect_one()) {
                        const uint32_t at = ring + r.slot * kPlainStage;
                        const uint64_t ad = mn_desc(codes ? at : ones), bd = mn_desc(at + kDecBytes);
#pragma unroll
                        for (int ks = 0; ks < kTokens / 16; ++ks)
                            mma_f16_pair(tmem + 256 * a.slot, ad + ks * (2048 >> 4), bd + ks * (2048 >> 4), idesc, (uint32_t)((g - g0) | ks));
                        mma_commit_pair(bar(bars.empty[r.slot]));
                        if (g == g1 - 1) mma_commit_pair(bar(bars.acc_full[a.slot]));
                    }
                    __syncwarp();
                    r.next();
                }
                a.next();
            }
        }
    } else if (warp >= 4) {
        write_pair_tiles<T>(p, bars.acc_full, bars.acc_empty, tmem, warp - 4, lane, rank, first, stride, chunks, abort_flag);
    }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
    __syncwarp();
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();  // no barrier of a CTA is signalled once it has gone
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// dy at rows of a multiple of 16 bytes, for the TMA
__global__ void __launch_bounds__(256) realign_kernel(const uint16_t *__restrict__ src, long long ld_src, uint16_t *__restrict__ dst, long long ld_dst,
                                                      int tokens, int n)
{
    for (long long t = blockIdx.y; t < tokens; t += gridDim.y)
        for (int i = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 8; i < n; i += (int)(gridDim.x * blockDim.x) * 8) {
            const uint16_t *row = src + t * ld_src + i;
            uint4 v;
            if (i + 8 <= n) {
                v = load16(row);
            } else {  // (bits, whichever type they are of)
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] = (i + 2 * k < n ? (uint32_t)row[2 * k] : 0u) | (i + 2 * k + 1 < n ? (uint32_t)row[2 * k + 1] << 16 : 0u);
                v = make_uint4(w[0], w[1], w[2], w[3]);
            }
            *reinterpret_cast<uint4 *>(dst + t * ld_dst + i) = v;
        }
}

long long padded_n(long long n) { return (n + 7) / 8 * 8; }

}  // namespace

cudaError_t weight_grad_status(int *out)  // (clears it)
{
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *out) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(int));
    return e;
}

}  // namespace accerl

using namespace accerl;

namespace {

// Which kernel, and what it needs beside its operands: sizes and dy's alignment decide.
struct Plan {
    bool pair = false, plain = false;
    int64_t dy_bytes = 0, x_bytes = 0;
};
Plan plan_of(const accerl_weight_grad_args *a)
{
    Plan r;
    const long long n_tiles = (a->n + kPairTile - 1LL) / kPairTile, k_tiles = (a->k + kPairTile - 1LL) / kPairTile;  // (whether db is wanted does not count: it is to change no bit of dw)
    r.pair = n_tiles * k_tiles >= 111;  // three tiles for every two pairs of a B200's 148 SMs
    r.plain = r.pair && n_tiles >= 5;
    if (((uintptr_t)a->dy & 15) || a->ld_dy % 8) r.dy_bytes = (2LL * a->tokens * padded_n(a->n) + 255) / 256 * 256;
    if (r.plain) r.x_bytes = (2LL * a->tokens * padded_n(a->k) + 255) / 256 * 256;
    return r;
}

}  // namespace

extern "C" int64_t accerl_ckpt_weight_grad_workspace(const accerl_weight_grad_args *a)
{
    if (!a || a->tokens < 1 || a->n < 1 || a->k < 1) return 0;
    const Plan plan = plan_of(a);
    return plan.dy_bytes + plan.x_bytes;
}

extern "C" accerl_status accerl_ckpt_weight_grad(const accerl_weight_grad_args *a, void *cuda_stream)
{
    if (!a || !a->dy || !a->q || !a->e || !a->dw) {
        set_error("ckpt_weight_grad: null argument");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->tokens < 1 || a->tokens >= kMostRows || a->n < 1 || a->k < 1 || a->k > (1 << 27) || a->n > (1 << 27) || (long long)a->n * a->k > (1LL << 40)) {
        set_error("ckpt_weight_grad: tokens, n and k must be positive, tokens below 2^31 - 2^16, n and k at most 2^27, n * k at most 2^40");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->dy_dtype == ACCERL_F32) {
        set_error("ckpt_weight_grad: dy must be bf16 or fp16");
        return ACCERL_ERR_UNSUPPORTED;
    }
    if (!good_dtype(a->dy_dtype) || (a->out_dtype != ACCERL_F32 && a->out_dtype != a->dy_dtype) ||
        (a->accumulate && a->out_dtype != ACCERL_F32)) {
        set_error("ckpt_weight_grad: dy is bf16 or fp16, dw and db fp32 or dy's type (fp32 to accumulate)");
        return ACCERL_ERR_INVALID_ARG;
    }
    const int cols32 = (a->k + 31) / 32 * 32, es = dtype_size(a->out_dtype);
    if (((uintptr_t)a->q & 15) || a->ld_q < cols32 || a->ld_q % 16 || a->ld_e < cols32 / 32) {
        set_error("ckpt_weight_grad: a checkpoint's q needs 16-byte alignment, ld_q >= %d (a multiple of 16) and ld_e >= %d", cols32, cols32 / 32);
        return ACCERL_ERR_INVALID_ARG;
    }
    if (((uintptr_t)a->dy & 1) || a->ld_dy < a->n || a->ld_dw < a->k || (((uintptr_t)a->dw | (uintptr_t)a->db) & (es - 1))) {
        set_error("ckpt_weight_grad: dy, dw or db is misaligned, or rows are closer than their length");
        return ACCERL_ERR_INVALID_ARG;
    }
    const int64_t need = accerl_ckpt_weight_grad_workspace(a);
    if (need && (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need)) {
        set_error("ckpt_weight_grad: the workspace needs %lld bytes, aligned to 256", (long long)need);
        return ACCERL_ERR_INVALID_ARG;
    }
    int device = 0, sm_count = 0;
    ACCERL_CUDA_TRY(cudaGetDevice(&device));
    ACCERL_CUDA_TRY(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const Plan plan = plan_of(a);
    const bool pair = plan.pair, copy = plan.dy_bytes > 0;
    const void *dy = copy ? a->workspace : a->dy;
    const long long ld_dy = copy ? padded_n(a->n) : a->ld_dy;
    void *x = static_cast<char *>(a->workspace) + plan.dy_bytes;
    CUtensorMap mq, md;
    accerl_status s = plan.plain ? tc_make_map(&mq, x, a->tokens, 2 * a->k, 2 * padded_n(a->k), kTokens, 128)
                                 : tc_make_map(&mq, a->q, a->tokens, cols32, a->ld_q, kTokens, 128);
    if (s == ACCERL_OK) s = tc_make_map(&md, dy, a->tokens, 2 * a->n, 2 * ld_dy, kTokens, 128);
    if (s != ACCERL_OK) return s;
    GradArgs p;
    p.e = a->e;
    p.dw = a->dw;
    p.db = a->db;
    p.ld_e = a->ld_e;
    p.ld_dw = a->ld_dw;
    p.tokens = a->tokens;
    p.n = a->n;
    p.k = a->k;
    p.out_dtype = a->out_dtype;
    p.accumulate = a->accumulate != 0;
    p.n_tile = pair ? kPairTile : std::min(256, (a->n + 63) / 64 * 64);
    // Tiles of 128 channels where four times those of 256 fit the chip: smaller parts to exchange, and clusters of fewer CTAs, which
    // find room more easily.  128 / 256 wide, tokens x channels x k, bf16 in a captured graph: 2047 x 256 x 2592 13.1 / 14.9 us,
    // 512 x 256 x 2592 9.8 / 11.9, 2048 x 1024 x 512 13.1 / 26.4, 300 x 300 x 900 11.9 / 15.0; but 2048 x 768 x 384 16.6 / 14.1 and, where
    // clusters have eight CTAs either way and twice as many do not run at once, 8192 x 256 x 1024 28.9 / 19.2.
    if (!pair && p.n_tile == 256 && ((long long)a->n + 255) / 256 * ((a->k + kTileK - 1) / kTileK) * 4 <= sm_count) p.n_tile = 128;
    p.n_tiles = (a->n + p.n_tile - 1) / p.n_tile;
    const int k_tile = pair ? kPairTile : kTileK;
    p.k_tiles = (a->k + k_tile - 1) / k_tile;
    p.cols32 = cols32;
    const long long tiles = (long long)p.n_tiles * (p.k_tiles + (a->db ? 1 : 0));
    if (tiles > (1 << 30)) {
        set_error("ckpt_weight_grad: n * k is too large");
        return ACCERL_ERR_INVALID_ARG;
    }
    p.tiles = (int)tiles;
    const int stages = (a->tokens + kTokens - 1) / kTokens;
    if ((tiles / std::max(1, sm_count / 2) + 1) * stages > (1 << 30)) {  // (a CTA counts its stages in an int)
        set_error("ckpt_weight_grad: tokens * n * k is too large");
        return ACCERL_ERR_INVALID_ARG;
    }
    // CTAs a tile of dw: the same whether db is wanted or not, and so the order of dw's sums.  As many as let db's tiles run beside
    // dw's (more do not pay without db either: not all clusters of three or more then run at once, 2048 x 768 x 768 takes 26.6 us
    // by fours, 16.4 by threes).  But two where dw's tiles alone leave room for two: db's tiles come second then (8192 x 1024 x 2304
    // with / without db 74 / 45 us by twos, 78 / 78 by ones; 2048 x 512 x 2304 30.7 / 20.5 and 26.7 / 26.7).
    const int dw_tiles = p.n_tiles * p.k_tiles, alone = sm_count / dw_tiles, with_db = sm_count / (dw_tiles + p.n_tiles);
    const int share = pair ? 2 : std::max(1, std::min({kMaxShare, alone == 2 ? alone : with_db, stages / 2}));
    const unsigned grid = pair        ? 2u * (unsigned)std::min(p.tiles, sm_count / 2)
                          : share > 1 ? (unsigned)(p.tiles * share) : (unsigned)std::min(p.tiles, sm_count);
    // (never less than a pair's CTA takes: these kernels hold all of tensor memory, and a cluster of which one CTA waits for
    // another kernel's cluster to give some up, and that for the first's other CTAs, would wait for good; with this much shared
    // memory no other cluster that uses tensor memory fits beside one of them)
    const size_t smem = plan.plain ? kPlainSmem
                        : pair     ? kPairSmem
                                   : std::max(kPairSmem, 1024 + kRaw * kRawBytes + kDec * kDecBytes + (size_t)kDy * p.n_tile * 2 * kTokens);
    if (copy) {
        const dim3 grid((unsigned)std::min((a->n + 2047) / 2048, 1024), (unsigned)std::min(a->tokens, 65535));
        realign_kernel<<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(a->dy), a->ld_dy, static_cast<uint16_t *>(a->workspace),
                                             padded_n(a->n), a->tokens, a->n);
        ACCERL_CUDA_TRY(cudaGetLastError());
    }
    if (plan.plain) {
        s = accerl_ckpt_load(a->q, a->ld_q, a->e, a->ld_e, a->tokens, a->k, x, padded_n(a->k), a->dy_dtype, cuda_stream);
        if (s != ACCERL_OK) return s;
    }
    const bool half = a->dy_dtype == ACCERL_F16;
    const auto kernel = plan.plain ? (half ? weight_grad_plain_kernel<__half> : weight_grad_plain_kernel<__nv_bfloat16>)
                        : pair ? (half ? weight_grad_pair_kernel<__half> : weight_grad_pair_kernel<__nv_bfloat16>)
                             : (half ? weight_grad_kernel<__half> : weight_grad_kernel<__nv_bfloat16>);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)share;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(plan.plain ? kPlainThreads : pair ? kPairThreads : kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ACCERL_CUDA_TRY(allow_smem((const void *)kernel, smem));
    ACCERL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mq, md, p));
    return ACCERL_OK;
}
