// int8 layers on activations that are quantised per token (one scale a token, one a channel).
//
// quant_rows_kernel: a warp or a CTA per row finds max |x| and rounds the row to int8; bound by HBM (or by the latency
// of one row).  A row stays in registers between its maximum and its rounding.  q = rint(x / s) is a division rounded
// to fp32; it is computed as x * (1 / s) and the division is done only where that product lies so near to a tie that
// its error (below 127 * 2^-22) could matter.
//
// (8192 rows of 4096 bf16: 23 us, 4.4 TB/s; of 3136 fp32: 27 us, 4.8 TB/s.)
//
// linear_token_kernel: the product for one token.  linear_few_kernel: for some.  Channels are the M of the tensor-core
// instructions and tokens their N, so that few tokens need few columns and the weights, which bound this case, stream
// through shared memory once (24 tokens, 4096 x 14336: 17 us with the quantiser in a captured graph, 7 of them the weights).  K is split over the CTAs of a cluster until the chip is covered; their int32 partial sums are added
// through distributed shared memory (integers: any order gives the same bits).  linear_pair_kernel: for many.
#include <cooperative_groups.h>

#include <algorithm>

#include "learn.cuh"
#include "tc_image.cuh"

namespace accerl {

namespace {

__device__ int g_status;  // of this file's bounded waits

// ------------------------------------------------------------------------------------------- quantisation
struct QuantArgs {
    const void *x;
    int8_t *q;
    float *scale;
    long long ld_x, ld_q, rows;
    int cols;
};

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

constexpr float kRounder = 12582912.f;  // 1.5 * 2^23: adding it rounds to an integer, in the low byte of the sum

__device__ __forceinline__ uint32_t low_bytes(float a, float b, float c, float d)
{
    return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

// by the definition's own division (rare: out of line, so that the loops stay in the instruction cache)
__device__ __noinline__ uint32_t divided4(float a, float b, float c, float d, float s)
{
    auto code = [&](float v) { return fminf(fmaxf(rintf(__fdiv_rn(v, s)), -127.f), 127.f) + kRounder; };
    return low_bytes(code(a), code(b), code(c), code(d));
}

// four values to four int8; `exact`: the scale's reciprocal is not to be trusted
__device__ __forceinline__ uint32_t quantised4(const float *v, float s, float inv, bool exact)
{
    float q[4], d = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float t = v[k] * inv;
        q[k] = t + kRounder;
        d = fmaxf(d, fabsf(t - (q[k] - kRounder)));
    }
    if (exact || d > 0.49996f) return divided4(v[0], v[1], v[2], v[3], s);
    return low_bytes(q[0], q[1], q[2], q[3]);
}

// what a row's largest magnitude makes of it
struct Scale {
    float s, inv;
    bool zero, exact;
    __device__ __forceinline__ explicit Scale(uint32_t top)
    {
        const bool broken = top >= 0x7f800000u;  // an infinity or a NaN
        s = broken ? NAN : __fdiv_rn(__uint_as_float(top), 127.f);
        zero = broken || s == 0.f;
        exact = s < 1e-30f;  // (tiny scales: 1 / s may overflow, s itself be coarse)
        inv = zero || exact ? 0.f : __fdiv_rn(1.f, s);
    }
};

template <typename T>
__device__ __forceinline__ void quantise_piece(const QuantArgs &p, int8_t *q_row, int first, const uint4 &raw, float s, float inv,
                                               bool exact, bool zero)
{
    constexpr int V = Row<T>::kVec;
    if (first >= p.cols) return;
    float v[V];
    unpack<T>(raw, v);
    uint32_t w[V / 4];
#pragma unroll
    for (int j = 0; j < V / 4; ++j) w[j] = zero ? 0u : quantised4(v + 4 * j, s, inv, exact);
    if (first + V <= p.cols) {
        if constexpr (V == 8) *reinterpret_cast<uint2 *>(q_row + first) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t *>(q_row + first) = w[0];
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (first + k < p.cols) q_row[first + k] = (int8_t)(w[k / 4] >> 8 * (k & 3));
    }
}

// WARP: a warp per row, four rows a CTA; else a CTA per row.  NV pieces of 16 bytes a thread stay in registers; a row
// that has more (LOOP) is read twice.  ALIGNED: rows at multiples of 16 bytes.
template <typename T, int NV, bool WARP, bool LOOP, bool ALIGNED>
__global__ void __launch_bounds__(WARP ? 128 : 1024) quant_rows_kernel(const __grid_constant__ QuantArgs p)
{
    constexpr int V = Row<T>::kVec;
    __shared__ uint32_t s_top[32];
    // (the launch before is done with everything it reads and writes; and the product, which fetches its weights as soon as it
    // starts, starts only after that)
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long row = WARP ? (long long)blockIdx.x * 4 + warp : (long long)blockIdx.x;
    if (WARP && row >= p.rows) return;
    const T *x = static_cast<const T *>(p.x) + row * p.ld_x;
    int8_t *q = p.q + row * p.ld_q;
    const int lanes = WARP ? 32 : (int)blockDim.x, step = lanes * V, first = (WARP ? lane : (int)threadIdx.x) * V;
    uint4 raw[NV];
    uint32_t top = 0;
    auto take = [&](const uint4 &piece) {
        float v[V];
        unpack<T>(piece, v);
#pragma unroll
        for (int k = 0; k < V; ++k) top = max(top, magnitude(v[k]));
    };
#pragma unroll
    for (int i = 0; i < NV; ++i) raw[i] = load_piece<T, ALIGNED>(x, first + i * step, p.cols, 0.f);
#pragma unroll
    for (int i = 0; i < NV; ++i) take(raw[i]);
    if constexpr (LOOP)
        for (int at = first + NV * step; at < p.cols; at += step) take(load_piece<T, ALIGNED>(x, at, p.cols, 0.f));
    top = __reduce_max_sync(0xffffffffu, top);
    if constexpr (!WARP) {
        if (lane == 0) s_top[warp] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, lane < lanes / 32 ? s_top[lane] : 0u);
    }
    const Scale sc(top);
    if (first == 0) p.scale[row] = sc.s;
#pragma unroll
    for (int i = 0; i < NV; ++i) quantise_piece<T>(p, q, first + i * step, raw[i], sc.s, sc.inv, sc.exact, sc.zero);
    if constexpr (LOOP)
        for (int at = first + NV * step; at < p.cols; at += step)
            quantise_piece<T>(p, q, at, load_piece<T, ALIGNED>(x, at, p.cols, 0.f), sc.s, sc.inv, sc.exact, sc.zero);
}

template <typename T, bool ALIGNED>
cudaError_t launch_quant(const QuantArgs &p, int sm_count, cudaStream_t st)
{
    const long long pieces = ((long long)p.cols + Row<T>::kVec - 1) / Row<T>::kVec;
    // Few rows: two pieces a thread, the shortest chain.  Many: four, since what a thread does once for its row (two
    // divisions, the reduction) is some hundred instructions (8192 x 4096 bf16: 22.7 us; with eight, which leaves fewer
    // warps on an SM, 25.4; 8192 x 3136 fp32: 26.8 either way).
    const bool few = p.rows < 2 * sm_count;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (!few && pieces <= 32 * 8) {
        cfg.gridDim = dim3((unsigned)((p.rows + 3) / 4));
        cfg.blockDim = dim3(128);
        return cudaLaunchKernelEx(&cfg, quant_rows_kernel<T, 8, true, false, ALIGNED>, p);
    }
    const long long want = few ? (pieces + 1) / 2 : (pieces + 3) / 4;
    const int threads = (int)std::min<long long>(1024, (want + 31) / 32 * 32);
    const auto kernel = threads * 2 >= pieces   ? quant_rows_kernel<T, 2, false, false, ALIGNED>
                        : threads * 4 >= pieces ? quant_rows_kernel<T, 4, false, false, ALIGNED>
                                                : quant_rows_kernel<T, 8, false, true, ALIGNED>;
    cfg.gridDim = dim3((unsigned)p.rows);
    cfg.blockDim = dim3((unsigned)threads);
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

cudaError_t launch_quant(const QuantArgs &p, int dtype, int sm_count, cudaStream_t st)
{
    return with_dtype(dtype, [&](auto v) {
        using T = decltype(v);
        return rows_aligned(p.x, p.ld_x, dtype) ? launch_quant<T, true>(p, sm_count, st) : launch_quant<T, false>(p, sm_count, st);
    });
}

// ------------------------------------------------------------------------------------------------ product
struct LinearArgs {
    const float *x_scale, *w_scale, *bias;
    void *y;
    long long ld_y;
    int tokens, n, k, y_dtype, relu;
    int chunks;  // of 128 bytes along K
    int stages;
};

__device__ __forceinline__ void store_y(const LinearArgs &p, int t, int n, float v)
{
    const long long at = (long long)t * p.ld_y + n;
    if (p.y_dtype == ACCERL_F32) static_cast<float *>(p.y)[at] = v;
    else if (p.y_dtype == ACCERL_BF16) static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p.y)[at] = __float2half_rn(v);
}

__device__ __forceinline__ float at_least(float v, float floor)  // (a NaN stays one)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(v), "f"(floor));
    return m;
}

// One token, of at most 64 KB once quantised: a warp takes a channel at a time, whose weights it has asked for before the CTA
// quantises the token (every CTA all of it, from L2) into shared memory; four products an instruction.  There is one
// product a byte of weights, and what counts is latency: no second launch, no tensor memory to set up, no cluster to wait
// for.  4096 x 4096 in a captured graph 5.6 us, with the kernels below 8.6, and 14 us against 8.7 with four tokens done
// this way: from two tokens on the tensor cores take them.
constexpr int kTokenThreads = 256, kTokenAhead = 8;  // pieces of 16 bytes of a channel in flight, a lane

struct TokenArgs {
    const void *x;
    const float *x_scale;
    const int8_t *w;
    long long ld_w;
    int room;  // of the token in shared memory: k rounded up to 512
};

template <typename XT>
__global__ void __launch_bounds__(kTokenThreads, 4)
linear_token_kernel(const __grid_constant__ LinearArgs p, const __grid_constant__ TokenArgs a)
{
    extern __shared__ __align__(16) uint8_t s_x[];
    __shared__ uint32_t s_top[kTokenThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = kTokenThreads / 32;
    const int channels = (int)gridDim.x * warps;
    int n = (int)blockIdx.x * warps + warp;
    uint4 w[kTokenAhead];
    auto ask = [&](int channel, int k0) {  // the pieces from k0 on
        const int8_t *row = a.w + (long long)channel * a.ld_w;
#pragma unroll
        for (int i = 0; i < kTokenAhead; ++i) {
            const int k = k0 + 512 * i + 16 * lane;
            w[i] = channel < p.n && k < p.k ? __ldcs(reinterpret_cast<const uint4 *>(row + k)) : make_uint4(0, 0, 0, 0);
        }
    };
    ask(n, 0);
    uint32_t *out = reinterpret_cast<uint32_t *>(s_x);
    float scale;
    if constexpr (sizeof(XT) == 1) {
        const int8_t *x = static_cast<const int8_t *>(a.x);
        for (int i = threadIdx.x; i < a.room / 4; i += kTokenThreads) {
            uint32_t v = 0;
            if (4 * i + 3 < p.k) v = reinterpret_cast<const uint32_t *>(x)[i];
            else
                for (int j = 0; j < 4; ++j)
                    if (4 * i + j < p.k) v |= (uint32_t)(uint8_t)x[4 * i + j] << 8 * j;
            out[i] = v;
        }
        scale = a.x_scale[0];
    } else {
        constexpr int V = Row<XT>::kVec;
        const XT *x = static_cast<const XT *>(a.x);
        uint32_t top = 0;
#pragma unroll 4
        for (int k = (int)threadIdx.x * V; k < p.k; k += kTokenThreads * V) {
            float v[V];
            unpack<XT>(load_piece<XT>(x, k, p.k, 0.f), v);
#pragma unroll
            for (int j = 0; j < V; ++j) top = max(top, magnitude(v[j]));
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) s_top[warp] = top;
        __syncthreads();
        top = __reduce_max_sync(0xffffffffu, s_top[lane % warps]);
        const Scale sc(top);
        scale = sc.s;
#pragma unroll 2
        for (int k = (int)threadIdx.x * V; k < a.room; k += kTokenThreads * V) {
            float v[V];
            unpack<XT>(load_piece<XT>(x, k, p.k, 0.f), v);
#pragma unroll
            for (int j = 0; j < V / 4; ++j) out[k / 4 + j] = sc.zero ? 0u : quantised4(v + 4 * j, sc.s, sc.inv, sc.exact);
        }
    }
    __syncthreads();
    for (; n < p.n; n += channels) {
        const float ws = p.w_scale[n], bias = p.bias ? p.bias[n] : 0.f;
        int acc = 0;
        for (int k0 = 0; k0 < p.k; k0 += 512 * kTokenAhead) {
            if (k0) ask(n, k0);
#pragma unroll
            for (int i = 0; i < kTokenAhead; ++i) {
                const int k = k0 + 512 * i;
                if (k >= p.k) break;
                const uint4 v = *reinterpret_cast<const uint4 *>(s_x + k + 16 * lane);
                acc = __dp4a((int)w[i].x, (int)v.x, acc);
                acc = __dp4a((int)w[i].y, (int)v.y, acc);
                acc = __dp4a((int)w[i].z, (int)v.z, acc);
                acc = __dp4a((int)w[i].w, (int)v.w, acc);
            }
        }
        ask(n + channels, 0);
        const int sum = __reduce_add_sync(0xffffffffu, acc);
        if (lane == 0) store_y(p, 0, n, at_least(fmaf((float)sum, scale * ws, bias), p.relu ? 0.f : -INFINITY));
    }
}

// as many CTAs as the chip holds at most: 4 an SM, 3 beside long tokens
accerl_status launch_token(const accerl_linear_i8_args *a, const LinearArgs &p, int sm_count, cudaStream_t st)
{
    const TokenArgs t{a->x, a->x_scale, a->w, a->ld_w, (a->k + 511) / 512 * 512};
    const int warps = kTokenThreads / 32, resident = sm_count * std::min(4, 220 * 1024 / (t.room + 1024));
    const auto kernel = a->x_dtype == ACCERL_I8     ? linear_token_kernel<int8_t>
                        : a->x_dtype == ACCERL_F32  ? linear_token_kernel<float>
                        : a->x_dtype == ACCERL_BF16 ? linear_token_kernel<__nv_bfloat16>
                                                    : linear_token_kernel<__half>;
    ACCERL_CUDA_TRY(allow_smem((const void *)kernel, t.room));
    kernel<<<(unsigned)std::min((a->n + warps - 1) / warps, resident), kTokenThreads, (size_t)t.room, st>>>(p, t);
    ACCERL_CUDA_TRY(cudaGetLastError());
    return ACCERL_OK;
}

constexpr int kFewThreads = 192, kMaxStages = 8, kMaxShare = 8;

// One tile of 128 channels x NT tokens; the CTAs of a cluster share its K.
// Warps 0..3 drain the accumulator (and finish), warp 4 loads, warp 5 issues the tensor-core instructions.
template <int NT, typename T>
__global__ void __launch_bounds__(kFewThreads)
linear_few_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                  const __grid_constant__ LinearArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ struct {
        uint64_t full[kMaxStages], empty[kMaxStages], acc;
        uint32_t tmem;
        int abort_flag;
    } bars;
    __shared__ float s_ws[128], s_bias[128];
    __shared__ __align__(16) float s_xs[NT];
    namespace cg = cooperative_groups;
    constexpr int kStage = 128 * 128 + NT * 128, kCols = NT < 32 ? 32 : NT;
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem), full0 = smem_u32(&bars.full[0]), empty0 = smem_u32(&bars.empty[0]);
    const int warp = threadIdx.x >> 5;
    const int share = (int)cg::this_cluster().num_blocks(), rank = (int)cg::this_cluster().block_rank();
    const int n0 = (int)(blockIdx.x / (unsigned)share) * 128, t0 = (int)blockIdx.y * NT;
    const int c0 = (int)((long long)p.chunks * rank / share), c1 = (int)((long long)p.chunks * (rank + 1) / share);
    volatile int *abort_flag = &bars.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(full0 + 8 * s, 1);
            mbar_init(empty0 + 8 * s, 1);
        }
        mbar_init(smem_u32(&bars.acc), 1);
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"((uint32_t)kCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = bars.tmem;

    if (warp == 4) {
        // weights are not the previous launch's (the quantiser's) doing: the first stages' are on their way before it ends
        const int early = min(p.stages, c1 - c0);
        if (elect_one()) {
            for (int i = 0; i < early; ++i) {
                mbar_expect_tx(full0 + 8 * i, kStage);
                tma_load_2d(base + i * kStage, &map_w, (c0 + i) * 128, n0, full0 + 8 * i);
            }
        }
        __syncwarp();
        asm volatile("griddepcontrol.wait;" ::: "memory");
        bool ok = true;
        for (int i = 0; i < c1 - c0 && ok; ++i) {
            const int s = i % p.stages;
            if (i >= p.stages) ok = mbar_wait(empty0 + 8 * s, (uint32_t)((i / p.stages - 1) & 1), abort_flag, &g_status, 1);
            if (ok && elect_one()) {
                const uint32_t at = base + s * kStage;
                if (i >= early) {
                    mbar_expect_tx(full0 + 8 * s, kStage);
                    tma_load_2d(at, &map_w, (c0 + i) * 128, n0, full0 + 8 * s);
                }
                tma_load_2d(at + 128 * 128, &map_x, (c0 + i) * 128, t0, full0 + 8 * s);
            }
            __syncwarp();
        }
    } else if (warp == 5) {
        bool ok = true;
        for (int i = 0; i < c1 - c0 && ok; ++i) {
            const int s = i % p.stages;
            ok = mbar_wait(full0 + 8 * s, (uint32_t)((i / p.stages) & 1), abort_flag, &g_status, 8);
            fence_after();
            if (ok && elect_one()) {
                const uint64_t a = make_desc(base + s * kStage, 128), b = make_desc(base + s * kStage + 128 * 128, 128);
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) mma_i8(tmem, a + 2 * ks, b + 2 * ks, idesc_for(NT), (uint32_t)(i | ks));
                mma_commit(empty0 + 8 * s);
                if (i == c1 - c0 - 1) mma_commit(smem_u32(&bars.acc));
            }
            __syncwarp();
        }
    } else {
        // what the sums are to be multiplied with, while they are made
        const int n = n0 + (int)threadIdx.x;
        s_ws[threadIdx.x] = n < p.n ? p.w_scale[n] : 0.f;
        s_bias[threadIdx.x] = n < p.n && p.bias ? p.bias[n] : 0.f;
        asm volatile("griddepcontrol.wait;" ::: "memory");  // (the tokens' scales are the quantiser's)
        if ((int)threadIdx.x < NT) s_xs[threadIdx.x] = t0 + (int)threadIdx.x < p.tokens ? p.x_scale[t0 + threadIdx.x] : 0.f;
        asm volatile("bar.sync 1, 128;" ::: "memory");
        mbar_wait(smem_u32(&bars.acc), 0, abort_flag, &g_status, 16);
        fence_after();
    }
    const float floor = p.relu ? 0.f : -INFINITY;
    int *part = reinterpret_cast<int *>(smem);  // [NT][128]: every operand has been read
    if (warp < 4) {
        const int n = n0 + (int)threadIdx.x, have = n < p.n ? min(NT, p.tokens - t0) : 0;
        const float ws = s_ws[threadIdx.x], bias = s_bias[threadIdx.x];
        T *y = static_cast<T *>(p.y) + (long long)t0 * p.ld_y + n;
#pragma unroll
        for (int j = 0; j < NT / 16; ++j) {
            if (16 * j >= p.tokens - t0) break;
            int acc[16];
            tmem_ld16(tmem + ((uint32_t)(warp * 32) << 16) + 16 * j, acc);
            tmem_wait_ld();
            if (share > 1) {
#pragma unroll
                for (int i = 0; i < 16; ++i) part[(16 * j + i) * 128 + threadIdx.x] = acc[i];
            } else {
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 xs = *reinterpret_cast<const float4 *>(&s_xs[16 * j + i]);
                    const float sc[4] = {xs.x, xs.y, xs.z, xs.w};
#pragma unroll
                    for (int l = 0; l < 4; ++l) {
                        if (16 * j + i + l < have) *y = from_float<T>(at_least(fmaf((float)acc[i + l], sc[l] * ws, bias), floor));
                        y += p.ld_y;
                    }
                }
            }
        }
        fence_before();
    }
    if (share > 1) {
        cg::this_cluster().sync();
        const int4 *four = reinterpret_cast<const int4 *>(part);
        // four channels of a token a thread, the parts' loads all in flight (each answers in about a microsecond)
        for (int i = rank * kFewThreads + (int)threadIdx.x; i < min(NT, p.tokens - t0) * 32; i += share * kFewThreads) {
            int4 x[kMaxShare];
#pragma unroll
            for (int c = 0; c < kMaxShare; ++c)
                if (c < share) x[c] = *cg::this_cluster().map_shared_rank(&four[i], c);
            int acc[4] = {};
#pragma unroll
            for (int c = 0; c < kMaxShare; ++c)
                if (c < share) {
                    acc[0] += x[c].x;
                    acc[1] += x[c].y;
                    acc[2] += x[c].z;
                    acc[3] += x[c].w;
                }
            const int t = i / 32, n4 = i % 32 * 4;
            T *y = static_cast<T *>(p.y) + (long long)(t0 + t) * p.ld_y + n0 + n4;
#pragma unroll
            for (int l = 0; l < 4; ++l)
                if (n0 + n4 + l < p.n) y[l] = from_float<T>(at_least(fmaf((float)acc[l], s_xs[t] * s_ws[n4 + l], s_bias[n4 + l]), floor));
        }
        cg::this_cluster().sync();
    }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
    __syncthreads();
    if (warp == 5)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kCols) : "memory");
}

template <int NT>
accerl_status launch_few(const CUtensorMap &mw, const CUtensorMap &mx, LinearArgs &p, int sm_count, bool after_quant, cudaStream_t st)
{
    constexpr int kStage = 128 * 128 + NT * 128;
    p.stages = std::min(kMaxStages, 110 * 1024 / kStage);
    const size_t smem = 1024 + (size_t)p.stages * kStage;
    const int tiles = (p.n + 127) / 128, token_tiles = (p.tokens + NT - 1) / NT;
    int share = 1;
    while (share < kMaxShare && (long long)tiles * token_tiles * share < sm_count && p.chunks >= 4 * share) share *= 2;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)share;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(tiles * share), (unsigned)token_tiles);
    cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = after_quant ? 2 : 1;
    const auto kernel = p.y_dtype == ACCERL_F32    ? linear_few_kernel<NT, float>
                        : p.y_dtype == ACCERL_BF16 ? linear_few_kernel<NT, __nv_bfloat16>
                                                   : linear_few_kernel<NT, __half>;
    ACCERL_CUDA_TRY(allow_smem((const void *)kernel, smem));
    ACCERL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mw, mx, p));
    return ACCERL_OK;
}

// Many tokens: pairs of CTAs on tiles of 256 channels x 256 tokens, persistent.  A CTA holds 128 channels and 128 tokens of a
// stage (32 KB for 128 bytes of K) and 128 of the accumulator's rows: an instruction of the pair reads 8 KB of operands per
// SM in 128 cycles, half of what a single CTA's 128 x 256 tile would.  Two accumulators fill tensor memory, so that eight
// warps (each 32 channels by 128 tokens, neighbouring lanes neighbours in a row of y) write a tile out while the next
// one is computed; that takes some 8 instructions a value, and with four warps bounded the kernel (525 us for
// 8192 x 4096 x 14336 with the quantiser).  Now 358 to 386 us by box (power), the product alone 283 (3.4 POP/s, tensor pipe 80 % busy).
constexpr int kPairTile = 256, kPairStages = 6, kPairStage = 2 * 128 * 128, kPairOut = 8, kPairThreads = 32 * (kPairOut + 2);
constexpr int kGroup = 8;  // token tiles whose channel tiles are walked together: their operands stay in L2

__device__ __forceinline__ void pair_tile(const LinearArgs &p, int tile, int *channel, int *token)
{
    const int ct = (p.n + kPairTile - 1) / kPairTile, tt = (p.tokens + kPairTile - 1) / kPairTile;
    const int group = tile / (ct * kGroup), rest = tile - group * ct * kGroup, rows = min(kGroup, tt - group * kGroup);
    *token = (group * kGroup + rest % rows) * kPairTile;
    *channel = rest / rows * kPairTile;
}

template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1)
linear_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x,
                   const __grid_constant__ LinearArgs p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ struct {
        uint64_t full[kPairStages], empty[kPairStages], acc_full[2], acc_empty[2];
        uint32_t tmem;
        int abort_flag;
    } bars;
    __shared__ float4 s_scale[kPairOut][8];
    namespace cg = cooperative_groups;
    uint8_t *smem = reinterpret_cast<uint8_t *>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cg::this_cluster().block_rank();
    const int tiles = ((p.n + kPairTile - 1) / kPairTile) * ((p.tokens + kPairTile - 1) / kPairTile);
    const int first = (int)blockIdx.x >> 1, stride = (int)gridDim.x >> 1;
    volatile int *abort_flag = &bars.abort_flag;
    auto bar = [](uint64_t &b) { return smem_u32(&b); };
    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(bar(bars.full[s]), 1);   // the first CTA's counts the loads of both
            mbar_init(bar(bars.empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(bar(bars.acc_full[a]), 1);
            mbar_init(bar(bars.acc_empty[a]), 2 * kPairOut);  // the first CTA's: the writing warps of both
        }
        bars.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == kPairOut + 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();
    fence_after();
    const uint32_t tmem = bars.tmem;
    bool ok = true;

    if (warp == kPairOut) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        int s = 0;
        uint32_t phase = 0;
        for (int u = first; u < tiles && ok; u += stride) {
            int n0, t0;
            pair_tile(p, u, &n0, &t0);
            for (int c = 0; c < p.chunks && ok; ++c) {
                ok = mbar_wait(bar(bars.empty[s]), phase ^ 1, abort_flag, &g_status, 1);
                if (ok && elect_one()) {
                    const uint32_t full = peer_addr(bar(bars.full[s]), 0);
                    if (rank == 0) mbar_expect_tx(bar(bars.full[s]), 2 * kPairStage);
                    tma_load_2d_pair(base + s * kPairStage, &map_w, c * 128, n0 + 128 * rank, full);
                    tma_load_2d_pair(base + s * kPairStage + 128 * 128, &map_x, c * 128, t0 + 128 * rank, full);
                }
                __syncwarp();
                if (++s == kPairStages) {
                    s = 0;
                    phase ^= 1;
                }
            }
        }
    } else if (warp == kPairOut + 1 && rank == 0) {
        constexpr uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
        int s = 0, a = 0;
        uint32_t phase = 0, aphase = 0;
        for (int u = first; u < tiles && ok; u += stride) {
            ok = mbar_wait(bar(bars.acc_empty[a]), aphase ^ 1, abort_flag, &g_status, 4);
            fence_after();
            for (int c = 0; c < p.chunks && ok; ++c) {
                ok = mbar_wait(bar(bars.full[s]), phase, abort_flag, &g_status, 8);
                fence_after();
                if (ok && elect_one()) {
                    const uint64_t ad = make_desc(base + s * kPairStage, 128), bd = make_desc(base + s * kPairStage + 128 * 128, 128);
#pragma unroll
                    for (int ks = 0; ks < 4; ++ks) mma_i8_pair(tmem + 256 * a, ad + 2 * ks, bd + 2 * ks, idesc, (uint32_t)(c | ks));
                    mma_commit_pair(bar(bars.empty[s]));
                    if (c == p.chunks - 1) mma_commit_pair(bar(bars.acc_full[a]));
                }
                __syncwarp();
                if (++s == kPairStages) {
                    s = 0;
                    phase ^= 1;
                }
            }
            if ((a ^= 1) == 0) aphase ^= 1;
        }
    } else if (warp < kPairOut) {
        asm volatile("griddepcontrol.wait;" ::: "memory");  // the tokens' scales are the quantiser's
        const float floor = p.relu ? 0.f : -INFINITY;
        int a = 0;
        uint32_t aphase = 0;
        for (int u = first; u < tiles && ok; u += stride) {
            int n0, t0;
            pair_tile(p, u, &n0, &t0);
            const int q = warp & 3, j0 = warp < 4 ? 0 : kPairTile / 2;  // a quarter of tensor memory, a half of the tokens
            const int n = n0 + 128 * rank + 32 * q + lane;
            const bool mine = n < p.n;
            const float ws = mine ? p.w_scale[n] : 0.f, bias = mine && p.bias ? p.bias[n] : 0.f;
            const int have = min(kPairTile, p.tokens - t0), j1 = min(have, j0 + kPairTile / 2);
            ok = mbar_wait(bar(bars.acc_full[a]), aphase, abort_flag, &g_status, 16);
            fence_after();
            T *y = static_cast<T *>(p.y) + (long long)(t0 + j0) * p.ld_y + n;
            for (int j = j0; j < j1; j += 32) {
                int acc[32];
                tmem_ld32(tmem + 256 * a + ((uint32_t)(q * 32) << 16) + j, acc);
                __syncwarp();
                reinterpret_cast<float *>(s_scale[warp])[lane] = j + lane < have ? __ldg(p.x_scale + t0 + j + lane) : 0.f;
                __syncwarp();
                tmem_wait_ld();
                const int rows = mine ? j1 - j : 0;
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 xs = s_scale[warp][i / 4];
                    const float sc[4] = {xs.x, xs.y, xs.z, xs.w};
#pragma unroll
                    for (int l = 0; l < 4; ++l) {
                        if (i + l < rows) *y = from_float<T>(at_least(fmaf((float)acc[i + l], sc[l] * ws, bias), floor));
                        y += p.ld_y;
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_pair(peer_addr(bar(bars.acc_empty[a]), 0));
            if ((a ^= 1) == 0) aphase ^= 1;
        }
    }
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
    __syncwarp();
    fence_before();
    __syncthreads();
    cg::this_cluster().sync();  // no barrier of a CTA is signalled once it has gone
    if (warp == kPairOut + 1)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

accerl_status launch_pair(const CUtensorMap &mw, const CUtensorMap &mx, const LinearArgs &p, int sm_count, bool after_quant, cudaStream_t st)
{
    const size_t smem = 1024 + (size_t)kPairStages * kPairStage;
    const long long tiles = ((p.n + kPairTile - 1LL) / kPairTile) * ((p.tokens + kPairTile - 1LL) / kPairTile);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(2u * (unsigned)std::min<long long>(tiles, sm_count / 2));
    cfg.blockDim = dim3(kPairThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = after_quant ? 2 : 1;
    const auto kernel = p.y_dtype == ACCERL_F32    ? linear_pair_kernel<float>
                        : p.y_dtype == ACCERL_BF16 ? linear_pair_kernel<__nv_bfloat16>
                                                   : linear_pair_kernel<__half>;
    ACCERL_CUDA_TRY(allow_smem((const void *)kernel, smem));
    ACCERL_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, mw, mx, p));
    return ACCERL_OK;
}

bool good_quant(const char *who, const void *x, long long ld_x, int dtype, long long rows, int cols)
{
    if (rows < 1 || cols < 1 || cols > (1 << 30) || rows > (1LL << 31) - 1 || rows > (1LL << 40) / cols) {
        set_error("%s: rows and columns must be positive (rows below 2^31, columns at most 2^30, together at most 2^40)", who);
        return false;
    }
    if (!good_dtype(dtype) || !x || ((uintptr_t)x & (dtype_size(dtype) - 1)) || ld_x < cols) {
        set_error("%s: unknown dtype, or x is null, misaligned or its rows are closer than their length", who);
        return false;
    }
    return true;
}

}  // namespace

cudaError_t linear_status(int *out)  // (clears it)
{
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *out) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(int));
    return e;
}

}  // namespace accerl

using namespace accerl;

extern "C" accerl_status accerl_quant_rows(const void *x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t cols, int8_t *q,
                                           int64_t ld_q, float *scale, void *cuda_stream)
{
    if (!good_quant("quant_rows", x, ld_x, dtype, rows, cols)) return ACCERL_ERR_INVALID_ARG;
    if (!q || !scale || ((uintptr_t)q & 15) || ((uintptr_t)scale & 3) || ld_q < cols || ld_q % 16) {
        set_error("quant_rows: q needs 16-byte alignment and ld_q >= cols (a multiple of 16), scale 4-byte alignment");
        return ACCERL_ERR_INVALID_ARG;
    }
    const QuantArgs p{x, q, scale, ld_x, ld_q, rows, cols};
    int device = 0, sm_count = 0;
    ACCERL_CUDA_TRY(cudaGetDevice(&device));
    ACCERL_CUDA_TRY(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, device));
    ACCERL_CUDA_TRY(launch_quant(p, dtype, sm_count, (cudaStream_t)cuda_stream));
    return ACCERL_OK;
}

// one token that linear_token_kernel's shared memory holds
static bool one_token(int32_t tokens, int32_t k) { return tokens == 1 && k <= 64 * 1024; }

static int64_t quantised_bytes(int64_t tokens, int64_t k) { return (tokens * ((k + 15) / 16 * 16) + 255) / 256 * 256; }

extern "C" int64_t accerl_linear_i8_workspace(int32_t tokens, int32_t k, int32_t x_dtype)
{
    if (x_dtype == ACCERL_I8 || tokens < 1 || k < 1 || one_token(tokens, k)) return 0;
    return quantised_bytes(tokens, k) + (4LL * tokens + 255) / 256 * 256;
}

extern "C" accerl_status accerl_linear_i8(const accerl_linear_i8_args *a, void *cuda_stream)
{
    if (!a || !a->x || !a->w || !a->w_scale || !a->y) {
        set_error("linear_i8: null argument");
        return ACCERL_ERR_INVALID_ARG;
    }
    if ((a->n + 255LL) / 256 * ((a->tokens + 255LL) / 256) > (1 << 30)) {
        set_error("linear_i8: tokens * n is too large");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->tokens < 1 || a->n < 1 || a->k < 1 || a->k > 131072 || a->tokens >= kMostRows || a->n >= kMostRows) {
        set_error("linear_i8: tokens, n and k must be positive, k at most 131072 (an int32 sum of products of 127), the others below 2^31 - 2^16");
        return ACCERL_ERR_INVALID_ARG;
    }
    const bool given = a->x_dtype == ACCERL_I8;
    if (given ? (!a->x_scale || ((uintptr_t)a->x & 15) || a->ld_x < a->k || a->ld_x % 16 || ((uintptr_t)a->x_scale & 3))
              : a->x_scale != nullptr) {
        set_error("linear_i8: int8 x needs x_scale, 16-byte alignment and ld_x >= k (a multiple of 16); other x takes no x_scale");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (!given && !good_quant("linear_i8", a->x, a->ld_x, a->x_dtype, a->tokens, a->k)) return ACCERL_ERR_INVALID_ARG;
    if (((uintptr_t)a->w & 15) || a->ld_w < a->k || a->ld_w % 16 || (((uintptr_t)a->w_scale | (uintptr_t)a->bias) & 3)) {
        set_error("linear_i8: w needs 16-byte alignment and ld_w >= k (a multiple of 16), scales and bias 4-byte alignment");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (!good_dtype(a->y_dtype) || ((uintptr_t)a->y & (dtype_size(a->y_dtype) - 1)) || a->ld_y < a->n) {
        set_error("linear_i8: y has an unknown dtype, is misaligned or its rows are closer than n");
        return ACCERL_ERR_INVALID_ARG;
    }
    const int64_t need = accerl_linear_i8_workspace(a->tokens, a->k, a->x_dtype);
    if (need && (!a->workspace || ((uintptr_t)a->workspace & 255) || a->workspace_bytes < need)) {
        set_error("linear_i8: the workspace needs %lld bytes, aligned to 256", (long long)need);
        return ACCERL_ERR_INVALID_ARG;
    }
    int device = 0, sm_count = 0;
    ACCERL_CUDA_TRY(cudaGetDevice(&device));
    ACCERL_CUDA_TRY(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    LinearArgs p{a->x_scale, a->w_scale, a->bias, a->y, a->ld_y, a->tokens, a->n, a->k, a->y_dtype, a->relu != 0, (a->k + 127) / 128, 0};
    if (one_token(a->tokens, a->k)) return launch_token(a, p, sm_count, st);
    const void *xq = a->x;
    const float *xs = a->x_scale;
    int64_t ld_xq = a->ld_x;
    CUtensorMap mw, mx;
    if (!given) {
        ld_xq = (a->k + 15) / 16 * 16;
        xq = a->workspace;
        xs = reinterpret_cast<const float *>(static_cast<char *>(a->workspace) + quantised_bytes(a->tokens, a->k));
    }
    // From 65 tokens on pairs, but for few tiles of a long K, which needs to be split (us, few-token kernel / pairs, bf16 out: 1024 x
    // 1024 x 2048 20.3 / 10.9, 2047 x 2592 x 256 17.6 / 14.5, 512 x 4096 x 2048 19.7 / 17.3, 100 x 4096 x 14336 23.7 / 17.1, 65 x
    // 1024 x 1024 13.5 / 8.9, 8192 x 3136 x 512 32.4 / 16.3; 300 x 8192 x 512 16.2 / 26.1).
    const long long pair_tiles = ((a->n + kPairTile - 1LL) / kPairTile) * ((a->tokens + kPairTile - 1LL) / kPairTile);
    const bool pair = a->tokens > 64 && !(pair_tiles <= 8 && a->k > 32 * 128);
    const int nt = a->tokens <= 16 ? 16 : a->tokens <= 32 ? 32 : a->tokens <= 64 ? 64 : 128;
    accerl_status s = tc_make_map(&mw, a->w, a->n, a->k, a->ld_w, 128, 128);
    if (s == ACCERL_OK) s = tc_make_map(&mx, xq, a->tokens, a->k, ld_xq, nt, 128);
    if (s != ACCERL_OK) return s;
    if (!given) {
        const QuantArgs q{a->x, static_cast<int8_t *>(a->workspace), const_cast<float *>(xs), a->ld_x, ld_xq, a->tokens, a->k};
        ACCERL_CUDA_TRY(launch_quant(q, a->x_dtype, sm_count, st));
    }
    p.x_scale = xs;
    if (pair) return launch_pair(mw, mx, p, sm_count, !given, st);
    return nt == 16   ? launch_few<16>(mw, mx, p, sm_count, !given, st)
           : nt == 32 ? launch_few<32>(mw, mx, p, sm_count, !given, st)
           : nt == 64 ? launch_few<64>(mw, mx, p, sm_count, !given, st)
                      : launch_few<128>(mw, mx, p, sm_count, !given, st);
}

extern "C" accerl_status accerl_device_check(void)
{
    ACCERL_CUDA_TRY(cudaDeviceSynchronize());
    int linear = 0, grad = 0, loss = 0;
    ACCERL_CUDA_TRY(linear_status(&linear));
    ACCERL_CUDA_TRY(weight_grad_status(&grad));
    ACCERL_CUDA_TRY(policy_loss_status(&loss));
    if (linear || grad || loss) {
        set_error("a bounded device-side wait gave up (linear_i8 0x%x, ckpt_weight_grad 0x%x, policy_loss 0x%x)", linear, grad,
                  loss);
        return ACCERL_ERR_TIMEOUT;
    }
    return ACCERL_OK;
}
