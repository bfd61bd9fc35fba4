// Activation checkpoints in 8 bits: kept beside the activation's forward pass, read back, and used in its backward pass.
//
// 32 values along a row share a power of two 2^E, the smallest with max |x| / 2^E < 127.5.  With bits the largest
// magnitude's, that is E = exponent - 6, one more where the mantissa is at least 255/128 (its rounding would give
// 128): E + 127 = ((bits + 0x10000) >> 23) - 6.  Dividing by a power of two is exact, so a value is rounded once, to
// the integer, and q 2^E has at most 7 significant bits: every later product sees exactly what was kept.
//
// All three kernels move rows in pieces of 16 bytes of the activation's type (8 or 4 values; a block's 4 or 8 pieces
// lie in neighbouring lanes) and are bound by HBM; what bounds the code is the instructions a value: at 5 bytes a value
// (bf16 in and out, 8 bits kept) the memory leaves about 27 of them.  So the rounding is an addition of 1.5 2^23 that
// leaves the integer in the low byte, bytes become floats by a byte permutation, and GELU's Phi is an exponential,
// which the derivative shares, times a polynomial of a reciprocal.  8192 x 14336 bf16: kept with GELU in 108 us (5.5 TB/s),
// read back in 50 us (7.1 TB/s, part of it still in L2).
#include "learn.cuh"

namespace accerl {

namespace {

constexpr int kThreads = 256, kAhead = 4, kUnit = 32 * kAhead;  // pieces of a unit of work, a warp's

struct CkptArgs {
    const void *in;  // x (save) or dy (backward)
    void *out;       // y, x^ or dx; null: none
    int8_t *q;
    uint8_t *e;
    long long ld_in, ld_out, ld_q, ld_e, rows, cols;
    long long pieces;  // of a row, the last block's padding among them
    long long units;
    unsigned segments;  // units of a row
};

enum { kSave, kLoad, kBackward };

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Phi(x) and exp(-x^2 / 2), T the type that results are rounded to.  Phi(-u) = exp(-u^2 / 2) R(u), and R, half the scaled
// complementary error function, is t P(t) with t = 1 / (1 + p u): p and P's coefficients have the least relative error on
// 0 <= u <= 14 (least squares, reweighted until the error is level).  Degree 7 and an exponent in two parts for fp32: with the
// hardware's exponential and reciprocal within 2e-6 of Phi down to x = -13, where Phi is 6e-39.  Degree 5 (4e-6) and an exponent
// rounded once (6e-6 at -13) for 16-bit types.  (8192 x 14336 fp32 kept in 178 us; 164 the cheap way, whose error is 20 times fp32's.)
template <typename T>
__device__ __forceinline__ float normal_cdf(float x, float *density)
{
    constexpr bool full = sizeof(T) == 4;
    const float u = full ? fminf(fabsf(x), 1e10f) : fabsf(x);  // (its square finite, for its rounding; a NaN comes back as a factor)
    const float t = rcp(fmaf(full ? 0.30458614f : 0.3081619f, u, 1.f));
    const float s = u * u, a = s * -0.72134752f;  // log2(e) / 2
    float d = ex2(a), p;
    if constexpr (full) {
        float rest = fmaf(s, -0.72134752f, -a);
        rest = fmaf(fmaf(u, u, -s), -0.72134752f, rest);
        rest = fmaf(s, -9.629815e-9f, rest);
        d = fmaf(d, rest * 0.69314718f, d);
        p = fmaf(t, 0.036763538f, -0.15393415f);
        p = fmaf(t, p, 0.18836482f);
        p = fmaf(t, p, -0.04007097f);
        p = fmaf(t, p, 0.12204569f);
        p = fmaf(t, p, 0.10301612f);
        p = fmaf(t, p, 0.12234280f);
        p = fmaf(t, p, 0.12147221f);
    } else {
        p = fmaf(t, -0.07539816f, 0.18911967f);
        p = fmaf(t, p, 0.007704712f);
        p = fmaf(t, p, 0.13640875f);
        p = fmaf(t, p, 0.1189781f);
        p = fmaf(t, p, 0.12318499f);
    }
    const float below = p * t * d;
    *density = d;
    return x < 0.f ? below : 1.f - below;
}

template <typename T, int ACT>
__device__ __forceinline__ float activation(float x)
{
    if constexpr (ACT == ACCERL_ACT_RELU) return x < 0.f ? 0.f : x;  // (NaN stays NaN)
    if constexpr (ACT == ACCERL_ACT_GELU) {
        float d;
        return x * normal_cdf<T>(x, &d);
    }
    if constexpr (ACT == ACCERL_ACT_SILU) return x * rcp(1.f + ex2(x * -1.44269504f));
    return x;
}
template <typename T, int ACT>
__device__ __forceinline__ float slope(float x)
{
    if constexpr (ACT == ACCERL_ACT_RELU) return x > 0.f ? 1.f : x <= 0.f ? 0.f : x;
    if constexpr (ACT == ACCERL_ACT_GELU) {
        float d;
        const float cdf = normal_cdf<T>(x, &d);
        return fmaf(x * 0.39894228f, d, cdf);
    }
    if constexpr (ACT == ACCERL_ACT_SILU) {
        const float s = rcp(1.f + ex2(x * -1.44269504f));
        return s * fmaf(x, 1.f - s, 1.f);
    }
    return 1.f;
}

// byte k of a word of four int8, as a float
__device__ __forceinline__ float byte_value(uint32_t flipped, int k)
{
    return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7440u | (unsigned)k)) - 8388736.f;  // 2^23 + 128
}

// A warp takes 128 neighbouring pieces of a row at a time, so that everything but a lane's offset is the warp's.
// ALIGNED: the rows of both arrays start at multiples of 16 bytes.
template <typename T, int MODE, int ACT, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, 5) ckpt_kernel(const __grid_constant__ CkptArgs p)
{
    constexpr int V = Row<T>::kVec, kWords = V / 4, kLanes = 32 / V;  // lanes of a block
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (unit >= p.units) return;
    const long long row = p.rows == 1 ? 0 : (long long)((unsigned)unit / p.segments);  // (several rows: fewer than 2^32 units)
    const long long begin = (unit - row * p.segments) * (kUnit * V);              // first element of the unit in its row
    const T *in = static_cast<const T *>(p.in) + row * p.ld_in + begin;
    T *out = static_cast<T *>(p.out) + row * p.ld_out + begin;
    int8_t *q = p.q + row * p.ld_q + begin;
    uint8_t *e = p.e + row * p.ld_e + begin / 32;
    // elements of the unit that exist, and with the last block's padding
    const int n = (int)min((long long)kUnit * V, p.cols - begin), n32 = (int)min((long long)kUnit * V, p.pieces * V - begin);
    const bool full = n == kUnit * V;

    uint4 raw[MODE != kLoad ? kAhead : 1];
    uint32_t code[MODE != kSave ? kAhead : 1][kWords];
    int kept = 0;
    if constexpr (MODE != kSave) kept = lane < n32 / 32 ? e[lane] : 0;  // a unit has at most 32 blocks
    // (slopes far out are 0 or 1: values there stay finite, so that 0 times them is 0)
    if constexpr (MODE == kBackward && (ACT == ACCERL_ACT_GELU || ACT == ACCERL_ACT_SILU)) kept = kept == 255 ? 255 : min(kept, 200);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int at = (i * 32 + lane) * V;
        if constexpr (MODE != kLoad) {
            if (full) raw[i] = ALIGNED ? __ldcs(reinterpret_cast<const uint4 *>(in + at)) : load16(in + at);
            else raw[i] = load_piece<T, ALIGNED>(in, at, n, 0.f);
        }
        if constexpr (MODE != kSave) {
#pragma unroll
            for (int j = 0; j < kWords; ++j) code[i][j] = 0;
            if (at < n32) {
                if constexpr (kWords == 2) {
                    const uint2 c = __ldcs(reinterpret_cast<const uint2 *>(q + at));
                    code[i][0] = c.x;
                    code[i][1] = c.y;
                } else {
                    code[i][0] = __ldcs(reinterpret_cast<const unsigned *>(q + at));
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int at = (i * 32 + lane) * V;
        float v[V];
        if constexpr (MODE == kSave) {
            unpack<T>(raw[i], v);
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < V; ++k) top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
#pragma unroll
            for (int o = 1; o < kLanes; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            const bool broken = top >= 0x7f800000u;  // an infinity or a NaN
            const int ev = broken ? 255 : max((int)((top + 0x10000u) >> 23) - 6, 1);
            const float inv = __uint_as_float((uint32_t)(254 - min(ev, 253)) << 23);  // (ev <= 249 for finite values)
            uint32_t w[kWords];
#pragma unroll
            for (int j = 0; j < kWords; ++j) {
                uint32_t b[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) b[k] = __float_as_uint(fmaf(v[4 * j + k], inv, 12582912.f));
                w[j] = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
                if (broken) w[j] = 0;
            }
            if (at < n32) {
                if constexpr (kWords == 2) *reinterpret_cast<uint2 *>(q + at) = make_uint2(w[0], w[1]);
                else *reinterpret_cast<uint32_t *>(q + at) = w[0];
                if (lane % kLanes == 0) e[i * V + lane / kLanes] = (uint8_t)ev;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = activation<T, ACT>(v[k]);
        } else {
            float dy[V];
            if constexpr (MODE == kBackward) unpack<T>(raw[i], dy);
            // (255: infinity times the block's zeros, NaN)
            const float s = __uint_as_float((uint32_t)__shfl_sync(0xffffffffu, kept, i * V + lane / kLanes) << 23);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float x = byte_value(code[i][k / 4] ^ 0x80808080u, k & 3) * s;
                v[k] = MODE == kBackward ? dy[k] * slope<T, ACT>(x) : x;
            }
        }
        if (MODE != kSave || p.out) {
            if (full) {
                if (ALIGNED) *reinterpret_cast<uint4 *>(out + at) = pack<T>(v);
                else store16(out + at, pack<T>(v));
            } else {
                store_piece<T, ALIGNED>(out, at, n, v);
            }
        }
    }
}

template <typename T, int MODE, bool ALIGNED>
auto kernel_of(int act)
{
    if constexpr (MODE != kLoad) {
        if (act == ACCERL_ACT_RELU) return ckpt_kernel<T, MODE, ACCERL_ACT_RELU, ALIGNED>;
        if (act == ACCERL_ACT_GELU) return ckpt_kernel<T, MODE, ACCERL_ACT_GELU, ALIGNED>;
        if (act == ACCERL_ACT_SILU) return ckpt_kernel<T, MODE, ACCERL_ACT_SILU, ALIGNED>;
    }
    return ckpt_kernel<T, MODE, ACCERL_ACT_NONE, ALIGNED>;
}

template <int MODE>
accerl_status launch(CkptArgs &p, int dtype, int act, void *cuda_stream)
{
    const bool dense = p.cols % 32 == 0 && (MODE == kLoad || p.ld_in == p.cols) && (!p.out || p.ld_out == p.cols) && p.ld_q == p.cols &&
                       p.ld_e == p.cols / 32;
    if (dense) {  // rows without gaps are one row
        p.cols *= p.rows;
        p.rows = 1;
    }
    p.pieces = (p.cols + 31) / 32 * 32 * dtype_size(dtype) / 16;
    p.segments = (unsigned)((p.pieces + kUnit - 1) / kUnit);
    p.units = p.rows * ((p.pieces + kUnit - 1) / kUnit);
    if (p.units > (p.rows == 1 ? 1LL << 33 : (1LL << 32) - 1)) {
        set_error("checkpoint: too many values");
        return ACCERL_ERR_INVALID_ARG;
    }
    const unsigned blocks = (unsigned)((p.units + kThreads / 32 - 1) / (kThreads / 32));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool aligned = (MODE == kLoad || rows_aligned(p.in, p.ld_in, dtype)) && (!p.out || rows_aligned(p.out, p.ld_out, dtype));
    ACCERL_CUDA_TRY(with_dtype(dtype, [&](auto v) {
        using T = decltype(v);
        const auto kernel = aligned ? kernel_of<T, MODE, true>(act) : kernel_of<T, MODE, false>(act);
        kernel<<<blocks, kThreads, 0, st>>>(p);
        return cudaGetLastError();
    }));
    return ACCERL_OK;
}

bool good_sizes(const char *who, long long rows, int cols, int dtype, int act)
{
    if (rows < 1 || cols < 1 || cols > (1 << 30) || rows > (1LL << 40) / cols) {
        set_error("%s: rows and cols must be positive (cols at most 2^30, rows * cols at most 2^40)", who);
        return false;
    }
    if (!good_dtype(dtype) || act < ACCERL_ACT_NONE || act > ACCERL_ACT_SILU) {
        set_error("%s: unknown dtype %d or activation %d", who, dtype, act);
        return false;
    }
    return true;
}

bool good_rows(const char *who, const char *name, const void *p, long long ld, int cols, int dtype)
{
    if (!p || ld < cols || ((uintptr_t)p & (dtype_size(dtype) - 1))) {
        set_error("%s: %s is null, misaligned or its rows are closer than cols", who, name);
        return false;
    }
    return true;
}

bool good_ckpt(const char *who, const void *q, long long ld_q, const void *e, long long ld_e, int cols)
{
    const int cols32 = (cols + 31) / 32 * 32;
    if (!q || !e || ((uintptr_t)q & 15) || ld_q < cols32 || ld_q % 16 || ld_e < cols32 / 32) {
        set_error("%s: a checkpoint's q needs 16-byte alignment, ld_q >= %d (a multiple of 16) and ld_e >= %d", who, cols32,
                  cols32 / 32);
        return false;
    }
    return true;
}

}  // namespace

}  // namespace accerl

using namespace accerl;

extern "C" accerl_status accerl_ckpt_save(const void *x, int64_t ld_x, int32_t dtype, int64_t rows, int32_t cols,
                                          int32_t act, void *y, int64_t ld_y, int8_t *q, int64_t ld_q, uint8_t *e,
                                          int64_t ld_e, void *cuda_stream)
{
    const char *who = "ckpt_save";
    if (!good_sizes(who, rows, cols, dtype, act) || !good_rows(who, "x", x, ld_x, cols, dtype) ||
        (y && !good_rows(who, "y", y, ld_y, cols, dtype)) || !good_ckpt(who, q, ld_q, e, ld_e, cols))
        return ACCERL_ERR_INVALID_ARG;
    if (y == x && ld_y != ld_x && rows > 1) {
        set_error("ckpt_save: y in place of x needs the same ld");
        return ACCERL_ERR_INVALID_ARG;
    }
    CkptArgs p{x, y, q, e, ld_x, ld_y, ld_q, ld_e, rows, cols, 0, 0, 0};
    return launch<kSave>(p, dtype, act, cuda_stream);
}

extern "C" accerl_status accerl_ckpt_load(const int8_t *q, int64_t ld_q, const uint8_t *e, int64_t ld_e, int64_t rows,
                                          int32_t cols, void *x, int64_t ld_x, int32_t dtype, void *cuda_stream)
{
    const char *who = "ckpt_load";
    if (!good_sizes(who, rows, cols, dtype, ACCERL_ACT_NONE) || !good_rows(who, "x", x, ld_x, cols, dtype) ||
        !good_ckpt(who, q, ld_q, e, ld_e, cols))
        return ACCERL_ERR_INVALID_ARG;
    CkptArgs p{nullptr, x, const_cast<int8_t *>(q), const_cast<uint8_t *>(e), 0, ld_x, ld_q, ld_e, rows, cols, 0, 0, 0};
    return launch<kLoad>(p, dtype, ACCERL_ACT_NONE, cuda_stream);
}

extern "C" accerl_status accerl_ckpt_act_backward(const void *dy, int64_t ld_dy, int32_t dtype, const int8_t *q,
                                                  int64_t ld_q, const uint8_t *e, int64_t ld_e, int64_t rows,
                                                  int32_t cols, int32_t act, void *dx, int64_t ld_dx, void *cuda_stream)
{
    const char *who = "ckpt_act_backward";
    if (!good_sizes(who, rows, cols, dtype, act) || !good_rows(who, "dy", dy, ld_dy, cols, dtype) ||
        !good_rows(who, "dx", dx, ld_dx, cols, dtype) || !good_ckpt(who, q, ld_q, e, ld_e, cols))
        return ACCERL_ERR_INVALID_ARG;
    if (dx == dy && ld_dx != ld_dy && rows > 1) {
        set_error("ckpt_act_backward: dx in place of dy needs the same ld");
        return ACCERL_ERR_INVALID_ARG;
    }
    CkptArgs p{dy, dx, const_cast<int8_t *>(q), const_cast<uint8_t *>(e), ld_dy, ld_dx, ld_q, ld_e, rows, cols, 0, 0, 0};
    return launch<kBackward>(p, dtype, act, cuda_stream);
}
