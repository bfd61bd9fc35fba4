// Clipped policy loss with a KL and an entropy term over rows of logits, forward and backward in one pass.
//
// In base 2, with t_v = (z_v - c) log2(e) (c the row's maximum), e_v = 2^t_v, S = sum e_v and the same
// t', S' of the reference row:
//   log2 p_v = t_v - log2 S,   KL log2(e) = sum e_v (t_v - t'_v) / S - log2(S / S'),   H log2(e) = log2 S - sum e_v t_v / S,
// so one pass over a row gives all it needs, and only centred quantities are subtracted.  The gradient is
//   w p_v (k0 + k1 (t_v - t'_v) + k2 t_v) + w c [v = a]
// with k0, k1, k2, c numbers of the row: it needs every logit once more.  A row therefore stays on chip between
// the two: in the registers of a group of lanes (narrow rows), of a warp, of a CTA, or of a cluster of CTAs that
// share their partial sums through distributed shared memory (a long row is split over several SMs, so that a
// single one of 128 001 logits takes no longer than a short one).  Logits are read from memory once and the gradient
// is written once; the kernel is bound by HBM.
#include <cooperative_groups.h>
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "exp64.cuh"
#include "learn.cuh"
#include "tc_ptx.cuh"

namespace accerl {

namespace {

__device__ int g_status;  // of this file's bounded waits

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

struct LossArgs {
    const void *logits, *ref;
    const void *actions;
    const float *logp_old, *advantages, *logp_ref, *weights;
    long long ld, ld_ref, ld_grad;
    int rows, A, actions64;
    int part_pieces;  // long rows: room of a CTA's part, in pieces
    float clip_low, clip_high, kl_coef, entropy_coef;
    void *grad;
    float *logp, *kl, *entropy, *terms;
};

__device__ __forceinline__ float exp2_fast(float x)  // 2 ulp, and 0 below -126 (nothing beside a row's largest term, 1)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float max_nan(float a, float b)  // a NaN wins
{
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}

__device__ __forceinline__ long long action_of(const LossArgs &p, long long row)
{
    return p.actions64 ? static_cast<const long long *>(p.actions)[row] : (long long)static_cast<const int *>(p.actions)[row];
}

__device__ __forceinline__ float weight_of(const LossArgs &p, long long row)
{
    return p.weights ? p.weights[row] : (float)(1.0 / (double)p.rows);
}

__device__ __forceinline__ double exp_of(double x) { return exp(x); }
__device__ __forceinline__ float exp_of(float x) { return expf(x); }
__device__ __forceinline__ double expm1_of(double x) { return expm1(x); }
__device__ __forceinline__ float expm1_of(float x) { return expm1f(x); }

// What a row's sums make of it: its outputs, and the gradient's coefficients (natural logarithms: delta_v = log p_v -
// log q_v, lp_v = log p_v):  d loss / d z_v = w p_v (base + kl_coef delta_v + entropy_coef lp_v) + w slope [v = a].
// R: double for narrow rows; float for long ones, where this is a chain of instructions that a whole CTA waits for
// (the difference of two log-probabilities is taken in double all the same).
template <typename R>
struct RowResult {
    R base, slope;
    R pg, r, kl, H;  // what the sums over rows take (r negative where the clamp decided)
};
template <typename R>
__device__ __forceinline__ RowResult<R> finish_row(const LossArgs &p, long long row, double logp, R kl_full, R H, bool empty, bool writer)
{
    R kl = kl_full, slope = 0, pg = 0, r = 0;
    bool inside = true;
    if (empty) {
        kl = H = 0;
    } else {
        const R adv = (R)p.advantages[row];
        const R x = (R)(logp - (double)p.logp_old[row]);
        r = exp_of(x);
        const R lo = (R)1 - (R)p.clip_low, hi = (R)1 + (R)p.clip_high;
        const R rc = r < lo ? lo : r > hi ? hi : r;  // (a NaN stays one)
        R plain = r * adv;
        if (__builtin_expect(r == (R)INFINITY, 0)) {  // (its product may be a number all the same)
            const R h = exp_of(x * (R)0.5);
            plain = adv == (R)0 ? (R)0 : h * adv * h;
        }
        const R clipped = rc * adv;
        inside = !(plain > clipped);
        pg = -(inside ? plain : clipped);
        slope = inside ? -plain : (R)0;
        if (p.logp_ref) {
            const R d = (R)((double)p.logp_ref[row] - logp), e = expm1_of(d);
            kl = e == (R)INFINITY ? e : e - d;  // (d may be infinite too)
            if (p.kl_coef != 0.f) slope -= (R)p.kl_coef * e;  // (e may be infinite)
        }
    }
    RowResult<R> o;
    o.pg = pg;
    o.r = inside ? r : -r;
    o.kl = kl;
    o.H = H;
    if (writer) {
        *reinterpret_cast<float2 *>(p.terms + 2 * row) = make_float2((float)o.pg, (float)o.r);
        p.logp[row] = (float)logp;
        p.kl[row] = (float)o.kl;
        p.entropy[row] = (float)o.H;
    }
    o.slope = slope;
    o.base = -slope + (R)p.entropy_coef * H - (p.ref && p.kl_coef != 0.f ? (R)p.kl_coef * kl : (R)0);
    return o;
}

__device__ __forceinline__ void skip_row(const LossArgs &p, long long row)
{
    p.logp[row] = p.kl[row] = p.entropy[row] = 0.f;
    *reinterpret_cast<float2 *>(p.terms + 2 * row) = make_float2(0.f, 0.f);
}

// -------------------------------------------------------------------------------------- sums over rows
constexpr int kStatsThreads = 1024, kStatsCluster = 8, kSums = 7;

// A row's share of the sums: weight, pg, kl, H, and r, negative where the clamp decided.
struct RowSums {
    double sum[kSums] = {};
    float most = -INFINITY;
    __device__ __forceinline__ void add(const LossArgs &p, float weight, double pg, double kl, double H, double r)
    {
        const double w = (double)weight;
        sum[0] += w * (pg + (p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0) - (double)p.entropy_coef * H);
        sum[1] += w * pg;
        sum[2] += w * kl;
        sum[3] += w * H;
        sum[4] += signbit(r) ? w : 0.0;
        sum[5] += w;
        sum[6] += w * fabs(r);
        most = max_nan(most, (float)kl);
    }
};

// Adds up the rows' shares of the threads of a cluster (of one CTA or eight) in a fixed order.  The cluster's first barrier
// phase has been arrived at.
__device__ __forceinline__ void write_stats(RowSums s, float *__restrict__ stats)
{
    namespace cg = cooperative_groups;
    __shared__ double s_sum[kStatsThreads / 32][kSums];
    __shared__ float s_max[kStatsThreads / 32];
    __shared__ double c_sum[kStatsCluster][kSums];  // used in the first CTA
    __shared__ float c_max[kStatsCluster];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) s.sum[j] += __shfl_xor_sync(0xffffffffu, s.sum[j], o);
        s.most = max_nan(s.most, __shfl_xor_sync(0xffffffffu, s.most, o));
    }
    if (lane == 0) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) s_sum[warp][j] = s.sum[j];
        s_max[warp] = s.most;
    }
    __syncthreads();
    asm volatile("barrier.cluster.wait;" ::: "memory");  // the first CTA has started
    if (warp == 0) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) s.sum[j] = lane < warps ? s_sum[lane][j] : 0.0;
        s.most = lane < warps ? s_max[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int j = 0; j < kSums; ++j) s.sum[j] += __shfl_xor_sync(0xffffffffu, s.sum[j], o);
            s.most = max_nan(s.most, __shfl_xor_sync(0xffffffffu, s.most, o));
        }
        if (lane == 0) {
            const unsigned rank = cg::this_cluster().block_rank();
#pragma unroll
            for (int j = 0; j < kSums; ++j) *cg::this_cluster().map_shared_rank(&c_sum[rank][j], 0) = s.sum[j];
            *cg::this_cluster().map_shared_rank(&c_max[rank], 0) = s.most;
        }
    }
    cg::this_cluster().sync();
    if (blockIdx.x == 0 && threadIdx.x < kSums) {
        double v = 0.0;
        for (unsigned i = 0; i < gridDim.x; ++i) v += c_sum[i][threadIdx.x];
        const int j = (int)threadIdx.x;
        stats[j < 6 ? j : 7] = (float)v;
        if (j == 0) {
            float most = -INFINITY;
            for (unsigned i = 0; i < gridDim.x; ++i) most = max_nan(most, c_max[i]);
            stats[6] = most == -INFINITY ? 0.f : most;
        }
    }
}

__global__ void __launch_bounds__(kStatsThreads)
loss_stats_kernel(const __grid_constant__ LossArgs p, float *__restrict__ stats)
{
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    RowSums s;
    const long long stride = (long long)gridDim.x * blockDim.x;
    constexpr int kAhead = 4;  // rows whose loads are in flight: the kernel is a chain of memory latencies
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < p.rows; i += kAhead * stride) {
        float w[kAhead], kl[kAhead], H[kAhead];
        float2 t[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const long long row = min(i + j * stride, (long long)p.rows - 1);
            w[j] = i + j * stride < p.rows ? weight_of(p, row) : 0.f;
            t[j] = __ldcg(reinterpret_cast<const float2 *>(p.terms + 2 * row));
            kl[j] = __ldcg(p.kl + row);
            H[j] = __ldcg(p.entropy + row);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            if (w[j] != 0.f) s.add(p, w[j], t[j].x, kl[j], H[j], t[j].y);
    }
    write_stats(s, stats);
}

// ------------------------------------------------------------------------------------------ narrow rows
// Up to 64 actions: a group of G lanes per row, at most 8 elements a lane, in double (two exponentials an element are
// free beside the latencies here, and whether a ratio is clipped is decided where the definition decides it).
// (100000 rows of 128 fp32: 94 us this way, 64 by the warp kernel below; 131072 of 18: 38 us.)
constexpr int kNarrow = 64, kNarrowPer = 8;

//
// STATS (few rows, one CTA): the sums over rows come out of the same launch.
template <typename T, bool REF, int G, bool STATS>
__global__ void __launch_bounds__(STATS ? 1024 : 128) loss_narrow_kernel(const __grid_constant__ LossArgs p, float *__restrict__ stats)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (STATS) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    __shared__ double table[64];
    fill_exp_table(table);
    __syncthreads();
    const int lane = threadIdx.x % G;
    const long long row = ((long long)blockIdx.x * blockDim.x + threadIdx.x) / G;
    const bool live = row < p.rows;
    const float w = live ? weight_of(p, row) : 0.f;
    const bool work = live && w != 0.f;
    const T *z_row = static_cast<const T *>(p.logits) + (live ? row : 0) * p.ld;
    const T *r_row = REF ? static_cast<const T *>(p.ref) + (live ? row : 0) * p.ld_ref : nullptr;
    float z[kNarrowPer], zr[REF ? kNarrowPer : 1];
    double mo = -INFINITY, mr = -INFINITY;
#pragma unroll
    for (int k = 0; k < kNarrowPer; ++k) {
        const int v = k * G + lane;
        const bool in = work && v < p.A;
        z[k] = in ? to_float(z_row[v]) : -INFINITY;
        mo = fmax(mo, (double)z[k]);
        if constexpr (REF) {
            zr[k] = in ? to_float(r_row[v]) : -INFINITY;
            mr = fmax(mr, (double)zr[k]);
        }
    }
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) {
        mo = fmax(mo, __shfl_xor_sync(0xffffffffu, mo, o));
        if (REF) mr = fmax(mr, __shfl_xor_sync(0xffffffffu, mr, o));
    }
    const bool none = mo == -INFINITY;
    if (none) mo = 0.0;
    if (mr == -INFINITY) mr = 0.0;
    double so = 0.0, ss = 0.0, sd = 0.0, st = 0.0, e[kNarrowPer];
#pragma unroll
    for (int k = 0; k < kNarrowPer; ++k) {
        const double t = (double)z[k] - mo;
        e[k] = exp_nonpositive(t, table);
        so += e[k];
        if (e[k] != 0.0) st += e[k] * t;
        if constexpr (REF) {
            const double tr = (double)zr[k] - mr;
            ss += exp_nonpositive(tr, table);
            if (e[k] != 0.0) sd += e[k] * (t - tr);
        }
    }
#pragma unroll
    for (int o = G / 2; o > 0; o >>= 1) {
        so += __shfl_xor_sync(0xffffffffu, so, o);
        st += __shfl_xor_sync(0xffffffffu, st, o);
        if (REF) {
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
            sd += __shfl_xor_sync(0xffffffffu, sd, o);
        }
    }
    const bool empty = none && so == 0.0;  // (the maximum passes over a NaN, the sum does not)
    // the action's logit from the lane that holds it (`grad` may be `logits`: memory is not read again)
    const long long a = work ? action_of(p, row) : -1;
    const bool known = a >= 0 && a < p.A;
    float za = 0.f;
#pragma unroll
    for (int k = 0; k < kNarrowPer; ++k)
        if (known && k == (int)a / G) za = z[k];
    za = __shfl_sync(0xffffffffu, za, known ? (int)a % G : 0, G);
    RowSums sums;
    T *g_row = p.grad ? static_cast<T *>(p.grad) + (live ? row : 0) * p.ld_grad : nullptr;
    if (live && !work) {
        if (lane == 0) skip_row(p, row);
        if (g_row)
            for (int v = lane; v < p.A; v += G) g_row[v] = from_float<T>(0.f);
    }
    if (work) {
        const double lso = log(so), lsr = REF ? log(ss) : 0.0;
        const double logp = known ? ((double)za - mo) - lso : (double)NAN;
        const double kl = REF ? sd / so - (lso - lsr) : 0.0, H = lso - st / so;
        // (a row without a finite logit: log 0 everywhere, and no distribution to have a gradient)
        const RowResult<double> f = finish_row<double>(p, row, empty && known ? -INFINITY : logp, kl, H, empty && known, lane == 0);
        if (STATS && lane == 0) sums.add(p, w, f.pg, f.kl, f.H, f.r);
        if (g_row) {
#pragma unroll
            for (int k = 0; k < kNarrowPer; ++k) {
                const int v = k * G + lane;
                if (v >= p.A) break;
                const double pv = e[k] / so, lp = ((double)z[k] - mo) - lso;
                double b = f.base + (double)p.entropy_coef * lp;
                if constexpr (REF) {
                    if (p.kl_coef != 0.f) b += (double)p.kl_coef * (lp - (((double)zr[k] - mr) - lsr));
                }
                double g = e[k] == 0.0 ? 0.0 : pv * b;
                if (v == a) g += f.slope;
                g_row[v] = from_float<T>(empty && known ? 0.f : (float)((double)w * g));
            }
        }
    }
    if (STATS) write_stats(sums, stats);
}

// -------------------------------------------------------------------------------------------- long rows
template <typename T>
__device__ __forceinline__ uint32_t max_words(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 4) {
        return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(b)));
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2 m = __hmax2_nan(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    } else {
        const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
}
template <typename T>
__device__ __forceinline__ uint32_t min_words(uint32_t a, uint32_t b)
{
    if constexpr (sizeof(T) == 4) {
        return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b)));
    } else if constexpr (std::is_same<T, __half>::value) {
        const __half2 m = __hmin2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    } else {
        const __nv_bfloat162 m = __hmin2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
        return *reinterpret_cast<const uint32_t *>(&m);
    }
}
// one or two logits: is one of the policy's above the low value where the reference's is below it (OR_AT: or there)?
template <typename T, bool OR_AT = false>
__device__ __forceinline__ bool meets(uint32_t z, uint32_t r, uint32_t low)
{
    if constexpr (sizeof(T) == 4) {
        const float l = __uint_as_float(low), q = __uint_as_float(r);
        return __uint_as_float(z) > l && (OR_AT ? q <= l : q < l);
    } else {
        using T2 = std::conditional_t<std::is_same<T, __half>::value, __half2, __nv_bfloat162>;
        const T2 l = *reinterpret_cast<const T2 *>(&low), q = *reinterpret_cast<const T2 *>(&r);
        return (__hgt2_mask(*reinterpret_cast<const T2 *>(&z), l) & (OR_AT ? __hle2_mask(q, l) : __hlt2_mask(q, l))) != 0;
    }
}
// What -inf, and anything below, is taken for (finite, so that its probability of 0 times its logarithm is 0), as a word of
// one or two elements.  Where the reference lies below it and the policy above, its logarithm counts: such rows (parts) are
// `odd`, summed up and differentiated element by element in double.
template <typename T>
__device__ __forceinline__ constexpr float low_value() { return std::is_same<T, __half>::value ? -65504.f : -33554432.f; }
// A row or part whose maximum is that far from 0 is `apart`: read again and kept relative to its maximum.  Below: so far down that
// what is taken for the low value might have a probability.  Above, and below: the shift -c log2(e), rounded, is off by up to 2
// at 2^25 (which cancels), and by more than an exponential bears further out.  (fp16 values are off by 2^-8 at most.)
template <typename T>
__device__ __forceinline__ bool is_below(float c) { return c <= 0.5f * low_value<T>(); }
template <typename T>
__device__ __forceinline__ bool is_above(float c) { return !std::is_same<T, __half>::value && c >= -0.5f * low_value<T>() && c != INFINITY; }
template <typename T>
__device__ __forceinline__ bool apart(float c) { return is_below<T>(c) || is_above<T>(c); }
// A reference with this maximum makes a row odd: ordinary values may lie far below it, or it is infinite or a NaN.
template <typename T>
__device__ __forceinline__ bool too_high(float cr) { return std::is_same<T, __half>::value ? !(cr < INFINITY) : !(cr < -0.5f * low_value<T>()); }
template <typename T>
__device__ __forceinline__ uint32_t low_word()
{
    const float v[2] = {low_value<T>(), low_value<T>()};
    return pack_word(v, (const T *)nullptr);
}
template <typename T>
__device__ __forceinline__ float word_max(uint32_t w)
{
    float v[2];
    unpack_word(w, v, (const T *)nullptr);
    return sizeof(T) == 4 ? v[0] : max_nan(v[0], v[1]);
}
template <typename T>
__device__ __forceinline__ float word_min(uint32_t w)
{
    float v[2];
    unpack_word(w, v, (const T *)nullptr);
    return sizeof(T) == 4 ? v[0] : fminf(v[0], v[1]);
}
__device__ __forceinline__ uint32_t *words(uint4 &v) { return reinterpret_cast<uint32_t *>(&v); }
__device__ __forceinline__ const uint32_t *words(const uint4 &v) { return reinterpret_cast<const uint32_t *>(&v); }

// Gradient coefficients of a row for sums relative to maxima C and CR:  w p_v (base + kl_coef delta_v + entropy_coef lp_v)
// = e_v (k0 + kt t_v - kr t'_v), logarithms in base 2; and what the action's logit gets on top.
struct RowCoef {
    float c, cr, k0, kt, kr, at_a;
};
// log2 of a positive sum: the exponent and the mantissa's logarithm apart, off by 1e-7 whatever its size
__device__ __forceinline__ double log2_of(double x)
{
    const int hi = __double2hiint(x);
    if (hi < 0x00100000 || hi >= 0x7ff00000) return (double)log2f((float)x);  // (0, infinity, NaN)
    const double m = __hiloint2double((hi & 0x000fffff) | 0x3ff00000, __double2loint(x));
    return (double)((hi >> 20) - 1023) + (double)log2f((float)m);
}

// -c log2(e) rounded, and not as part of a multiply-add: the same everywhere
__device__ __forceinline__ float minus_log2(float c) { return -__fmul_rn(c, kLog2e); }

// What every t of a row with maximum c is too large by, since its shift is rounded (half a step of c log2(e): at logits around
// 1000 some 1e-4).  Sums, KL, entropy and the gradient hold differences of t and lose it, a log-probability does not.
// (The rounding error of a product is a float, so this is exact.)
template <typename T>
__device__ __forceinline__ float excess_of(float c) { return apart<T>(c) ? 0.f : fmaf(c, kLog2e, minus_log2(c)); }

// `excess`: of the policy's t, of which the sums are made
template <bool REF>
__device__ __forceinline__ RowCoef row_coef(const LossArgs &p, long long row, float w, bool known, float za, float C, float CR, double so,
                                            double st, double ss, double sd, float excess, bool writer)
{
    const bool empty = known && C == -INFINITY;
    const float fo = (float)so, fs = (float)ss, inv = 1.f / fo;
    const double lso = log2_of(so);
    // log2(S / S') from the difference of the sums where they are near each other
    const float d = (float)(so - ss) / fs, ratio = REF ? (fabsf(d) < 0.5f ? log1pf(d) * kLog2e : (float)(lso - log2_of(ss))) : 0.f;
    const float H = (float)kLn2 * (float)(lso - (double)((float)st * inv));
    float kl = REF ? (float)kLn2 * ((float)sd * inv - ratio) : 0.f;
    if (REF && __builtin_expect(fabsf(kl) > 1e37f, 0)) {  // (its parts may lie beyond fp32, it does only where it is infinite)
        const double x = kLn2 * (double)inv * sd - kLn2 * (double)ratio;
        kl = x < (double)INFINITY ? (float)fmin(x, 3.4028234663852886e38) : (float)x;
    }
    const double at_c = (double)za - (double)C + kLn2 * (double)excess;  // (apart from the sums, which take longer)
    const double logp = empty ? (double)-INFINITY : known ? at_c - kLn2 * lso : (double)NAN;
    const RowResult<float> f = finish_row<float>(p, row, logp, kl, H, empty, writer);
    const float scale = w * inv, kk = REF ? p.kl_coef * (float)kLn2 : 0.f, ke = p.entropy_coef * (float)kLn2;
    RowCoef r;
    r.c = C;
    r.cr = CR;
    r.k0 = empty ? 0.f : scale * (f.base - ke * (float)lso - (kk != 0.f ? kk * ratio : 0.f));
    r.kt = empty ? 0.f : scale * (ke + kk);
    r.kr = empty ? 0.f : scale * kk;
    r.at_a = empty ? 0.f : w * f.slope;
    return r;
}

// t of a piece's logits kept relative to `base` (0, or the maximum of a part that is apart), when the row's maximum is c; far
// below it probabilities are 0, and logarithms kept finite
template <typename T>
__device__ __forceinline__ float shift_of(float base, float c)
{
    return c == -INFINITY ? 0.f : base == 0.f ? minus_log2(c) : max_nan(fmaf(base - c, kLog2e, excess_of<T>(c)), -1e30f);
}

template <typename T, bool REF>
__device__ __forceinline__ void add_sums(const uint4 &raw, const uint4 &raw_r, float nc, float ncr, float &so, float &st, float &ss, float &sd)
{
    constexpr int V = Row<T>::kVec;
    float z[V], zr[V];
    unpack<T>(raw, z);
    if constexpr (REF) unpack<T>(raw_r, zr);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float t = fmaf(z[k], kLog2e, nc), e = exp2_fast(t);
        so += e;
        st = fmaf(e, t, st);
        if constexpr (REF) {
            const float tr = fmaf(zr[k], kLog2e, ncr);
            ss += exp2_fast(tr);
            sd = fmaf(e, t - tr, sd);
        }
    }
}

template <typename T, bool REF>
__device__ __forceinline__ void put_gradient(const LossArgs &p, T *g_row, int at, int a, const uint4 &raw, const uint4 &raw_r, const RowCoef &f,
                                             float sh, float shr)
{
    constexpr int V = Row<T>::kVec;
    float z[V], zr[V], g[V];
    unpack<T>(raw, z);
    if constexpr (REF) unpack<T>(raw_r, zr);
#pragma unroll
    for (int k = 0; k < V; ++k) {  // (t and t' once more: what is left of the coefficients' terms without their shifts would be off by the offset)
        const float t = fmaf(z[k], kLog2e, sh);
        float b = fmaf(f.kt, t, f.k0);
        if constexpr (REF) b = fmaf(-f.kr, fmaf(zr[k], kLog2e, shr), b);
        g[k] = exp2_fast(t) * b;
    }
    if ((unsigned)(a - at) < (unsigned)V) {
#pragma unroll
        for (int k = 0; k < V; ++k)
            if (at + k == a) g[k] += f.at_a;
    }
    store_piece<T>(g_row, at, p.A, g);
}

// t of one logit in double, relative to what the sums of a row or part with maximum c are relative to
template <typename T>
__device__ __forceinline__ double t_of(float x, float c)
{
    return x == -INFINITY ? (double)-INFINITY : apart<T>(c) ? ((double)x - (double)c) * (double)kLog2e : fma((double)x, (double)kLog2e, (double)minus_log2(c));
}

// the sums of elements begin, begin + step ... of an odd row or part: e, e t, e', e (t - t')
template <typename T>
__device__ __forceinline__ void odd_sums(const T *z_row, const T *r_row, int begin, int end, int step, float c, float cr, double (&sum)[4])
{
    sum[0] = sum[1] = sum[2] = sum[3] = 0.0;
    for (int v = begin; v < end; v += step) {
        const double t = t_of<T>(to_float(z_row[v]), c), tr = t_of<T>(to_float(r_row[v]), cr);
        const double e = exp2(t);  // (what fp32 has no number for counts beside a logarithm of 1e38)
        sum[0] += e;
        sum[2] += exp2_fast((float)tr);
        if (e != 0.0) {
            sum[1] += e * t;
            sum[3] += e * (t - tr);
        }
    }
}

// Does the policy lie above the low value where the reference lies below?  A thread's pieces of a part, both raised; the
// reference's memory is looked at only where its word is at the low value.  Elements begin .. end of `r` are the row's.
template <typename T>
__device__ __noinline__ bool odd_meets(const uint4 *z_s, const uint4 *r_s, const T *r, int n, int begin, int end)
{
    constexpr int V = Row<T>::kVec;
    const uint32_t low_w = low_word<T>();
    for (int j = threadIdx.x; j < n; j += blockDim.x) {
        const uint4 z = z_s[j], q = r_s[j];
        bool may = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) may |= meets<T, true>(words(z)[i], words(q)[i], low_w);
        if (!may) continue;
        float zv[V];
        unpack<T>(z, zv);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int v = j * V + k;
            if (v >= begin && v < end && zv[k] > low_value<T>() && to_float(r[v]) < low_value<T>()) return true;
        }
    }
    return false;
}

// and their gradients (f: of the row)
template <typename T>
__device__ __noinline__ void odd_gradient(const T *z_row, const T *r_row, T *g_row, int begin, int end, int step, int a, const RowCoef &f)
{
    for (int v = begin; v < end; v += step) {
        const double t = t_of<T>(to_float(z_row[v]), f.c);
        const double e = exp2(t);
        double b = (double)f.k0 + (double)f.kt * t;
        if (f.kr != 0.f) b -= (double)f.kr * t_of<T>(to_float(r_row[v]), f.cr);
        g_row[v] = from_float<T>((e != 0.0 ? (float)(e * b) : 0.f) + (v == a ? f.at_a : 0.f));
    }
}

// A whole odd row by a warp.  (Apart, and with nothing of the caller's to come back to: what is kept across a call costs the
// rows that are not odd registers, 8 to 14 % of their time.)
template <typename T>
__device__ __noinline__ void odd_row(const LossArgs &p, long long row, float w, int a, float za)
{
    const int lane = threadIdx.x & 31;
    const T *z_row = static_cast<const T *>(p.logits) + row * p.ld, *r_row = static_cast<const T *>(p.ref) + row * p.ld_ref;
    float C = -INFINITY, CR = -INFINITY;
    for (int v = lane; v < p.A; v += 32) {
        C = max_nan(C, to_float(z_row[v]));
        CR = max_nan(CR, to_float(r_row[v]));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        C = max_nan(C, __shfl_xor_sync(0xffffffffu, C, o));
        CR = max_nan(CR, __shfl_xor_sync(0xffffffffu, CR, o));
    }
    double sum[4];
    odd_sums<T>(z_row, r_row, lane, p.A, 32, C, CR, sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    const RowCoef f = row_coef<true>(p, row, w, a >= 0, za, C, CR, sum[0], sum[1], sum[2], sum[3], excess_of<T>(C), lane == 0);
    if (p.grad) odd_gradient<T>(z_row, r_row, static_cast<T *>(p.grad) + row * p.ld_grad, lane, p.A, 32, a, f);
}

// Rows of up to 256 pieces of 16 bytes: a warp per row, the row in its registers (45486 rows of 551 fp32: 75 us, a CTA a
// row 214; its wait for memory and its shuffles are a chain, so registers are kept few: 1, 2, 4 or 8 pieces a lane).
constexpr int kWarpPieces = 8;
template <typename T, bool REF, int NV>
__global__ void __launch_bounds__(128, NV * (REF ? 2 : 1) <= 4 ? 6 : NV * (REF ? 2 : 1) <= 8 ? 5 : 4) loss_warp_kernel(const __grid_constant__ LossArgs p)
{
    constexpr int V = Row<T>::kVec;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const float w = weight_of(p, row);
    const T *z_row = static_cast<const T *>(p.logits) + row * p.ld;
    const T *r_row = REF ? static_cast<const T *>(p.ref) + row * p.ld_ref : z_row;
    T *g_row = p.grad ? static_cast<T *>(p.grad) + row * p.ld_grad : nullptr;
    const int first = lane * V - phase_of(z_row), step = 32 * V;
    if (w == 0.f) {
        if (lane == 0) skip_row(p, row);
        const float zero[V] = {};
        if (g_row)
            for (int i = 0; i < NV; ++i) store_piece<T>(g_row, first + i * step, p.A, zero);
        return;
    }
    uint4 raw[NV], raw_r[REF ? NV : 1];
    raw_r[0] = make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        raw[i] = load_piece<T, true>(z_row, first + i * step, p.A, -INFINITY);
        if constexpr (REF) raw_r[i] = load_piece<T>(r_row, first + i * step, p.A, low_value<T>());
    }
    const long long wanted = action_of(p, row);
    const int a = wanted >= 0 && wanted < p.A ? (int)wanted : -1;
    const float za = a >= 0 ? to_float(z_row[a]) : NAN;
    const uint32_t low_w = low_word<T>();
    float low[2];
    unpack_word(low_w, low, (const T *)nullptr);
    // the maximum; -inf raised to the low value; pieces are relative to `base` (0, or the maximum of a row that is apart)
    auto prepare = [&](auto &x, const T *x_row, float &base) {
        uint32_t m = low_w;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                words(x[i])[j] = max_words<T>(words(x[i])[j], low_w);
                m = max_words<T>(m, words(x[i])[j]);
            }
        float c = word_max<T>(m);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) c = max_nan(c, __shfl_xor_sync(0xffffffffu, c, o));
        base = 0.f;
        if (apart<T>(c)) {
            c = -INFINITY;
            for (int v = lane; v < p.A; v += 32) c = fmaxf(c, to_float(x_row[v]));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
            if (c != -INFINITY) {
                base = c;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float z[V];
                    x[i] = load_piece<T>(x_row, first + i * step, p.A, -INFINITY);
                    unpack<T>(x[i], z);
#pragma unroll
                    for (int k = 0; k < V; ++k) z[k] = fmaxf(z[k] - c, low[0]);
                    x[i] = pack<T>(z);
                }
            }
        }
        return c;
    };
    float base, base_r = 0.f;
    const float C = prepare(raw, z_row, base);
    float CR = -INFINITY;
    if constexpr (REF) {
        uint32_t least = low_w;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) least = min_words<T>(least, words(raw_r[i])[j]);
        bool odd = false;
        if (word_min<T>(least) < low[0]) {
            odd = apart<T>(C);  // (what the policy's words stand for is not in them)
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) odd |= meets<T>(words(raw[i])[j], words(raw_r[i])[j], low_w);
        }
        odd = __any_sync(0xffffffffu, odd);
        CR = prepare(raw_r, r_row, base_r);
        if (odd || too_high<T>(CR)) return odd_row<T>(p, row, w, a, za);
    }
    float so = 0.f, st = 0.f, ss = 0.f, sd = 0.f;
    float sh = shift_of<T>(base, C), shr = shift_of<T>(base_r, CR);
#pragma unroll
    for (int i = 0; i < NV; ++i) add_sums<T, REF>(raw[i], raw_r[REF ? i : 0], sh, shr, so, st, ss, sd);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        so += __shfl_xor_sync(0xffffffffu, so, o);
        st += __shfl_xor_sync(0xffffffffu, st, o);
        if (REF) {
            ss += __shfl_xor_sync(0xffffffffu, ss, o);
            sd += __shfl_xor_sync(0xffffffffu, sd, o);
        }
    }
    const RowCoef f = row_coef<REF>(p, row, w, a >= 0, za, C, CR, so, st, CR == -INFINITY ? 0.0 : (double)ss, sd, excess_of<T>(C), lane == 0);
    if (!g_row) return;
    asm volatile("" : "+f"(sh), "+f"(shr));  // (t anew: kept from the sums it would take the registers that hold the row)
#pragma unroll
    for (int i = 0; i < NV; ++i) put_gradient<T, REF>(p, g_row, first + i * step, a, raw[i], raw_r[REF ? i : 0], f, sh, shr);
}

struct Partial {  // of one CTA: maxima, and sums relative to their shifts
    double so, st, ss, sd;
    float c, cr;
    int rare;  // 1: odd; 2: odd if the whole row is masked
};

// what t of a part with maximum c lacks to t of the row, whose maximum is C
template <typename T>
__device__ __forceinline__ float rebase(float c, float C) { return fmaf(c - C, kLog2e, excess_of<T>(C) - excess_of<T>(c)); }
// A whole odd row by a cluster, elements begin .. end by this CTA.  `parts`: the CTAs' maxima, which all have read; `scratch`: of
// the CTA, [kRowThreads / 32][4]; `coef`: of the CTA.
constexpr int kMaxCluster = 16, kRowThreads = 256;
template <typename T>
__device__ __noinline__ void odd_cluster_row(const LossArgs &p, long long row, float w, int a, float za, int begin, int end, Partial *parts,
                                             double *scratch, RowCoef *coef)
{
    namespace cg = cooperative_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
    const int share = (int)cg::this_cluster().num_blocks(), rank = (int)cg::this_cluster().block_rank();
    const T *z_row = static_cast<const T *>(p.logits) + row * p.ld, *r_row = static_cast<const T *>(p.ref) + row * p.ld_ref;
    float C = -INFINITY, CR = -INFINITY;
    for (int i = 0; i < share; ++i) {
        C = max_nan(C, parts[i].c);
        CR = max_nan(CR, parts[i].cr);
    }
    cg::this_cluster().sync();  // (the parts are written again)
    double sum[4];
    odd_sums(z_row, r_row, begin + (int)threadIdx.x, end, (int)blockDim.x, C, CR, sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if (lane < 4) scratch[4 * warp + lane] = lane == 0 ? sum[0] : lane == 1 ? sum[1] : lane == 2 ? sum[2] : sum[3];
    __syncthreads();
    if ((int)threadIdx.x < share) {
        double v[4] = {};
        for (int i = 0; i < warps; ++i)
            for (int k = 0; k < 4; ++k) v[k] += scratch[4 * i + k];
        Partial *to = cg::this_cluster().map_shared_rank(&parts[rank], threadIdx.x);
        to->so = v[0], to->st = v[1], to->ss = v[2], to->sd = v[3];
    }
    cg::this_cluster().sync();
    if (threadIdx.x == 0) {
        double v[4] = {};
        for (int i = 0; i < share; ++i) v[0] += parts[i].so, v[1] += parts[i].st, v[2] += parts[i].ss, v[3] += parts[i].sd;
        *coef = row_coef<true>(p, row, w, a >= 0, za, C, CR, v[0], v[1], v[2], v[3], excess_of<T>(C), rank == 0);
    }
    __syncthreads();
    if (p.grad)
        odd_gradient<T>(z_row, r_row, static_cast<T *>(p.grad) + row * p.ld_grad, begin + (int)threadIdx.x, end, (int)blockDim.x, a, *coef);
}

// Longer rows: the CTAs of a cluster share a row (one CTA up to 72 KB of it, the reference's included), each keeps its part in
// shared memory from one read of it to the gradient.  Bulk copies bring it in; what is not whole 16 bytes, or lies otherwise
// to 16 bytes than the logits do, goes through registers.  Three or four CTAs fit an SM: while one waits for its part or
// for its cluster, the others compute and write.  What bounds it beside HBM is the instructions a logit (some
// 17, 34 with a reference row, counted under a profiler; at the rate of HBM there is time for 22 and 33): so -inf is made
// finite and the maximum found two 16-bit logits at a time, t is one multiply-add of the logit, and what depends on the row
// only is worked out by one warp.  Sums of a warp are float, from there on double.  4096 rows of 49999 bf16: 171 to 177 us,
// 4.7 TB/s; 2048 of 128001 with a reference: 497 us.
template <typename T, bool REF>
__global__ void __launch_bounds__(kRowThreads, 4) loss_rows_kernel(const __grid_constant__ LossArgs p)
{
    constexpr int V = Row<T>::kVec;
    extern __shared__ __align__(128) uint4 s_piece[];  // [REF ? 2 : 1][pieces of a part]
    __shared__ Partial parts[kMaxCluster];
    __shared__ float4 s_sum[kRowThreads / 32];
    __shared__ float s_max[2][kRowThreads / 32];
    __shared__ RowCoef s_row;
    __shared__ uint64_t s_bar;
    __shared__ int s_abort, s_odd;
    namespace cg = cooperative_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = (int)blockDim.x >> 5;
    const int share = (int)cg::this_cluster().num_blocks(), rank = (int)cg::this_cluster().block_rank();
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long row = (long long)(blockIdx.x / (unsigned)share);
    const float w = weight_of(p, row);
    const T *z_row = static_cast<const T *>(p.logits) + row * p.ld;
    const T *r_row = REF ? static_cast<const T *>(p.ref) + row * p.ld_ref : z_row;
    T *g_row = p.grad ? static_cast<T *>(p.grad) + row * p.ld_grad : nullptr;
    // pieces start at multiples of 16 bytes of the logits
    const int phase = phase_of(z_row), pieces = (phase + p.A + V - 1) / V;
    const int j0 = (int)((long long)pieces * rank / share), n = (int)((long long)pieces * (rank + 1) / share) - j0;
    const int first = j0 * V - phase;  // element of the part's first piece
    if (w == 0.f) {
        asm volatile("barrier.cluster.wait;" ::: "memory");
        if (rank == 0 && threadIdx.x == 0) skip_row(p, row);
        const float zero[V] = {};
        if (g_row)
            for (int j = threadIdx.x; j < n; j += blockDim.x) store_piece<T>(g_row, first + j * V, p.A, zero);
        return;
    }
    uint4 *z_s = s_piece, *r_s = s_piece + (REF ? p.part_pieces : 0);
    const bool alike = phase_of(r_row) == phase;
    const int whole0 = first < 0 ? 1 : 0, whole1 = first + n * V > p.A ? n - 1 : n;  // whole pieces of the part
    if (threadIdx.x < 2 * (kRowThreads / 32)) s_max[threadIdx.x / (kRowThreads / 32)][threadIdx.x % (kRowThreads / 32)] = -INFINITY;
    if (threadIdx.x == 0) {
        s_abort = 0;
        mbar_init(smem_u32(&s_bar), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        const uint32_t bytes = whole1 > whole0 ? (uint32_t)(whole1 - whole0) * 16u : 0u;
        mbar_expect_tx(smem_u32(&s_bar), bytes * (REF && alike ? 2u : 1u));
        if (bytes) {
            bulk_load(smem_u32(z_s + whole0), z_row + first + whole0 * V, bytes, smem_u32(&s_bar));
            if (REF && alike) bulk_load(smem_u32(r_s + whole0), r_row + first + whole0 * V, bytes, smem_u32(&s_bar));
        }
    }
    if (threadIdx.x < 2) {  // the part's ends
        const int j = threadIdx.x == 0 ? 0 : n - 1;
        if (n > 0 && (j < whole0 || j >= whole1)) {
            z_s[j] = load_piece<T>(z_row, first + j * V, p.A, -INFINITY);
            if (REF && alike) r_s[j] = load_piece<T>(r_row, first + j * V, p.A, low_value<T>());
        }
    }
    if (REF && !alike)
        for (int j = threadIdx.x; j < n; j += blockDim.x) r_s[j] = load_piece<T>(r_row, first + j * V, p.A, low_value<T>());
    const long long wanted = action_of(p, row);
    const int a = wanted >= 0 && wanted < p.A ? (int)wanted : -1;
    const float za = a >= 0 ? to_float(z_row[a]) : NAN;  // (`grad` may be `logits`: read before the barriers below)
    __syncthreads();
    mbar_wait(smem_u32(&s_bar), 0, &s_abort, &g_status, 1);

    const uint32_t low_w = low_word<T>();
    float low[2];
    unpack_word(low_w, low, (const T *)nullptr);
    // a pass of the part: -inf raised to the low value, the maximum; in every thread of the CTA
    bool lower = false, odd = false;  // the reference below the low value; and the policy above it there
    auto prepare = [&](uint4 *x_s, int which) {
        uint32_t m = low_w, least = low_w;
        for (int j = threadIdx.x; j < n; j += blockDim.x) {
            uint4 v = x_s[j];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (which) least = min_words<T>(least, words(v)[i]);
                words(v)[i] = max_words<T>(words(v)[i], low_w);
                m = max_words<T>(m, words(v)[i]);
            }
            x_s[j] = v;
        }
        if (which && word_min<T>(least) < low[0]) {  // (apart from the loop above, which is every row's)
            lower = true;
            odd = odd_meets<T>(z_s, x_s, r_row + first, n, first < 0 ? -first : 0, p.A - first);
        }
        float c = word_max<T>(m);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) c = max_nan(c, __shfl_xor_sync(0xffffffffu, c, o));
        if (lane == 0) s_max[which][warp] = c;
    };
    auto block_max = [&](int which) {
        float c = s_max[which][lane & (kRowThreads / 32 - 1)];
#pragma unroll
        for (int o = kRowThreads / 64; o > 0; o >>= 1) c = max_nan(c, __shfl_xor_sync(0xffffffffu, c, o));
        return c;
    };
    // a part that is apart: read again, relative to its own maximum (returned; -inf: no logit)
    auto low_part = [&](uint4 *x_s, const T *x_row, int which) {
        float c = -INFINITY;
        for (int v = max(first, 0) + (int)threadIdx.x; v < min(first + n * V, p.A); v += blockDim.x) c = fmaxf(c, to_float(x_row[v]));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
        __syncthreads();
        if (lane == 0) s_max[which][warp] = c;
        __syncthreads();
        c = block_max(which);
        if (c != -INFINITY)
            for (int j = threadIdx.x; j < n; j += blockDim.x) {
                float z[V];
                unpack<T>(load_piece<T>(x_row, first + j * V, p.A, -INFINITY), z);
#pragma unroll
                for (int k = 0; k < V; ++k) z[k] = fmaxf(z[k] - c, low[0]);
                x_s[j] = pack<T>(z);
            }
        return c;
    };
    prepare(z_s, 0);
    if (REF) prepare(r_s, 1);
    odd = __syncthreads_or(odd);
    float c = block_max(0), cr = REF ? block_max(1) : -INFINITY, base = 0.f, base_r = 0.f;
    // (entries masked in both arrays: what the policy's words stood for was not in them, but it counts only if the whole row is
    // like that, which the CTAs learn from one another)
    int rare = 0;
    if (apart<T>(c)) {
        if (REF && __syncthreads_or(lower && is_below<T>(c))) rare = 2;
        c = low_part(z_s, z_row, 0);
        base = c == -INFINITY ? 0.f : c;
    }
    if (REF && (odd || too_high<T>(cr))) rare = 1;
    if (REF && apart<T>(cr)) {
        cr = low_part(r_s, r_row, 1);
        base_r = cr == -INFINITY ? 0.f : cr;
    }
    float so = 0.f, st = 0.f, ss = 0.f, sd = 0.f;
    {
        const float sh = shift_of<T>(base, c), shr = shift_of<T>(base_r, cr);
#pragma unroll 2
        for (int j = threadIdx.x; j < n; j += blockDim.x) add_sums<T, REF>(z_s[j], r_s[j], sh, shr, so, st, ss, sd);
    }
    float sums[4] = {so, st, ss, sd};
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < (REF ? 4 : 2); ++i) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], o);
    if (lane == 0) s_sum[warp] = make_float4(sums[0], sums[1], sums[2], sums[3]);
    __syncthreads();
    asm volatile("barrier.cluster.wait;" ::: "memory");  // every CTA of the cluster has started
    if (warp == 0) {
        Partial mine;
        const float4 part = lane < warps ? s_sum[lane] : make_float4(0.f, 0.f, 0.f, 0.f);
        double v[4] = {part.x, part.y, part.z, part.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int o = kRowThreads / 64; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        if (share > kRowThreads / 32) {  // (the sums are in the lanes that have a warp each; a lane sends to each CTA)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __shfl_sync(0xffffffffu, v[i], lane % (kRowThreads / 32));
        }
        mine.so = c == -INFINITY ? 0.0 : v[0];
        mine.st = c == -INFINITY ? 0.0 : v[1];
        mine.ss = cr == -INFINITY ? 0.0 : v[2];
        mine.sd = c == -INFINITY ? 0.0 : v[3];
        mine.c = c;
        mine.cr = cr;
        mine.rare = rare;
        if (lane < share) *cg::this_cluster().map_shared_rank(&parts[rank], lane) = mine;
    }
    cg::this_cluster().sync();
    if (warp == 0) {
        Partial b = parts[lane < share ? lane : 0];
        if (lane >= share) {
            b.so = b.st = b.ss = b.sd = 0.0;
            b.c = b.cr = -INFINITY;
        }
        float C = b.c, CR = b.cr;
#pragma unroll
        for (int o = kMaxCluster / 2; o > 0; o >>= 1) {
            C = max_nan(C, __shfl_xor_sync(0xffffffffu, C, o));
            CR = max_nan(CR, __shfl_xor_sync(0xffffffffu, CR, o));
        }
        // a part's sums, relative to the row's shifts (as the gradient takes them) instead of its own
        const float d = b.so != 0.0 ? rebase<T>(b.c, C) : 0.f, dr = b.ss != 0.0 ? rebase<T>(b.cr, CR) : 0.f;
        const double f = (double)exp2f(d), df = (double)d, dd = (double)(d - dr);
        double v[4] = {f * b.so, f != 0.0 ? f * (b.st + df * b.so) : 0.0, (double)exp2f(dr) * b.ss, f != 0.0 ? f * (b.sd + dd * b.so) : 0.0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int o = kMaxCluster / 2; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        // (the vote is of all lanes; those from 16 on have no part, and another C)
        const int any = REF ? __reduce_or_sync(0xffffffffu, b.rare) : 0;
        if (REF && lane == 0) s_odd = (any & 1) || (any && is_below<T>(C));
        if (!any || !((any & 1) || is_below<T>(C))) {
            const RowCoef r = row_coef<REF>(p, row, w, a >= 0, za, C, CR, v[0], v[1], v[2], v[3], excess_of<T>(C), rank == 0 && lane == 0);
            if (lane == 0) s_row = r;
        }
    }
    __syncthreads();
    if (REF && s_odd)  // (the same in every CTA of the cluster)
        return odd_cluster_row<T>(p, row, w, a, za, max(first, 0), min(first + n * V, p.A), parts, reinterpret_cast<double *>(s_piece), &s_row);
    if (g_row) {
        RowCoef f = s_row;
        float sh = shift_of<T>(base, f.c), shr = shift_of<T>(base_r, f.cr);
        if (base == 0.f && apart<T>(f.c)) {  // a part that is not in a row that is
            if (c == -INFINITY) {
                sh = -1e30f;  // (no logit here)
            } else {  // (far up: what the shift is off by where the part's logits are near enough to matter)
                const float scale = exp2f(-fminf(fmaxf(fmaf(f.c, kLog2e, sh), -4.f), 4.f));
                f.k0 *= scale, f.kt *= scale, f.kr *= scale;
            }
        }
        if (REF && (f.kr == 0.f || (base_r == 0.f && is_below<T>(f.cr)))) shr = 0.f;  // (it does not count; no logit here, and the policy's are masked)
#pragma unroll 2
        for (int j = threadIdx.x; j < n; j += blockDim.x) put_gradient<T, REF>(p, g_row, first + j * V, a, z_s[j], r_s[j], f, sh, shr);
    }
    if (s_abort)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
}

// ------------------------------------------------------------------- many very long rows with a reference
// A CTA per row, persistent, the row streaming through a ring in shared memory twice: for the sums, and, backwards, for the
// gradient.  The second time it comes from L2, as far as that holds the rows of all CTAs.  Against
// the kernel above a row's end (barriers, one warp's arithmetic: some 2 us in which an SM does little else) comes once for
// a whole row instead of once for an eighth of one, and the loads of what follows go on meanwhile: 497 -> 414 us for
// 2048 rows of 128001.  It is bound by the instructions a pair of logits (some 34; 16 warps instead of 24: 492 us), so every
// thread keeps a maximum of its own and rebases its sums when it rises.  Without a reference, which halves them, the
// kernel above is no slower.
constexpr int kStreamWarps = 24, kStreamThreads = 32 * kStreamWarps, kStreamPer = 2, kStreamStages = 4;
constexpr int kStreamPieces = kStreamPer * kStreamThreads;  // of an array, a stage
constexpr int kStreamSmem = kStreamStages * 2 * 16 * kStreamPieces;

template <typename T>
__global__ void __launch_bounds__(kStreamThreads + 32, 1) loss_stream_kernel(const __grid_constant__ LossArgs p)
{
    constexpr int V = Row<T>::kVec, kStages = kStreamStages;
    constexpr bool REF = true;
    extern __shared__ __align__(128) uint4 s_piece[];  // [kStages][2][kStreamPieces]
    __shared__ uint64_t s_full[kStages], s_empty[kStages];
    __shared__ Partial s_part[kStreamWarps];
    __shared__ RowCoef s_row;
    __shared__ int s_odd, s_abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_empty[i]), kStreamWarps);
        }
        s_abort = s_odd = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    // a row's whole pieces [w0, w1) and the chunks of them that fill a stage
    auto whole = [&](const T *z_row, int *phase, int *w0, int *w1) {
        *phase = phase_of(z_row);
        const int pieces = (*phase + p.A + V - 1) / V;
        *w0 = *phase > 0;
        *w1 = pieces * V - *phase > p.A ? pieces - 1 : pieces;
        return (*w1 - *w0 + kStreamPieces - 1) / kStreamPieces;
    };
    int slot = 0, phase, w0, w1;
    uint32_t turn = 0;
    auto next = [&] {
        if (++slot == kStages) {
            slot = 0;
            turn ^= 1;
        }
    };
    if (warp == kStreamWarps) {
        // ------------------------------------------------------------------------------------- loads
        for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
            if (weight_of(p, row) == 0.f) continue;
            const T *z_row = static_cast<const T *>(p.logits) + row * p.ld, *r_row = static_cast<const T *>(p.ref) + row * p.ld_ref;
            const int chunks = whole(z_row, &phase, &w0, &w1);
            for (int i = 0; i < (p.grad ? 2 : 1) * chunks; ++i) {
                const int c = i < chunks ? i : 2 * chunks - 1 - i, j = w0 + c * kStreamPieces;
                if (!mbar_wait(smem_u32(&s_empty[slot]), turn ^ 1, &s_abort, &g_status, 2)) break;
                if (elect_one()) {
                    const uint32_t bytes = 16u * (uint32_t)min(kStreamPieces, w1 - j), at = smem_u32(s_piece + slot * 2 * kStreamPieces);
                    mbar_expect_tx(smem_u32(&s_full[slot]), 2 * bytes);
                    bulk_load(at, z_row + j * V - phase, bytes, smem_u32(&s_full[slot]));
                    bulk_load(at + 16 * kStreamPieces, r_row + j * V - phase, bytes, smem_u32(&s_full[slot]));
                }
                __syncwarp();
                next();
            }
        }
    } else {
        auto all = [] { asm volatile("bar.sync 1, %0;" ::"n"(kStreamThreads) : "memory"); };
        const uint32_t low_w = low_word<T>();
        float low[2];
        unpack_word(low_w, low, (const T *)nullptr);
        // (both arrays' words, in both passes: a logarithm far below the rest, times a coefficient, is to stay finite, since it
        // meets a probability of 0)
        auto raise = [&](uint4 &x) {
#pragma unroll
            for (int i = 0; i < 4; ++i) words(x)[i] = max_words<T>(words(x)[i], low_w);
        };
        for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
            const float w = weight_of(p, row);
            const T *z_row = static_cast<const T *>(p.logits) + row * p.ld, *r_row = static_cast<const T *>(p.ref) + row * p.ld_ref;
            T *g_row = p.grad ? static_cast<T *>(p.grad) + row * p.ld_grad : nullptr;
            const int chunks = whole(z_row, &phase, &w0, &w1);
            if (w == 0.f) {
                if (threadIdx.x == 0) skip_row(p, row);
                const float zero[V] = {};
                if (g_row)
                    for (int v = (int)threadIdx.x * V - phase; v < p.A; v += kStreamThreads * V) store_piece<T>(g_row, v, p.A, zero);
                continue;
            }
            // the pieces at the row's ends that are not whole: the first thread's and the second's
            const int ragged = threadIdx.x == 0 && w0 > 0 ? -phase : threadIdx.x == 1 && w1 * V - phase < p.A ? w1 * V - phase : INT_MIN;
            const long long wanted = action_of(p, row);
            const int a = wanted >= 0 && wanted < p.A ? (int)wanted : -1;
            const float za = a >= 0 ? to_float(z_row[a]) : NAN;
            Partial s;
            float so = 0.f, st = 0.f, ss = 0.f, sd = 0.f, c = low[0], cr = low[0];
            bool meet = false;  // the reference below the low value where the policy is above it
            // what a thread's sums are relative to: its maximum, or 0 as long as it has met nothing above the low value
            auto shift = [&](float most) { return most <= low[0] ? 0.f : minus_log2(most); };
            float nc = 0.f, ncr = 0.f;  // their shifts
            auto take = [&](uint4 raw, uint4 raw_r) {
                uint32_t m = low_w, mr = low_w, below = 0;
                const uint4 was = raw_r;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    words(raw)[i] = max_words<T>(words(raw)[i], low_w);
                    m = max_words<T>(m, words(raw)[i]);
                    if constexpr (REF) {
                        words(raw_r)[i] = max_words<T>(words(raw_r)[i], low_w);
                        mr = max_words<T>(mr, words(raw_r)[i]);
                        below |= words(raw_r)[i] ^ words(was)[i];
                    }
                }
                const float top = word_max<T>(m);
                if (top > c) {
                    c = top;
                    const float to = minus_log2(c), d = so != 0.f ? to - nc : 0.f, f = exp2_fast(d);
                    st = f * (st + d * so);
                    sd = f * (sd + d * so);
                    so *= f;
                    nc = to;
                }
                if constexpr (REF) {
                    if (below) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) meet |= meets<T>(words(raw)[i], words(was)[i], low_w);
                    }
                    const float top_r = word_max<T>(mr);
                    if (top_r > cr) {
                        cr = top_r;
                        const float to = minus_log2(cr);
                        sd -= (to - ncr) * so;
                        ss *= exp2_fast(ss != 0.f ? to - ncr : 0.f);
                        ncr = to;
                    }
                }
                add_sums<T, REF>(raw, raw_r, nc, ncr, so, st, ss, sd);
            };
            if (ragged != INT_MIN)
                take(load_piece<T>(z_row, ragged, p.A, -INFINITY), load_piece<T>(r_row, ragged, p.A, low[0]));
            for (int i = 0; i < chunks; ++i) {
                const int j = w0 + i * kStreamPieces + (int)threadIdx.x;
                mbar_wait(smem_u32(&s_full[slot]), turn, &s_abort, &g_status, 1);
                const uint4 *at = s_piece + slot * 2 * kStreamPieces + threadIdx.x;
#pragma unroll
                for (int h = 0; h < kStreamPer; ++h)
                    if (j + h * kStreamThreads < w1) take(at[h * kStreamThreads], at[kStreamPieces + h * kStreamThreads]);
                // (always so; it waits for the values to be in every lane's registers, not merely asked for)
                if (__all_sync(0xffffffffu, c >= low[0] && cr >= low[0]) && lane == 0) mbar_arrive(smem_u32(&s_empty[slot]));
                next();
            }
            // a warp's sums, relative to its maxima
            s.c = c;
            s.cr = cr;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                s.c = max_nan(s.c, __shfl_xor_sync(0xffffffffu, s.c, o));
                s.cr = max_nan(s.cr, __shfl_xor_sync(0xffffffffu, s.cr, o));
            }
            {
                const float d = so != 0.f ? shift(s.c) - nc : 0.f, dr = shift(s.cr) - ncr, f = exp2f(d);
                st = f != 0.f ? f * (st + d * so) : 0.f;
                sd = f != 0.f ? f * (sd + (d - dr) * so) : 0.f;
                so *= f;
                ss *= exp2f(ss != 0.f ? dr : 0.f);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                so += __shfl_xor_sync(0xffffffffu, so, o);
                st += __shfl_xor_sync(0xffffffffu, st, o);
                if (REF) {
                    ss += __shfl_xor_sync(0xffffffffu, ss, o);
                    sd += __shfl_xor_sync(0xffffffffu, sd, o);
                }
            }
            s.so = so, s.st = st, s.ss = ss, s.sd = sd;
            if (lane == 0) s_part[warp] = s;
            if (meet || ss != ss) s_odd = 1;  // (a NaN passes by the maximum, not by the sum)
            all();
            float C = s_part[lane % kStreamWarps].c, CR = s_part[lane % kStreamWarps].cr;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                C = max_nan(C, __shfl_xor_sync(0xffffffffu, C, o));
                CR = max_nan(CR, __shfl_xor_sync(0xffffffffu, CR, o));
            }
            // One of the rows far from 0 (masks of the type's lowest value only, or none left at all), a broken reference, or the
            // reference below the low value where the policy is not: the row is done from memory, value by value.
            const bool odd = apart<T>(C) || is_below<T>(CR) || too_high<T>(CR) || s_odd;
            if (odd) {
                C = CR = -INFINITY;
                for (int v = threadIdx.x; v < p.A; v += kStreamThreads) {
                    C = max_nan(C, to_float(z_row[v]));
                    CR = max_nan(CR, to_float(r_row[v]));
                }
                all();  // (the parts have been read)
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    C = max_nan(C, __shfl_xor_sync(0xffffffffu, C, o));
                    CR = max_nan(CR, __shfl_xor_sync(0xffffffffu, CR, o));
                }
                if (lane == 0) s_part[warp].c = C, s_part[warp].cr = CR;
                all();
                for (int i = 0; i < kStreamWarps; ++i) {
                    C = max_nan(C, s_part[i].c);
                    CR = max_nan(CR, s_part[i].cr);
                }
                all();
                double v4[4];
                odd_sums(z_row, r_row, threadIdx.x, p.A, kStreamThreads, C, CR, v4);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v4[i] += __shfl_xor_sync(0xffffffffu, v4[i], o);
                s.c = C, s.cr = CR, s.so = v4[0], s.st = v4[1], s.ss = v4[2], s.sd = v4[3];
                if (C == -INFINITY) s.so = s.st = s.sd = 0.0;
                if (lane == 0) s_part[warp] = s;
                all();
            }
            if (warp == 0) {
                const Partial b = s_part[lane % kStreamWarps];
                const float d = b.so != 0.0 ? rebase<T>(b.c, C) : 0.f, dr = b.ss != 0.0 ? rebase<T>(b.cr, CR) : 0.f;
                const double f = lane < kStreamWarps ? (double)exp2f(d) : 0.0, df = (double)d, dd = (double)(d - dr);
                double v[4] = {f * b.so, f != 0.0 ? f * (b.st + df * b.so) : 0.0, lane < kStreamWarps ? (double)exp2f(dr) * b.ss : 0.0,
                               f != 0.0 ? f * (b.sd + dd * b.so) : 0.0};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
                const RowCoef f0 = row_coef<REF>(p, row, w, a >= 0, za, C, CR, v[0], v[1], v[2], v[3], excess_of<T>(C), lane == 0);
                if (lane == 0) {
                    s_row = f0;
                    if (s_odd) s_odd = 0;  // (then every warp has come past two barriers since it looked)
                }
            }
            all();
            if (!g_row) continue;
            const RowCoef f = s_row;
            const float sh = shift_of<T>(0.f, f.c), shr = shift_of<T>(0.f, f.cr);
            if (!odd && ragged != INT_MIN) {
                uint4 raw = load_piece<T>(z_row, ragged, p.A, low[0]), raw_r = load_piece<T>(r_row, ragged, p.A, low[0]);
                raise(raw);
                raise(raw_r);
                put_gradient<T, REF>(p, g_row, ragged, a, raw, raw_r, f, sh, shr);
            }
            for (int i = chunks - 1; i >= 0; --i) {
                const int j = w0 + i * kStreamPieces + (int)threadIdx.x;
                mbar_wait(smem_u32(&s_full[slot]), turn, &s_abort, &g_status, 1);
                const uint4 *at = s_piece + slot * 2 * kStreamPieces + threadIdx.x;
#pragma unroll
                for (int h = 0; h < kStreamPer; ++h)
                    if (!odd && j + h * kStreamThreads < w1) {
                        uint4 raw = at[h * kStreamThreads], raw_r = at[kStreamPieces + h * kStreamThreads];
                        raise(raw);
                        raise(raw_r);
                        put_gradient<T, REF>(p, g_row, (j + h * kStreamThreads) * V - phase, a, raw, raw_r, f, sh, shr);
                    }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s_empty[slot]));
                next();
            }
            if (odd) odd_gradient(z_row, r_row, g_row, threadIdx.x, p.A, kStreamThreads, a, f);
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (s_abort)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);  // copies still in flight land first
}

// ---------------------------------------------------------------------------------------------- launch
template <typename T, bool REF, bool STATS>
auto narrow_kernel(int g)
{
    return g == 1 ? loss_narrow_kernel<T, REF, 1, STATS> : g == 2 ? loss_narrow_kernel<T, REF, 2, STATS>
         : g == 4 ? loss_narrow_kernel<T, REF, 4, STATS> : loss_narrow_kernel<T, REF, 8, STATS>;
}

// `done`: the sums over rows have been taken too (rows that fit one CTA: a second launch costs some 3 us)
template <typename T, bool REF>
cudaError_t launch_narrow(const LossArgs &p, float *stats, bool *done, cudaStream_t st)
{
    int g = 1;
    while (g * kNarrowPer < p.A) g *= 2;
    const long long threads = (long long)p.rows * g;
    *done = threads <= 1024;
    if (*done) narrow_kernel<T, REF, true>(g)<<<1, (unsigned)std::max<long long>(64, (threads + 31) / 32 * 32), 0, st>>>(p, stats);
    else narrow_kernel<T, REF, false>(g)<<<(unsigned)((threads + 127) / 128), 128, 0, st>>>(p, nullptr);
    return cudaGetLastError();
}

template <typename T, bool REF>
cudaError_t launch_rows(LossArgs &p, int sm_count, cudaStream_t st)
{
    constexpr int V = Row<T>::kVec;
    const int pieces = (p.A + V - 1 + V - 1) / V;  // a row may start up to V - 1 elements behind a multiple of 16 bytes
    if (pieces <= 32 * kWarpPieces) {
        const auto kernel = pieces <= 32     ? loss_warp_kernel<T, REF, 1>
                            : pieces <= 64   ? loss_warp_kernel<T, REF, 2>
                            : pieces <= 128  ? loss_warp_kernel<T, REF, 4>
                                             : loss_warp_kernel<T, REF, 8>;
        kernel<<<(unsigned)(((long long)p.rows + 3) / 4), 128, 0, st>>>(p);
        return cudaGetLastError();
    }
    // With a reference, rows from 256 KB on (both arrays'), one for every SM or more: streamed.  By the cluster kernel / streamed, us:
    // 148 rows of 128000 bf16 51 / 41, 150 51 / 64 (a second turn for two rows), 200 64 / 66, 300 86 / 92, 444 120 / 98, 888 225 / 184;
    // 2048 of 151936 679 / 467, of 262128 (whose second reading L2 does not serve) 1118 / 820; 2048 of 64000 fp32 414 / 339; shorter
    // ones, 4096 of 32000 bf16, 225 / 274.
    if constexpr (REF) {
        const long long row_bytes = 32LL * pieces;
        const bool alike = !((((uintptr_t)p.ref ^ (uintptr_t)p.logits) | (uintptr_t)((p.ld - p.ld_ref) * (long long)sizeof(T))) & 15);
        if (p.rows >= sm_count && row_bytes >= 256 * 1024 && alike) {
            const auto kernel = loss_stream_kernel<T>;
            const cudaError_t e = allow_smem((const void *)kernel, kStreamSmem);
            if (e != cudaSuccess) return e;
            kernel<<<(unsigned)sm_count, kStreamThreads + 32, kStreamSmem, st>>>(p);
            return cudaGetLastError();
        }
    }
    // As few CTAs a row as keep three of them on an SM (72 KB each); more where the rows alone do not cover the chip.
    const int most = 72 * 1024 / (REF ? 32 : 16);
    int share = 1;
    while (share < kMaxCluster && share * most < pieces) share *= 2;
    while (share < 8 && (long long)p.rows * share < sm_count && pieces >= share * 256) share *= 2;
    p.part_pieces = (pieces + share - 1) / share + 1;
    const size_t smem = (size_t)p.part_pieces * (REF ? 32 : 16);
    const int threads = std::min(kRowThreads, (p.part_pieces + 63) / 64 * 32);
    const auto kernel = loss_rows_kernel<T, REF>;
    cudaError_t e = allow_smem((const void *)kernel, smem);
    if (e == cudaSuccess && share > 8) e = cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)share;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)((long long)p.rows * share));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace

}  // namespace accerl

namespace accerl {

cudaError_t policy_loss_status(int *out)  // (clears it)
{
    cudaError_t e = cudaMemcpyFromSymbol(out, g_status, sizeof(int));
    const int zero = 0;
    if (e == cudaSuccess && *out) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(int));
    return e;
}

}  // namespace accerl

using namespace accerl;

extern "C" accerl_status accerl_policy_loss(const accerl_policy_loss_args *a, void *cuda_stream)
{
    if (!a || !a->logits || !a->actions || !a->logp_old || !a->advantages || !a->logp || !a->kl || !a->entropy ||
        !a->stats || !a->terms) {
        set_error("policy_loss: null argument");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->logits_ref && a->logp_ref) {
        set_error("policy_loss: logits_ref and logp_ref exclude each other");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (!good_dtype(a->dtype)) {
        set_error("policy_loss: unknown dtype %d", a->dtype);
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->rows < 1 || a->rows > (1 << 26) || a->n_actions < 1 || a->n_actions > 262128) {
        set_error("policy_loss: rows must be in 1..2^26 and n_actions in 1..262128");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (a->ld_logits < a->n_actions || (a->logits_ref && a->ld_logits_ref < a->n_actions) ||
        (a->grad && a->ld_grad < a->n_actions) || (a->grad == a->logits && a->ld_grad != a->ld_logits)) {
        set_error("policy_loss: a row distance is below n_actions (or differs between grad and the logits it replaces)");
        return ACCERL_ERR_INVALID_ARG;
    }
    if (!(a->clip_low >= 0.f) || !(a->clip_high >= 0.f) || !isfinite(a->kl_coef) || !isfinite(a->entropy_coef)) {
        set_error("policy_loss: clips must be non-negative, coefficients finite");
        return ACCERL_ERR_INVALID_ARG;
    }
    const int es = dtype_size(a->dtype);
    if ((((uintptr_t)a->logits | (uintptr_t)a->logits_ref | (uintptr_t)a->grad) & (es - 1)) ||
        ((uintptr_t)a->actions & (a->actions64 ? 7 : 3)) || ((uintptr_t)a->terms & 7) ||
        (((uintptr_t)a->logp_old | (uintptr_t)a->advantages | (uintptr_t)a->logp_ref | (uintptr_t)a->weights |
          (uintptr_t)a->logp | (uintptr_t)a->kl | (uintptr_t)a->entropy | (uintptr_t)a->stats) & 3)) {
        set_error("policy_loss: misaligned pointer");
        return ACCERL_ERR_INVALID_ARG;
    }
    LossArgs p;
    p.logits = a->logits;
    p.ref = a->logits_ref;
    p.actions = a->actions;
    p.logp_old = a->logp_old;
    p.advantages = a->advantages;
    p.logp_ref = a->logp_ref;
    p.weights = a->weights;
    p.ld = a->ld_logits;
    p.ld_ref = a->ld_logits_ref;
    p.ld_grad = a->ld_grad;
    p.rows = a->rows;
    p.A = a->n_actions;
    p.actions64 = a->actions64;
    p.clip_low = a->clip_low;
    p.clip_high = a->clip_high;
    p.kl_coef = a->kl_coef;
    p.entropy_coef = a->entropy_coef;
    p.grad = a->grad;
    p.logp = a->logp;
    p.kl = a->kl;
    p.entropy = a->entropy;
    p.terms = a->terms;
    p.part_pieces = 0;
    int device = 0, sm_count = 0;
    ACCERL_CUDA_TRY(cudaGetDevice(&device));
    ACCERL_CUDA_TRY(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, device));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    bool done = false;
    ACCERL_CUDA_TRY(with_dtype(a->dtype, [&](auto v) {
        using T = decltype(v);
        if (p.A <= kNarrow) return p.ref ? launch_narrow<T, true>(p, a->stats, &done, st) : launch_narrow<T, false>(p, a->stats, &done, st);
        return p.ref ? launch_rows<T, true>(p, sm_count, st) : launch_rows<T, false>(p, sm_count, st);
    }));
    if (done) return ACCERL_OK;
    const unsigned ctas = p.rows <= 2048 ? 1 : kStatsCluster;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(p.rows < kStatsThreads ? (unsigned)(p.rows + 31) / 32 * 32 : kStatsThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 2;
    ACCERL_CUDA_TRY(cudaLaunchKernelEx(&cfg, loss_stats_kernel, p, a->stats));
    return ACCERL_OK;
}
