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
#include <math.h>

#include "exp64.cuh"
#include "learn.cuh"

namespace accerl {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr double kLn2 = 0.6931471805599453;

struct LossArgs {
    const void *logits, *ref;
    const void *actions;
    const float *logp_old, *advantages, *logp_ref, *weights;
    long long ld, ld_ref, ld_grad;
    int rows, A, actions64;
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

__device__ __forceinline__ long long action_of(const LossArgs &p, long long row)
{
    return p.actions64 ? static_cast<const long long *>(p.actions)[row] : (long long)static_cast<const int *>(p.actions)[row];
}

__device__ __forceinline__ float weight_of(const LossArgs &p, long long row)
{
    return p.weights ? p.weights[row] : (float)(1.0 / (double)p.rows);
}

// What a row's sums make of it: its outputs, and the gradient's coefficients (natural logarithms: delta_v = log p_v -
// log q_v, lp_v = log p_v):  d loss / d z_v = w p_v (base + kl_coef delta_v + entropy_coef lp_v) + w slope [v = a].
struct RowResult {
    double base, slope;
};
__device__ __forceinline__ RowResult finish_row(const LossArgs &p, long long row, double logp, double kl_full, double H,
                                                bool empty, bool writer)
{
    double kl = kl_full, slope = 0.0, pg = 0.0, r = 0.0;
    if (empty) {
        kl = H = 0.0;
    } else {
        const double adv = (double)p.advantages[row];
        r = exp(logp - (double)p.logp_old[row]);
        const double lo = 1.0 - (double)p.clip_low, hi = 1.0 + (double)p.clip_high;
        const double rc = r < lo ? lo : r > hi ? hi : r;  // (a NaN stays one)
        const double plain = r * adv, clipped = rc * adv;
        const bool inside = !(plain > clipped);
        pg = -(inside ? plain : clipped);
        slope = inside ? -plain : 0.0;
        if (p.logp_ref) {
            const double d = (double)p.logp_ref[row] - logp, e = expm1(d);
            kl = e - d;
            slope -= (double)p.kl_coef * e;
        }
        if (writer && p.terms) *reinterpret_cast<float2 *>(p.terms + 2 * row) = make_float2((float)pg, inside ? (float)r : -(float)r);
    }
    if (writer) {
        if (empty) *reinterpret_cast<float2 *>(p.terms + 2 * row) = make_float2(0.f, 0.f);
        p.logp[row] = (float)logp;
        p.kl[row] = (float)kl;
        p.entropy[row] = (float)H;
    }
    RowResult o;
    o.slope = slope;
    o.base = -slope + (double)p.entropy_coef * H - (p.ref && p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0);
    return o;
}

__device__ __forceinline__ void skip_row(const LossArgs &p, long long row)
{
    p.logp[row] = p.kl[row] = p.entropy[row] = 0.f;
    *reinterpret_cast<float2 *>(p.terms + 2 * row) = make_float2(0.f, 0.f);
}

// ------------------------------------------------------------------------------------------ narrow rows
// Up to 64 actions: a group of G lanes per row, at most 8 elements a lane, in double (two exponentials an element are
// free beside the latencies here, and whether a ratio is clipped is decided where the definition decides it).
constexpr int kNarrow = 64, kNarrowPer = 8;

template <typename T, bool REF, int G>
__global__ void __launch_bounds__(128) loss_narrow_kernel(const __grid_constant__ LossArgs p)
{
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
    const bool empty = mo == -INFINITY;
    if (empty) mo = 0.0;
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
    // the action's logit from the lane that holds it (`grad` may be `logits`: memory is not read again)
    const long long a = work ? action_of(p, row) : -1;
    const bool known = a >= 0 && a < p.A;
    float za = 0.f;
#pragma unroll
    for (int k = 0; k < kNarrowPer; ++k)
        if (known && k == (int)a / G) za = z[k];
    za = __shfl_sync(0xffffffffu, za, known ? (int)a % G : 0, G);
    if (!live) return;
    T *g_row = static_cast<T *>(p.grad) + row * p.ld_grad;
    if (!work) {
        if (lane == 0) skip_row(p, row);
        if (p.grad)
            for (int v = lane; v < p.A; v += G) g_row[v] = from_float<T>(0.f);
        return;
    }
    const double lso = log(so), lsr = REF ? log(ss) : 0.0;
    const double logp = known ? ((double)za - mo) - lso : (double)NAN;
    const double kl = REF ? sd / so - (lso - lsr) : 0.0, H = lso - st / so;
    // (a row without a finite logit: log 0 everywhere, and no distribution to have a gradient)
    const RowResult f = finish_row(p, row, empty && known ? -INFINITY : logp, kl, H, empty && known, lane == 0);
    if (!p.grad) return;
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

// -------------------------------------------------------------------------------------------- long rows
struct Partial {  // of one warp or more: maxima, sums relative to them
    float c, so, st, cr, ss, sd;
};
__device__ __forceinline__ Partial shuffled(const Partial &a, int o)
{
    Partial b;
    b.c = __shfl_xor_sync(0xffffffffu, a.c, o);
    b.so = __shfl_xor_sync(0xffffffffu, a.so, o);
    b.st = __shfl_xor_sync(0xffffffffu, a.st, o);
    b.cr = __shfl_xor_sync(0xffffffffu, a.cr, o);
    b.ss = __shfl_xor_sync(0xffffffffu, a.ss, o);
    b.sd = __shfl_xor_sync(0xffffffffu, a.sd, o);
    return b;
}
// sums of `a` relative to the maxima c and cr (those of a part without any element are -inf, its sums 0)
__device__ __forceinline__ void rebase(Partial &a, float c, float cr)
{
    const float d = a.so != 0.f ? (a.c - c) * kLog2e : 0.f, dr = a.ss != 0.f ? (a.cr - cr) * kLog2e : 0.f;
    const float f = exp2f(d), fr = exp2f(dr);
    a.st = f * (a.st + d * a.so);
    a.sd = f * (a.sd + (d - dr) * a.so);
    a.so *= f;
    a.ss *= fr;
    a.c = c;
    a.cr = cr;
}
__device__ __forceinline__ Partial warp_merged(Partial a)
{
    float c = a.c, cr = a.cr;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        c = fmaxf(c, __shfl_xor_sync(0xffffffffu, c, o));
        cr = fmaxf(cr, __shfl_xor_sync(0xffffffffu, cr, o));
    }
    rebase(a, c, cr);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Partial b = shuffled(a, o);
        a.so += b.so;
        a.st += b.st;
        a.ss += b.ss;
        a.sd += b.sd;
    }
    return a;
}

constexpr int kMaxCluster = 16, kMaxWarps = 16;

// WARP: a warp per row, four rows a CTA; else the CTAs of a cluster share a row.  A thread holds NV pieces of 16 bytes
// (and as many of the reference's).
template <typename T, bool REF, int NV, bool WARP>
__global__ void __launch_bounds__(WARP ? 128 : 512) loss_rows_kernel(const __grid_constant__ LossArgs p)
{
    constexpr int V = Row<T>::kVec;
    __shared__ Partial parts[WARP ? 1 : kMaxCluster * kMaxWarps];
    namespace cg = cooperative_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int share = 1, rank = 0;  // CTAs of the row
    if constexpr (!WARP) {
        share = (int)cg::this_cluster().num_blocks();
        rank = (int)cg::this_cluster().block_rank();
        asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    }
    const long long row = WARP ? (long long)blockIdx.x * 4 + warp : (long long)(blockIdx.x / (unsigned)share);
    if (WARP && row >= p.rows) return;
    const int lanes = WARP ? 32 : (int)blockDim.x * share, first_lane = WARP ? lane : rank * (int)blockDim.x + (int)threadIdx.x;
    const float w = weight_of(p, row);
    const T *z_row = static_cast<const T *>(p.logits) + row * p.ld;
    const T *r_row = REF ? static_cast<const T *>(p.ref) + row * p.ld_ref : z_row;
    T *g_row = p.grad ? static_cast<T *>(p.grad) + row * p.ld_grad : nullptr;
    // pieces start at multiples of 16 bytes of the logits (the other arrays may lie otherwise)
    const int first = first_lane * V - phase_of(z_row), step = lanes * V;
    if (w == 0.f) {
        if (!WARP) asm volatile("barrier.cluster.wait;" ::: "memory");
        if (first_lane == 0) skip_row(p, row);
        if (g_row) {
            const float zero[V] = {};
#pragma unroll
            for (int i = 0; i < NV; ++i) store_piece<T>(g_row, first + i * step, p.A, zero);
        }
        return;
    }
    uint4 raw[NV], raw_r[REF ? NV : 1];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        raw[i] = load_piece<T, true>(z_row, first + i * step, p.A, -INFINITY);
        if constexpr (REF) raw_r[i] = load_piece<T>(r_row, first + i * step, p.A, -INFINITY);
    }
    const long long a = action_of(p, row);
    const bool known = a >= 0 && a < p.A;
    const float za = known ? to_float(z_row[a]) : NAN;

    Partial s;
    float m = -INFINITY, mr = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float z[V];
        unpack<T>(raw[i], z);
#pragma unroll
        for (int k = 0; k < V; ++k) m = fmaxf(m, z[k]);
        if constexpr (REF) {
            unpack<T>(raw_r[i], z);
#pragma unroll
            for (int k = 0; k < V; ++k) mr = fmaxf(mr, z[k]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
        if (REF) mr = fmaxf(mr, __shfl_xor_sync(0xffffffffu, mr, o));
    }
    s.c = m;
    s.cr = mr;
    {
        const float c = m == -INFINITY ? 0.f : m, cr = mr == -INFINITY ? 0.f : mr;
        s.so = s.st = s.ss = s.sd = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float z[V], zr[V];
            unpack<T>(raw[i], z);
            if constexpr (REF) unpack<T>(raw_r[i], zr);
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const float t = (z[k] - c) * kLog2e, e = exp2_fast(t);
                s.so += e;
                s.st += e != 0.f ? e * t : 0.f;
                if constexpr (REF) {
                    const float tr = (zr[k] - cr) * kLog2e;
                    s.ss += exp2_fast(tr);
                    s.sd += e != 0.f ? e * (t - tr) : 0.f;
                }
            }
        }
    }
    s = warp_merged(s);
    if constexpr (!WARP) {
        asm volatile("barrier.cluster.wait;" ::: "memory");  // every CTA of the cluster has started
        const int warps = (int)blockDim.x >> 5, total = warps * share;
        if (lane < share) *cg::this_cluster().map_shared_rank(&parts[rank * warps + warp], lane) = s;
        cg::this_cluster().sync();
        Partial mine;
        mine.c = mine.cr = -INFINITY;
        for (int i = lane; i < total; i += 32) {
            mine.c = fmaxf(mine.c, parts[i].c);
            mine.cr = fmaxf(mine.cr, parts[i].cr);
        }
        mine.so = mine.st = mine.ss = mine.sd = 0.f;
        for (int i = lane; i < total; i += 32) {
            Partial b = parts[i];
            rebase(b, mine.c, mine.cr);
            mine.so += b.so;
            mine.st += b.st;
            mine.ss += b.ss;
            mine.sd += b.sd;
        }
        s = warp_merged(mine);
    }
    const bool empty = known && s.so == 0.f;
    const float c = s.c == -INFINITY ? 0.f : s.c, cr = s.cr == -INFINITY ? 0.f : s.cr;
    const float inv = 1.f / s.so, lso = log2f(s.so), lsr = REF ? log2f(s.ss) : 0.f;
    const double kl = REF ? kLn2 * ((double)s.sd / (double)s.so - (double)log2f(s.so / s.ss)) : 0.0;
    const double H = kLn2 * ((double)lso - (double)s.st / (double)s.so);
    const double logp = empty ? (double)-INFINITY : kLn2 * ((double)((za - c) * kLog2e) - (double)lso);
    const RowResult f = finish_row(p, row, logp, kl, H, empty, first_lane == 0);
    if (!g_row) return;
    // p_v (base + kl_coef delta_v + entropy_coef lp_v) with the logarithms in base 2
    const float kk = REF ? (float)(p.kl_coef * kLn2) : 0.f, ke = (float)(p.entropy_coef * kLn2);
    const float wi = w * inv;
    const float k0 = (float)(f.base - (double)ke * lso - (kk != 0.f ? (double)kk * ((double)lso - lsr) : 0.0));
    const float at_a = (float)((double)w * f.slope);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = first + i * step;
        float z[V], zr[V], g[V];
        unpack<T>(raw[i], z);
        if constexpr (REF) unpack<T>(raw_r[i], zr);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const float t = (z[k] - c) * kLog2e, e = exp2_fast(t);
            float b = fmaf(ke, t, k0);
            if constexpr (REF) {
                if (kk != 0.f) b = fmaf(kk, t - (zr[k] - cr) * kLog2e, b);
            }
            g[k] = e != 0.f ? e * wi * b : 0.f;
        }
        if (a >= at && a < at + V) {
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (at + k == a) g[k] += at_a;
        }
        if (empty) {
#pragma unroll
            for (int k = 0; k < V; ++k) g[k] = 0.f;
        }
        store_piece<T>(g_row, at, p.A, g);
    }
}

// -------------------------------------------------------------------------------------- sums over rows
constexpr int kStatsThreads = 1024, kStatsCluster = 8, kSums = 7;

// One cluster (of one CTA or eight), double sums in a fixed order.
__global__ void __launch_bounds__(kStatsThreads)
loss_stats_kernel(const __grid_constant__ LossArgs p, float *__restrict__ stats)
{
    namespace cg = cooperative_groups;
    __shared__ double s_sum[kStatsThreads / 32][kSums];
    __shared__ float s_max[kStatsThreads / 32];
    __shared__ double c_sum[kStatsCluster][kSums];  // used in the first CTA
    __shared__ float c_max[kStatsCluster];
    asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    double sum[kSums] = {};
    float mx = -INFINITY;
    const long long stride = (long long)gridDim.x * blockDim.x;
    for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < p.rows; i += stride) {
        const double w = (double)weight_of(p, i);
        const float2 t = __ldcg(reinterpret_cast<const float2 *>(p.terms + 2 * i));
        const float kl = __ldcg(p.kl + i), H = __ldcg(p.entropy + i);
        if (w == 0.0) continue;
        const double pg = (double)t.x, r = fabs((double)t.y);
        sum[0] += w * (pg + (p.kl_coef != 0.f ? (double)p.kl_coef * kl : 0.0) - (double)p.entropy_coef * H);
        sum[1] += w * pg;
        sum[2] += w * (double)kl;
        sum[3] += w * (double)H;
        sum[4] += signbit(t.y) ? w : 0.0;
        sum[5] += w;
        sum[6] += w * r;
        mx = fmaxf(mx, kl);
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    if (lane == 0) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) s_sum[warp][j] = sum[j];
        s_max[warp] = mx;
    }
    __syncthreads();
    asm volatile("barrier.cluster.wait;" ::: "memory");  // the first CTA has started
    if (warp == 0) {
#pragma unroll
        for (int j = 0; j < kSums; ++j) sum[j] = lane < warps ? s_sum[lane][j] : 0.0;
        mx = lane < warps ? s_max[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int j = 0; j < kSums; ++j) sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], o);
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        }
        if (lane == 0) {
            const unsigned rank = cg::this_cluster().block_rank();
#pragma unroll
            for (int j = 0; j < kSums; ++j) *cg::this_cluster().map_shared_rank(&c_sum[rank][j], 0) = sum[j];
            *cg::this_cluster().map_shared_rank(&c_max[rank], 0) = mx;
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
            for (unsigned i = 0; i < gridDim.x; ++i) most = fmaxf(most, c_max[i]);
            stats[6] = most == -INFINITY ? 0.f : most;
        }
    }
}

// ---------------------------------------------------------------------------------------------- launch
template <typename T, bool REF>
cudaError_t launch_narrow(const LossArgs &p, cudaStream_t st)
{
    int g = 1;
    while (g * kNarrowPer < p.A) g *= 2;
    const long long threads = (long long)p.rows * g;
    const unsigned blocks = (unsigned)((threads + 127) / 128);
    const auto kernel = g == 1   ? loss_narrow_kernel<T, REF, 1>
                        : g == 2 ? loss_narrow_kernel<T, REF, 2>
                        : g == 4 ? loss_narrow_kernel<T, REF, 4>
                                 : loss_narrow_kernel<T, REF, 8>;
    kernel<<<blocks, 128, 0, st>>>(p);
    return cudaGetLastError();
}

template <typename T, bool REF>
cudaError_t launch_rows(const LossArgs &p, cudaStream_t st)
{
    constexpr int V = Row<T>::kVec;
    const int pieces = (p.A + V - 1 + V - 1) / V;  // a row may start up to V - 1 elements behind a multiple of 16 bytes
    if (pieces <= 32 * 8) {
        const unsigned blocks = (unsigned)(((long long)p.rows + 3) / 4);
        if (pieces <= 32 * 4) loss_rows_kernel<T, REF, 4, true><<<blocks, 128, 0, st>>>(p);
        else loss_rows_kernel<T, REF, 8, true><<<blocks, 128, 0, st>>>(p);
        return cudaGetLastError();
    }
    int threads = 128, share = 1;
    while (threads < 512 && threads * 4 < pieces) threads *= 2;
    while (share < 8 && threads * 4 * share < pieces) share *= 2;
    const bool eight = threads * 4 * share < pieces;
    if (threads * 8 * share < pieces) share *= 2;
    const auto kernel = eight ? loss_rows_kernel<T, REF, 8, false> : loss_rows_kernel<T, REF, 4, false>;
    if (share > 8) {
        const cudaError_t e = cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)share;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)((long long)p.rows * share));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace

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
    cudaStream_t st = (cudaStream_t)cuda_stream;
    ACCERL_CUDA_TRY(with_dtype(a->dtype, [&](auto v) {
        using T = decltype(v);
        if (p.A <= kNarrow) return p.ref ? launch_narrow<T, true>(p, st) : launch_narrow<T, false>(p, st);
        return p.ref ? launch_rows<T, true>(p, st) : launch_rows<T, false>(p, st);
    }));
    const unsigned ctas = p.rows <= 8192 ? 1 : kStatsCluster;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(p.rows < kStatsThreads ? (unsigned)(p.rows + 31) / 32 * 32 : kStatsThreads);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ACCERL_CUDA_TRY(cudaLaunchKernelEx(&cfg, loss_stats_kernel, p, a->stats));
    return ACCERL_OK;
}
