// What the Learner's operators share: element types, 16-byte pieces of rows, argument checks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"

namespace accerl {

// rows of the products: tiles past the last row are counted in an int
constexpr int kMostRows = INT32_MAX - 65535;

inline int dtype_size(int dtype) { return dtype == ACCERL_F32 ? 4 : 2; }
inline bool good_dtype(int dtype) { return dtype == ACCERL_F32 || dtype == ACCERL_BF16 || dtype == ACCERL_F16; }

// Calls f with a value of the element type that `dtype` names.
template <typename F>
inline auto with_dtype(int dtype, F &&f)
{
    if (dtype == ACCERL_BF16) return f(__nv_bfloat16());
    if (dtype == ACCERL_F16) return f(__half());
    return f(float());
}

// status words of the bounded waits of the Learner's files on the current device; reading clears them
cudaError_t policy_loss_status(int *out);
cudaError_t linear_status(int *out);
cudaError_t weight_grad_status(int *out);

// 16 bytes of a row: kVec elements
template <typename T>
struct Row {
    static constexpr int kVec = 16 / (int)sizeof(T);
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// two elements of a 32-bit word (one for float: `b` is not written)
__device__ __forceinline__ void unpack_word(uint32_t w, float *v, const float *) { v[0] = __uint_as_float(w); }
__device__ __forceinline__ void unpack_word(uint32_t w, float *v, const __nv_bfloat16 *)
{
    v[0] = __uint_as_float(w << 16);
    v[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack_word(uint32_t w, float *v, const __half *)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    v[0] = f.x;
    v[1] = f.y;
}
__device__ __forceinline__ uint32_t pack_word(const float *v, const float *) { return __float_as_uint(v[0]); }
__device__ __forceinline__ uint32_t pack_word(const float *v, const __nv_bfloat16 *)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ uint32_t pack_word(const float *v, const __half *)
{
    const __half2 h = __floats2half2_rn(v[0], v[1]);
    return *reinterpret_cast<const uint32_t *>(&h);
}

template <typename T>
__device__ __forceinline__ void unpack(const uint4 &raw, float (&v)[Row<T>::kVec])
{
    constexpr int E = Row<T>::kVec / 4;
    unpack_word(raw.x, v, (const T *)nullptr);
    unpack_word(raw.y, v + E, (const T *)nullptr);
    unpack_word(raw.z, v + 2 * E, (const T *)nullptr);
    unpack_word(raw.w, v + 3 * E, (const T *)nullptr);
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float (&v)[Row<T>::kVec])
{
    constexpr int E = Row<T>::kVec / 4;
    return make_uint4(pack_word(v, (const T *)nullptr), pack_word(v + E, (const T *)nullptr),
                      pack_word(v + 2 * E, (const T *)nullptr), pack_word(v + 3 * E, (const T *)nullptr));
}

// 16 bytes at any multiple of the element's size.  Off a multiple of 16 they go by 32-bit words, off a multiple of 4 (the
// 16-bit types only) with the halves put together from neighbouring words: a warp's accesses then touch the same lines
// four or five times, which L1 serves at about the rate of HBM; element by element it would be eight times.  (A word is
// read whole where one of its halves is wanted: it lies in the same 4 bytes of the same allocation.)
__device__ __forceinline__ uint4 load16(const void *p)
{
    const uintptr_t a = (uintptr_t)p;
    if ((a & 15) == 0) return __ldcs(static_cast<const uint4 *>(p));
    const uint32_t *w = reinterpret_cast<const uint32_t *>(a & ~(uintptr_t)3);
    uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
    if (a & 2) {
        v.x = __funnelshift_r(v.x, v.y, 16);
        v.y = __funnelshift_r(v.y, v.z, 16);
        v.z = __funnelshift_r(v.z, v.w, 16);
        v.w = __funnelshift_r(v.w, w[4], 16);
    }
    return v;
}
__device__ __forceinline__ void store16(void *p, const uint4 &v)
{
    const uintptr_t a = (uintptr_t)p;
    if ((a & 15) == 0) {
        *static_cast<uint4 *>(p) = v;
        return;
    }
    if (a & 2) {
        *static_cast<uint16_t *>(p) = (uint16_t)v.x;
        uint32_t *w = reinterpret_cast<uint32_t *>(a + 2);
        w[0] = __funnelshift_r(v.x, v.y, 16);
        w[1] = __funnelshift_r(v.y, v.z, 16);
        w[2] = __funnelshift_r(v.z, v.w, 16);
        *reinterpret_cast<uint16_t *>(a + 14) = (uint16_t)(v.w >> 16);
        return;
    }
    uint32_t *w = static_cast<uint32_t *>(p);
    w[0] = v.x;
    w[1] = v.y;
    w[2] = v.z;
    w[3] = v.w;
}

// Elements first .. first + kVec of a row of n, those outside it `fill`.  ALIGNED: the address of element `first` is a
// multiple of 16 bytes.
template <typename T, bool ALIGNED = false>
__device__ __forceinline__ uint4 load_piece(const T *row, int first, int n, float fill)
{
    constexpr int V = Row<T>::kVec;
    if (first >= 0 && first + V <= n)
        return ALIGNED ? __ldcs(reinterpret_cast<const uint4 *>(row + first)) : load16(row + first);
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = first + k >= 0 && first + k < n ? to_float(row[first + k]) : fill;
    return pack<T>(v);
}
template <typename T, bool ALIGNED = false>
__device__ __forceinline__ void store_piece(T *row, int first, int n, const float (&v)[Row<T>::kVec])
{
    constexpr int V = Row<T>::kVec;
    if (first >= 0 && first + V <= n) {
        if (ALIGNED) *reinterpret_cast<uint4 *>(row + first) = pack<T>(v);
        else store16(row + first, pack<T>(v));
        return;
    }
#pragma unroll
    for (int k = 0; k < V; ++k)
        if (first + k >= 0 && first + k < n) row[first + k] = from_float<T>(v[k]);
}

// do all rows of an array start at multiples of 16 bytes?
inline bool rows_aligned(const void *p, long long ld, int dtype) { return !(((uintptr_t)p | (uintptr_t)(ld * dtype_size(dtype))) & 15); }

// elements of type T by which an address lies behind a multiple of 16 bytes
template <typename T>
__device__ __forceinline__ int phase_of(const T *p)
{
    return (int)(((uintptr_t)p & 15) / sizeof(T));
}

}  // namespace accerl
