// Arithmetic on the four element types, shared by the kernels that compute (the codec's own only move bits):
// Num<DT>::Elem is what lies in memory, Num<DT>::Acc what sums are held in (binary32; binary64 for BT_F64),
// widening is exact, narrowing rounds once to nearest even.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "bt_internal.cuh"

namespace bt {

template <int DT>
struct Num;
template <>
struct Num<BT_F32> {
    using Elem = float;
    using Acc  = float;
    __device__ static __forceinline__ float widen(float v) { return v; }
    __device__ static __forceinline__ float narrow(float v) { return v; }
};
template <>
struct Num<BT_F64> {
    using Elem = double;
    using Acc  = double;
    __device__ static __forceinline__ double widen(double v) { return v; }
    __device__ static __forceinline__ double narrow(double v) { return v; }
};
template <>
struct Num<BT_F16> {
    using Elem = __half;
    using Acc  = float;
    __device__ static __forceinline__ float  widen(__half v) { return __half2float(v); }
    __device__ static __forceinline__ __half narrow(float v) { return __float2half_rn(v); }
};
template <>
struct Num<BT_BF16> {
    using Elem = __nv_bfloat16;
    using Acc  = float;
    __device__ static __forceinline__ float         widen(__nv_bfloat16 v) { return __bfloat162float(v); }
    __device__ static __forceinline__ __nv_bfloat16 narrow(float v) { return __float2bfloat16_rn(v); }
};

// a 16-byte vector's elements, widened; and back
template <int DT>
constexpr int kLanes = 16 / static_cast<int>(sizeof(typename Num<DT>::Elem));

template <int DT>
__device__ __forceinline__ void widen_vec(const uint4 &w, typename Num<DT>::Acc (&v)[kLanes<DT>])
{
    if constexpr (DT == BT_BF16) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k]     = __uint_as_float(u[k] << 16);
            v[2 * k + 1] = __uint_as_float(u[k] & 0xFFFF0000u);
        }
    } else if constexpr (DT == BT_F16) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&u[k]));
            v[2 * k]       = f.x;
            v[2 * k + 1]   = f.y;
        }
    } else if constexpr (DT == BT_F32) {
        v[0] = __uint_as_float(w.x), v[1] = __uint_as_float(w.y), v[2] = __uint_as_float(w.z), v[3] = __uint_as_float(w.w);
    } else {
        v[0] = __hiloint2double(static_cast<int>(w.y), static_cast<int>(w.x));
        v[1] = __hiloint2double(static_cast<int>(w.w), static_cast<int>(w.z));
    }
}

template <int DT>
__device__ __forceinline__ uint4 narrow_vec(const typename Num<DT>::Acc (&v)[kLanes<DT>])
{
    uint4 w;
    if constexpr (DT == BT_BF16 || DT == BT_F16) {
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (DT == BT_BF16) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
                u[k]                   = *reinterpret_cast<const uint32_t *>(&p);
            } else {
                const __half2 p = __floats2half2_rn(v[2 * k], v[2 * k + 1]);
                u[k]            = *reinterpret_cast<const uint32_t *>(&p);
            }
        }
        w = make_uint4(u[0], u[1], u[2], u[3]);
    } else if constexpr (DT == BT_F32) {
        w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    } else {
        w = make_uint4(static_cast<uint32_t>(__double2loint(v[0])), static_cast<uint32_t>(__double2hiint(v[0])),
                       static_cast<uint32_t>(__double2loint(v[1])), static_cast<uint32_t>(__double2hiint(v[1])));
    }
    return w;
}

// Two sums side by side.  Binary32: a register pair, whose operations the architecture performs two at a time.
template <typename A>
struct Two {
    A lo, hi;
    __device__ static __forceinline__ Two of(A lo, A hi) { return Two{lo, hi}; }
    __device__ __forceinline__ A low() const { return lo; }
    __device__ __forceinline__ A high() const { return hi; }
};
template <>
struct Two<float> {
    uint64_t v;
    __device__ static __forceinline__ Two of(float lo, float hi)
    {
        Two r;
        asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
        return r;
    }
    __device__ __forceinline__ float low() const
    {
        return __uint_as_float(static_cast<uint32_t>(v));
    }
    __device__ __forceinline__ float high() const
    {
        return __uint_as_float(static_cast<uint32_t>(v >> 32));
    }
};
template <typename A>
__device__ __forceinline__ Two<A> both(A v) { return Two<A>::of(v, v); }
__device__ __forceinline__ Two<float> operator*(Two<float> a, Two<float> b)
{
    Two<float> r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Two<double> operator*(Two<double> a, Two<double> b) { return {a.lo * b.lo, a.hi * b.hi}; }
// a b + c
__device__ __forceinline__ Two<float> fma2(Two<float> a, Two<float> b, Two<float> c)
{
    Two<float> r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}
__device__ __forceinline__ Two<double> fma2(Two<double> a, Two<double> b, Two<double> c) { return {fma(a.lo, b.lo, c.lo), fma(a.hi, b.hi, c.hi)}; }

// a 16-byte vector's elements, widened two by two; and back
template <int DT>
constexpr int kPairs = kLanes<DT> / 2;
template <int DT>
__device__ __forceinline__ void widen_pairs(const uint4 &w, Two<typename Num<DT>::Acc> (&v)[kPairs<DT>])
{
    typename Num<DT>::Acc e[kLanes<DT>];
    widen_vec<DT>(w, e);
#pragma unroll
    for (int k = 0; k < kPairs<DT>; ++k) v[k] = Two<typename Num<DT>::Acc>::of(e[2 * k], e[2 * k + 1]);
}
template <int DT>
__device__ __forceinline__ uint4 narrow_pairs(const Two<typename Num<DT>::Acc> (&v)[kPairs<DT>])
{
    typename Num<DT>::Acc e[kLanes<DT>];
#pragma unroll
    for (int k = 0; k < kPairs<DT>; ++k) e[2 * k] = v[k].low(), e[2 * k + 1] = v[k].high();
    return narrow_vec<DT>(e);
}

template <typename A>
__device__ __forceinline__ A warp_sum(A v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// ---- what the argument checks of the calls use
inline int      element_size(int dtype) { return dtype == BT_F64 ? 8 : dtype == BT_F32 ? 4 : (dtype == BT_F16 || dtype == BT_BF16) ? 2 : 0; }
inline bool     on_boundary(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
__host__ __device__ inline uint64_t round_up_div(uint64_t a, uint64_t b) { return a / b + (a % b != 0); }

// the SMs of the current device (0 if the runtime refuses to say)
inline int sm_count()
{
    int device = 0, sms = 0;
    if (reported(cudaGetDevice(&device)) != cudaSuccess) return 0;
    if (reported(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) return 0;
    return sms;
}

}  // namespace bt
