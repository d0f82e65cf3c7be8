// Exchanges between the lanes of a wave and the waves of a workgroup, and an exponential.
#pragma once

#include "pictura_internal.h"

namespace pictura {

// Lanes exchange through the vector unit's own data paths (row shifts and
// broadcasts): some 60 cycles for a reduction over the wave, where six shuffles
// through LDS take ten times that.
template <int kCtrl, int kRows>
__device__ __forceinline__ uint32_t lanes(uint32_t old, uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, kCtrl, kRows, 0xf, false);
}

template <int kCtrl, int kRows>
__device__ __forceinline__ uint64_t lanes(uint64_t old, uint64_t x)
{
    return (uint64_t)lanes<kCtrl, kRows>((uint32_t)(old >> 32), (uint32_t)(x >> 32)) << 32 |
           lanes<kCtrl, kRows>((uint32_t)old, (uint32_t)x);
}

template <int kCtrl, int kRows>
__device__ __forceinline__ double lanes(double old, double x)
{
    return __longlong_as_double((long long)lanes<kCtrl, kRows>((uint64_t)__double_as_longlong(old),
                                                               (uint64_t)__double_as_longlong(x)));
}

template <int kCtrl, int kRows>
__device__ __forceinline__ float lanes(float old, float x)
{
    return __uint_as_float(lanes<kCtrl, kRows>(__float_as_uint(old), __float_as_uint(x)));
}

// x of this lane combined with those before it: within 16 lanes (L = 16), or
// over the wave (L = 64).  `none` is what lanes that do not exist hold.
template <int L, class V, class F>
__device__ __forceinline__ V lane_scan(V x, V none, F f)
{
    x = f(x, lanes<0x111, 0xf>(none, x));
    if constexpr (L > 2) x = f(x, lanes<0x112, 0xf>(none, x));
    if constexpr (L > 4) x = f(x, lanes<0x114, 0xf>(none, x));
    if constexpr (L > 8) x = f(x, lanes<0x118, 0xf>(none, x));
    if constexpr (L > 16) x = f(x, lanes<0x142, 0xa>(none, x));
    if constexpr (L > 32) x = f(x, lanes<0x143, 0xc>(none, x));
    return x;
}

__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }

__device__ __forceinline__ uint64_t from_lane(uint64_t x, int lane)
{
    return (uint64_t)from_lane((uint32_t)(x >> 32), lane) << 32 | from_lane((uint32_t)x, lane);
}

__device__ __forceinline__ double from_lane(double x, int lane)
{
    return __longlong_as_double((long long)from_lane((uint64_t)__double_as_longlong(x), lane));
}

__device__ __forceinline__ float from_lane(float x, int lane) { return __uint_as_float(from_lane(__float_as_uint(x), lane)); }

struct Add {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// Running sum over the wave's lanes, this one included; and the whole sum or maximum.
template <class V>
__device__ __forceinline__ V wave_scan(V x) { return lane_scan<64>(x, (V)0, Add{}); }

template <class V>
__device__ __forceinline__ V wave_sum(V x) { return from_lane(wave_scan(x), 63); }

__device__ __forceinline__ float wave_max(float x) { return from_lane(lane_scan<64>(x, -INFINITY, Max{}), 63); }

// Sum or maximum over a workgroup of NW waves, the same in every thread.  lds[NW]
// must not be in use by the threads before this call's barrier: two calls in a
// row take two arrays.
template <int NW, class V>
__device__ __forceinline__ V block_sum(V x, V* lds)
{
    x = wave_sum(x);
    if constexpr (NW == 1) return x;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return from_lane(lane_scan<NW>(lds[threadIdx.x & (NW - 1)], (V)0, Add{}), NW - 1);
}

template <int NW>
__device__ __forceinline__ float block_max(float x, float* lds)
{
    x = wave_max(x);
    if constexpr (NW == 1) return x;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return from_lane(lane_scan<NW>(lds[threadIdx.x & (NW - 1)], -INFINITY, Max{}), NW - 1);
}

// exp d for d <= 0.  d log2 e rounded once is off by up to 2^-24 of itself, which
// the exponential of a large |d| shows; fp32 gradients take the rest of the product
// along: that of d with a constant of two terms, the first product's rounding by an fma
// (Dekker, "A floating-point technique for extending the available precision", 1971).
constexpr float kLog2e = 1.44269502f, kLog2eRest = 1.92596299e-8f;   // log2 e is their sum

__device__ __forceinline__ float exp_of(float d)
{
    const float h = d * kLog2e;
    const float e = __builtin_amdgcn_exp2f(h);
    const float l = fmaf(d, kLog2eRest, fmaf(d, kLog2e, -h));
    return fmaf(e, l * 0.693147182f, e);
}

}  // namespace pictura
