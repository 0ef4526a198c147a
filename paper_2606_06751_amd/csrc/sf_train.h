// sf_train.h -- element types and small device helpers shared by the kernels
// of stagefrontier_train.h.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "stagefrontier_train.h"

namespace sfk {

template <int DT>
struct Elem;
template <>
struct Elem<SF_F32> {
    typedef float T;
};
template <>
struct Elem<SF_BF16> {
    typedef __bf16 T;
};
template <>
struct Elem<SF_F16> {
    typedef _Float16 T;
};

// Elements of 16 bytes, and such a vector at element alignment (gfx950 loads
// and stores 16 bytes at any address).
template <int DT>
constexpr int kVec = 16 / (int)sizeof(typename Elem<DT>::T);
template <int DT>
using VecU = typename Elem<DT>::T __attribute__((ext_vector_type(kVec<DT>), aligned(sizeof(typename Elem<DT>::T))));
template <int DT>
using VecF = float __attribute__((ext_vector_type(kVec<DT>)));

// The same in global memory, for addresses that reach a kernel as numbers.
template <int DT>
using GlobalVec = __attribute__((address_space(1))) VecU<DT>;
template <int DT>
using GlobalElem = __attribute__((address_space(1))) typename Elem<DT>::T;

static inline int elem_size(int dtype) { return dtype == SF_F32 ? 4 : 2; }

// Elements from p up to the next ALIGN-byte boundary, at most n.
template <int DT, int ALIGN>
__device__ __forceinline__ int64_t head_elems(const void* p, int64_t n)
{
    const int64_t h = (int64_t)((0 - (uintptr_t)p) & (ALIGN - 1)) / (int64_t)sizeof(typename Elem<DT>::T);
    return h < n ? h : n;
}

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.92596299112661746887e-8f;  // log2 e - kLog2e
constexpr double kLog2eD = 1.44269504088896340736;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLn2Low = -1.90465429995776804525e-9f;  // ln 2 - kLn2
constexpr float kF32Max = 3.402823466e38f;

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// One DPP move; lanes outside ROW_MASK get `old`.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_f32(float old, float v)
{
    return __int_as_float(
        __builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(v), CTRL, ROW_MASK, 0xF, false));
}
__device__ __forceinline__ float last_lane(float v)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sum and maximum over a wave, wave-uniform: within rows of 16 lanes by
// exchanges that pair each lane with one of the other half, then row by row
// into the last lane.
__device__ __forceinline__ float wave_sum_f32(float v)
{
    v += dpp_f32<0xB1, 0xF>(0.0f, v);   // quad_perm [1,0,3,2]
    v += dpp_f32<0x4E, 0xF>(0.0f, v);   // quad_perm [2,3,0,1]
    v += dpp_f32<0x141, 0xF>(0.0f, v);  // row_half_mirror
    v += dpp_f32<0x140, 0xF>(0.0f, v);  // row_mirror
    v += dpp_f32<0x142, 0xA>(0.0f, v);  // row_bcast:15 -> rows 1, 3
    v += dpp_f32<0x143, 0xC>(0.0f, v);  // row_bcast:31 -> rows 2, 3
    return last_lane(v);
}
__device__ __forceinline__ float wave_max_f32(float v)
{
    v = fmaxf(v, dpp_f32<0xB1, 0xF>(v, v));
    v = fmaxf(v, dpp_f32<0x4E, 0xF>(v, v));
    v = fmaxf(v, dpp_f32<0x141, 0xF>(v, v));
    v = fmaxf(v, dpp_f32<0x140, 0xF>(v, v));
    v = fmaxf(v, dpp_f32<0x142, 0xA>(v, v));
    v = fmaxf(v, dpp_f32<0x143, 0xC>(v, v));
    return last_lane(v);
}

// Sums of 64-bit values over a wave, wave-uniform, by the same moves of their
// halves: short code, which a kernel of a few microseconds waits for.
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ uint64_t dpp_u64(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROW_MASK, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROW_MASK, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t last_lane_u64(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), 63);
    return (uint64_t)hi << 32 | lo;
}
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ double dpp_f64(double v)
{
    return __longlong_as_double((long long)dpp_u64<CTRL, ROW_MASK>((uint64_t)__double_as_longlong(v)));
}
__device__ __forceinline__ double wave_sum_f64(double v)
{
    v += dpp_f64<0xB1, 0xF>(v);
    v += dpp_f64<0x4E, 0xF>(v);
    v += dpp_f64<0x141, 0xF>(v);
    v += dpp_f64<0x140, 0xF>(v);
    v += dpp_f64<0x142, 0xA>(v);
    v += dpp_f64<0x143, 0xC>(v);
    return __longlong_as_double((long long)last_lane_u64((uint64_t)__double_as_longlong(v)));
}
__device__ __forceinline__ int64_t wave_sum_i64(int64_t x)
{
    uint64_t v = (uint64_t)x;
    v += dpp_u64<0xB1, 0xF>(v);
    v += dpp_u64<0x4E, 0xF>(v);
    v += dpp_u64<0x141, 0xF>(v);
    v += dpp_u64<0x140, 0xF>(v);
    v += dpp_u64<0x142, 0xA>(v);
    v += dpp_u64<0x143, 0xC>(v);
    return (int64_t)last_lane_u64(v);
}

}  // namespace sfk
