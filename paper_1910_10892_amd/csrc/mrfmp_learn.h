// Shared by the learning operators (layer norm, bucketed pairwise function, policy loss): element types, row
// reductions, and the host side's error report.  All of them stream over rows of a matrix once; statistics and sums
// are held in 32 bits at least, whatever the type of the elements.
#pragma once

#include "../../include/mrfmp.h"
#include "mrfmp_device.h"

#include <math.h>
#include <stdio.h>

namespace mrf_host {
extern thread_local char g_error_detail[256];

inline int launch_status(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return MRF_OK;
    snprintf(g_error_detail, sizeof(g_error_detail), "%s: %s", what, hipGetErrorString(e));
    return MRF_ERR_HIP;
}

// Entries of a row at most: a lane's index may run past the row's end by what a launch takes at once (8,192 entries), and stays below 2^31.
constexpr long long LONGEST_ROW = 0x7fff0000LL;

inline bool known_type(int t) { return t == MRF_F32 || t == MRF_F16 || t == MRF_BF16; }
}  // namespace mrf_host

typedef _Float16 mrf_f16;
typedef __bf16 mrf_bf16;

template <class T> __device__ inline float mrf_to_f32(T v) { return (float)v; }
// (one rounding to nearest even, where the value is stored; everything before it is 32 bits)
template <class T> __device__ inline T mrf_from_f32(float v) { return (T)v; }

// ---- reductions over TL neighbouring lanes (a power of two up to 64), the result in every one of them.  Fixed tree.
__device__ inline float mrf_xor16_f32(float v, bool sum)
{
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto s = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    const unsigned u0 = s[0], u1 = s[1];      // (bit_cast of an element of the pair itself would take the first both times)
    const float x = __builtin_bit_cast(float, u0), y = __builtin_bit_cast(float, u1);
    return sum ? x + y : fminf(x, y);
}

__device__ inline float mrf_xor32_f32(float v, bool sum)
{
    const unsigned b = __builtin_bit_cast(unsigned, v);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const unsigned u0 = s[0], u1 = s[1];      // (bit_cast of an element of the pair itself would take the first both times)
    const float x = __builtin_bit_cast(float, u0), y = __builtin_bit_cast(float, u1);
    return sum ? x + y : fminf(x, y);
}

template <int TL> __device__ inline float mrf_lanes_sum(float v)
{
    static_assert(TL >= 1 && TL <= 64 && (TL & (TL - 1)) == 0, "lanes of a row");
    if constexpr (TL >= 2) v += mrf_dpp_f32<0xB1>(v);
    if constexpr (TL >= 4) v += mrf_dpp_f32<0x4E>(v);
    if constexpr (TL >= 8) v += mrf_dpp_f32<0x141>(v);
    if constexpr (TL >= 16) v += mrf_dpp_f32<0x140>(v);
    if constexpr (TL >= 32) v = mrf_xor16_f32(v, true);
    if constexpr (TL >= 64) v = mrf_xor32_f32(v, true);
    return v;
}

template <int TL> __device__ inline float mrf_lanes_min(float v)
{
    static_assert(TL >= 1 && TL <= 64 && (TL & (TL - 1)) == 0, "lanes of a row");
    if constexpr (TL >= 2) v = fminf(v, mrf_dpp_f32<0xB1>(v));
    if constexpr (TL >= 4) v = fminf(v, mrf_dpp_f32<0x4E>(v));
    if constexpr (TL >= 8) v = fminf(v, mrf_dpp_f32<0x141>(v));
    if constexpr (TL >= 16) v = fminf(v, mrf_dpp_f32<0x140>(v));
    if constexpr (TL >= 32) v = mrf_xor16_f32(v, false);
    if constexpr (TL >= 64) v = mrf_xor32_f32(v, false);
    return v;
}
