// What the append kernels of the paged cache share: 16-byte units of heads in fp32, sums over the lanes of a head, norm and rotation.
#pragma once
#include "tr_internal.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A 16-byte unit of a head in fp32: 8 bf16 or 4 fp32 channels.
template <int DTYPE> struct Vec;
template <> struct Vec<TR_BF16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void open(u32x4 u, float (&x)[8])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[8])
    {
        typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
        bf16x8 y;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (__bf16)x[i];
        return __builtin_bit_cast(u32x4, y);
    }
};
template <> struct Vec<TR_F32> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void open(u32x4 u, float (&x)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(u[i]);
    }
    static __device__ __forceinline__ u32x4 close(const float (&x)[4])
    {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(x[i]);
        return u;
    }
};

// Sum over LANES neighbouring lanes, within a row of 16 on the vector unit's cross-lane path.
template <int LANES> __device__ __forceinline__ float lanes_sum(float x)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32, "");
    auto bits = [&]() { return __builtin_bit_cast(int, x); };
    auto add = [&](int y) { x += __builtin_bit_cast(float, y); };
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0xB1, 0xf, 0xf, false));                   // quad_perm [1,0,3,2]
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x4E, 0xf, 0xf, false));                   // quad_perm [2,3,0,1]
    add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x141, 0xf, 0xf, false));                  // row_half_mirror
    if (LANES >= 16) add(__builtin_amdgcn_update_dpp(bits(), bits(), 0x140, 0xf, 0xf, false)); // row_mirror
    if (LANES == 32) x += __shfl_xor(x, 16);
    return x;
}

// The value of the lane half a head away, where the whole head turns.
template <int LANES> __device__ __forceinline__ float other_half(float x)
{
    const int b = __builtin_bit_cast(int, x);
    if constexpr (LANES == 16) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, 0x128, 0xf, 0xf, false)); // row_ror 8
    else if constexpr (LANES == 8) { // of eight lanes, and of each four: the mirror of the mirror
        const int m = __builtin_amdgcn_update_dpp(b, b, 0x141, 0xf, 0xf, false);
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(m, m, 0x1B, 0xf, 0xf, false));
    } else return __shfl_xor(x, LANES / 2);
}

} // namespace
