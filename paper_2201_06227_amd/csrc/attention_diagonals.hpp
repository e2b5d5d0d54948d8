// The gradient of a bias by distance from blocks of score gradients.
#pragma once
#include "attention.hpp"

namespace egeria {

// The bf16 products round towards minus infinity on the average, by 1e-9 of operands of size one, which a table's gradient, a long sum
// of p (dP - delta) that cancels, would gather.  So every other row or column of dP is made with the opposite sign: `turned` is its operand,
// `sign_of` what the product is taken by.
template <typename F>
__device__ __forceinline__ F turned(F f, int index)
{
    if constexpr (sizeof(F) == 16) return __builtin_bit_cast(F, __builtin_bit_cast(v4u, f) ^ v4u((index & 1) ? 0x80008000u : 0u));
    else return f;                                                          // fp32: exact halves are as often up as down
}
template <typename F>
__device__ __forceinline__ float sign_of(int index) { return sizeof(F) == 16 && (index & 1) ? -1.0f : 1.0f; }

// Base-2 log-sum-exp of a row less a whole number, which the caller gives back as a power of two: exponents s c - L are rounded to the
// precision of their own size, and that is log2 of the keys where scores are of size one.  (The product is exact inside the fma; the rest
// is that of log2 e.)  Beyond kFine that rest is less than the result's own rounding: the plain product, as the dk / dv kernel has it.
constexpr float kFine = 65536.0f;
__device__ __forceinline__ float lowered(float lse, float whole)
{
    return fabsf(lse) > kFine ? lse * kLog2e - whole : fmaf(lse, 1.92596303e-8f, fmaf(lse, kLog2e, -whole));
}

__device__ __forceinline__ float sum16(const v16f &s)
{
    return (((s[0] + s[1]) + (s[2] + s[3])) + ((s[4] + s[5]) + (s[6] + s[7]))) + (((s[8] + s[9]) + (s[10] + s[11])) + ((s[12] + s[13]) + (s[14] + s[15])));
}

// Adds a block of dS to sums by distance: into[d] for d = key - query of the block.  SIGN 1: dS^T (keys down, queries across); -1: dS.
// (In terms of the former:) A value in lane l of a row of 16 lanes and register r has distance u - l, u being the register's key modulo 16, up to multiples of
// 16 and of the half's 4 that all lanes of the row share.  Moved down by u lanes, values of one distance lie in one lane, those
// that leave the row at the bottom come in at the top 16 distances further: two additions with a shift of lanes each, no LDS.  What
// is left are the sums of 4 times 16 distances for each half of the wave, which has a table of its own: plain additions, in a
// fixed order.  (As additions of all 1024 values in LDS, atomic ones that never collide, dq of 64 x 256 x 12 x 64 took 188 us instead
// of 55.)
template <int R>
__device__ __forceinline__ void shift_add(const v16f &s, float (&a)[3])
{
    constexpr int key = 8 * (R >> 2) + (R & 3), u = key & 15, w = key >> 4;
    const int x = __float_as_int(s[R]);
    if constexpr (u == 0) a[w] += s[R];
    else {
        a[w] += __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x100 | u, 0xf, 0xf, true));                // lane i takes from i + u
        a[w + 1] += __int_as_float(__builtin_amdgcn_update_dpp(0, x, 0x110 | (16 - u), 0xf, 0xf, true));     // from i - (16 - u)
    }
    if constexpr (R < 15) shift_add<R + 1>(s, a);
}
template <int SIGN>
__device__ __forceinline__ void add_diagonals(const v16f &s, float *into, int lane)
{
    float a[3] = {0.0f, 0.0f, 0.0f};
    shift_add<0>(s, a);
    // a[v] of lane l: distance 16 v + 4 half - 16 (row of lanes in the half) - l % 16
    const float up1 = lane_xor<16>(a[1]), up2 = lane_xor<16>(a[2]);
    const bool low = !(lane & 16);
    float *at = into + SIGN * (4 * (lane >> 5) - (lane & 15));
    const float x = low ? a[0] + up1 : a[0], y = a[1] + up2, z = a[2];
    at[low ? 0 : SIGN * -16] += x;
    if (low) {
        at[SIGN * 16] += y;
        at[SIGN * 32] += z;
    }
    wave_lds_turn();                                                        // the next block's lanes add where others of this one have
}

}  // namespace egeria
