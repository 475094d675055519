// Blocks of activations in 8 bits, as the kernels read and write them (sdnn_pack.hip writes and restores them, the backward pass of
// the layer norm reads them as they are).
//
// The values of a block [n][B], in its order, in groups of 128; a group has one scale t, a float of 8 significant bits (a bf16),
// the smallest with  most t >= the group's largest value.  A value is stored as the nearest multiple of t, halves away from zero:
//   cap == 0  both signs; most = 127: code c stands for c t, -128 for what is not finite
//   cap > 0   0 <= x <= cap; most = 253: code 0 for 0, 255 for cap, 254 for NaN, and 1 .. 253 for 0 < x < cap (no such value becomes
//             0, none becomes cap: the derivative of the clamped ReLU is exact)
// c t is exact in fp32 (8 bits times 8 bits), and finite: for the largest floats t is 2^121 (1 + 2/128) at most, of which they are 126.03 (cap: 2^120
// times that, 252.1), so that the codes whose products would be infinite are not reached.  A value is off by at most t / 2, one below t / 2 with a cap by less
// than t; t / 2 is 0.4 % (cap: 0.2 %) of the group's largest value, and where t is subnormal (a largest value below 2^-119; cap: 2^-118) up to 2^-134 more.
#pragma once
#include <cfloat>
#include <cstdint>
#include <hip/hip_runtime.h>

#include "sdnn_internal.h"

#define PACK_GROUP 128

static inline int64_t pack8_groups(int64_t count) { return (count + PACK_GROUP - 1) / PACK_GROUP; }
static inline int64_t pack8_bytes(int64_t count) { return ((PACK_GROUP + 2) * pack8_groups(count) + 255) & ~(int64_t)255; }

// The largest value that a group's scale is made for, of those that become multiples of it.
template <bool SIGNED> __device__ __forceinline__ float pack8_size(float x, float cap)
{
    if constexpr (SIGNED) return fabsf(x) <= FLT_MAX ? fabsf(x) : 0.0f;
    return x < cap ? x : 0.0f; // (below zero: less than any largest value; NaN: not less than the cap)
}
// The scale of a group whose largest value is `largest`, as the 16 bits that are stored.
template <bool SIGNED> __device__ __forceinline__ unsigned pack8_scale(float largest)
{
    constexpr float most = SIGNED ? 127.0f : 253.0f;
    unsigned t = __float_as_uint(largest * (1.0f / most)) >> 16; // that, or one or two more: the product and cutting off lose
#pragma unroll
    for (int k = 0; k < 2; ++k) t += most * __uint_as_float(t << 16) < largest ? 1u : 0u; // (exact: eight bits times eight)
    return t;
}
// What values are multiplied by before they are rounded: 1 / t, and 2^-30 of it more.  The fp32 value next to a half of t is 2^-24 of
// it away, so that the halves, which the product may miss by its rounding, are lifted over the border, and nothing else is.
__device__ __forceinline__ double pack8_inverse(unsigned t)
{
    const double d = (double)__uint_as_float(t << 16), r = __builtin_amdgcn_rcp(d); // to 2^-20 and better; one step of Newton's: 2^-40
    return t ? fma(r, fma(-d, r, 1.0) + 0x1p-30, r) : 0.0;
}
template <bool SIGNED> __device__ __forceinline__ unsigned pack8_code(float x, float cap, double inverse)
{
    if constexpr (SIGNED) {
        const int c = (int)fma((double)fabsf(x), inverse, 0.5);
        return fabsf(x) <= FLT_MAX ? (unsigned)(x < 0.0f ? -c : c) & 255u : 128u;
    }
    unsigned c = (unsigned)max((int)fma((double)x, inverse, 0.5), 1);
    c = x > 0.0f ? c : x != x ? 254u : 0u;
    return x >= cap ? 255u : c;
}
// below: the largest float below cap
template <bool SIGNED> __device__ __forceinline__ float pack8_value_of(unsigned code, float scale, float cap, float below)
{
    if constexpr (SIGNED) return code == 128u ? __builtin_nanf("") : (float)(int)(signed char)code * scale;
    float v = fminf((float)code * scale, below);
    v = code == 254u ? __builtin_nanf("") : v;
    return code == 255u ? cap : v;
}

// ---- host side, shared by the operators on single blocks ----------------------------------------------------------------
template <class... A> static inline int sdnn_fail(int code, const char *fmt, A... a)
{
    sdnn_set_global_error(fmt, a...);
    return code;
}
static inline int sdnn_launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SDNN_OK : sdnn_fail(SDNN_EHIP, "launch: %s", hipGetErrorString(e));
}
// d_packed of a call; sdnn_pack.hip
int sdnn_check_pack8(const void *d_packed, size_t packed_bytes, int32_t n, int32_t B, float cap);
