// Rows held in 8 bits: one-byte codes with one fp32 scale for a group of columns (128 of them, or the row).
//
//   scale = most / L, most the group's largest absolute value, L the largest code (448 for e4m3, 127 for int8)
//   code  = the one nearest to L x / most, halves to even        value = code * scale
//
// A group of zeros has scale 0; one that holds a NaN or an infinity has scale NaN and codes 0, so that its values read back
// as NaN.  int8 spends its codes evenly up to the group's largest value (an error of at most scale / 2), e4m3 keeps four
// significant bits of every value and is what the tensor cores take.
#pragma once

#include <cuda_fp8.h>

#include "numeric.cuh"

namespace cobalt {

constexpr int kPackGroup = 128;              // columns of a group that is not the whole row

#ifdef __CUDACC__

struct CodeE4M3 {
    static constexpr float kLargest = 448.0f;
    static __device__ __forceinline__ uint32_t encode2(float a, float b)
    {
        return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    }
    static __device__ __forceinline__ uint32_t encode4(const float (&t)[4]) { return encode2(t[0], t[1]) | (encode2(t[2], t[3]) << 16); }
    static __device__ __forceinline__ void decode4(uint32_t w, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * i)), __NV_E4M3);
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
    // Whether t, good to two units, may be on the other side of a border between codes (20 bits below the three of the
    // mantissa; below 2^-6 the steps no longer go by the exponent).
    static __device__ __forceinline__ bool near_border(float t)
    {
        return ((__float_as_uint(t) + 16u - 0x80000u) & 0xFFFFFu) < 32u || (fabsf(t) < 0.015625f && t != 0.0f);
    }
    static __device__ __forceinline__ uint32_t encode_exact(double u) { return __nv_cvt_double_to_fp8(u, __NV_SATFINITE, __NV_E4M3); }
};

struct CodeI8 {
    static constexpr float kLargest = 127.0f;
    static constexpr float kRound = 12582912.0f;                   // 1.5 * 2^23: its sum with t ends in the nearest integer
    static __device__ __forceinline__ uint32_t encode4(const float (&t)[4])
    {
        const uint32_t lo = __byte_perm(__float_as_uint(t[0] + kRound), __float_as_uint(t[1] + kRound), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(t[2] + kRound), __float_as_uint(t[3] + kRound), 0x0040);
        return __byte_perm(lo, hi, 0x5410);
    }
    static __device__ __forceinline__ void decode4(uint32_t w, float (&f)[4])
    {
        const uint32_t b = w ^ 0x80808080u;                        // code + 128 as the last byte of 2^23
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(b, 0x4B000000u, 0x7440u | i)) - 8388736.0f;
    }
    static __device__ __forceinline__ bool near_border(float t)
    {
        return fabsf(fabsf(t - ((t + kRound) - kRound)) - 0.5f) < 1e-4f;
    }
    static __device__ __forceinline__ uint32_t encode_exact(double u) { return static_cast<uint32_t>(__double2int_rn(u)) & 0xFFu; }
};

// The largest absolute value as an integer: ordered like the values, infinities and NaN above all others.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t abs_max(uint32_t most, float v) { return max(most, abs_bits(v)); }

// What a group's codes and scale follow from.
struct GroupScale {
    float most, factor, scale;               // factor: L / most, 0 where every code is 0
    template <typename Code>
    static __device__ __forceinline__ GroupScale of(uint32_t most_bits)
    {
        GroupScale g;
        g.most = __uint_as_float(most_bits);
        const bool finite = most_bits < 0x7F800000u;
        // (rounded down at the end of the range, where L times a scale rounded up would be infinite)
        g.scale = !finite ? __uint_as_float(0x7FC00000u) : g.most > 3e38f ? __fdiv_rz(g.most, Code::kLargest) : g.most / Code::kLargest;
        g.factor = finite && most_bits > 0 ? Code::kLargest / g.most : 0.0f;
        return g;
    }
};

// Four codes.  The product with `factor` is good to two units, so the few values that it leaves near a border (and all of a
// group so small that `factor` overflows) are done again from the quotient itself in 64 bits; 16-bit values do lie on borders.
template <typename Code>
__device__ __forceinline__ uint32_t encode_group4(const float (&x)[4], const GroupScale& g)
{
    float t[4];
    bool redo = g.factor > 1e30f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        t[i] = g.factor > 0.0f ? x[i] * g.factor : 0.0f;           // (a group without a scale may hold infinities)
        redo |= Code::near_border(t[i]);
    }
    uint32_t codes = Code::encode4(t);
    if (redo) {
        codes = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (g.factor > 0.0f)
                codes |= (Code::encode_exact(static_cast<double>(x[i]) * Code::kLargest / static_cast<double>(g.most)) & 0xFFu) << (8 * i);
    }
    return codes;
}

#endif  // __CUDACC__

}  // namespace cobalt
