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
    static constexpr float kLargest = 448.0f, kMostScale = 7.595588095e+35f;   // (448 times it is just finite)
    static __device__ __forceinline__ uint32_t encode2(float a, float b)
    {
        return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    }
    static __device__ __forceinline__ uint32_t encode4(const float (&t)[4]) { return encode2(t[0], t[1]) | (encode2(t[2], t[3]) << 16); }
    // The values of the low two bytes as a pair of fp16 numbers.
    static __device__ __forceinline__ uint32_t half2_bits(uint32_t w)
    {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w), __NV_E4M3);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ void decode4(uint32_t w, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t h = half2_bits(w >> (16 * i));
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
    static __device__ __forceinline__ uint32_t encode_exact(double u) { return __nv_cvt_double_to_fp8(u, __NV_SATFINITE, __NV_E4M3); }
};

struct CodeI8 {
    static constexpr float kLargest = 127.0f, kMostScale = 2.679388389e+36f;   // (127 times it is just finite)
    static constexpr float kRound = 12582912.0f;                   // 1.5 * 2^23: its sum with t ends in the nearest integer
    static __device__ __forceinline__ uint32_t last_bytes(const float (&t)[4])
    {
        const uint32_t lo = __byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040);
        const uint32_t hi = __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040);
        return __byte_perm(lo, hi, 0x5410);
    }
    static __device__ __forceinline__ void decode4(uint32_t w, float (&f)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i)));
    }
    // The same without the conversion unit, for callers that have it busy with exponentials: code + 128 as the last byte of an fp16
    // number from 1024 on.
    static __device__ __forceinline__ void decode4_fp16(uint32_t w, float (&f)[4])
    {
        const uint32_t b = w ^ 0x80808080u, pairs[2] = {__byte_perm(b, 0x64646464u, 0x4140), __byte_perm(b, 0x64646464u, 0x4342)};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __half2 h = __hadd2(*reinterpret_cast<const __half2*>(&pairs[i]), __half2half2(__ushort_as_half(0xE480)));      // - 1152
            const float2 v = __half22float2(h);
            f[2 * i] = v.x;
            f[2 * i + 1] = v.y;
        }
    }
    static __device__ __forceinline__ uint32_t encode_exact(double u) { return static_cast<uint32_t>(__double2int_rn(u)) & 0xFFu; }
};

// The largest absolute value as an integer: ordered like the values, infinities and NaN above all others.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t abs_max(uint32_t most, float v) { return max(most, abs_bits(v)); }

// What a group's codes and scale follow from.
struct GroupScale {
    float most, factor, scale;               // factor: L / most to 2^-22, 0 where every code is 0, infinity below 2^-119
    template <typename Code>
    static __device__ __forceinline__ GroupScale of(uint32_t most_bits)
    {
        GroupScale g;
        g.most = __uint_as_float(most_bits);
        float inverse;
        asm("rcp.approx.f32 %0, %1;" : "=f"(inverse) : "f"(g.most));
        // a product with the rounded 1 / L (two units off at most), held below what L would take past the range
        const bool finite = most_bits < 0x7F800000u;
        g.scale = finite ? fminf(g.most * (1.0f / Code::kLargest), Code::kMostScale) : __uint_as_float(0x7FC00000u);
        g.factor = finite && most_bits > 0 ? Code::kLargest * inverse : 0.0f;
        return g;
    }
};

// Whether the product t = x factor is so near a border between codes that its error, 2^-22 of itself, matters.
__device__ __forceinline__ bool near_border_i8(float x, float factor)
{
    const float t = fmaf(x, factor, CodeI8::kRound);
    return fabsf(fmaf(x, factor, CodeI8::kRound - t)) > 0.49996f;  // (2^-22 of 127 is 3.0e-5)
}
__device__ __forceinline__ bool near_border_e4m3(float t)
{
    // 20 bits lie below the mantissa's three; below 2^-6 the steps are 2^-9 throughout
    if (fabsf(t) < 0.015625f) {
        const float u = fmaf(t, 512.0f, CodeI8::kRound);
        return fabsf(fmaf(t, 512.0f, CodeI8::kRound - u)) > 0.4999f;
    }
    return ((__float_as_uint(t) + 8u - 0x80000u) & 0xFFFFFu) < 16u;
}

// The codes of N values, four a word, from their products with `factor`, whichever way a value at a border goes.  (A group without a
// factor may hold infinities; its codes are cleared at the end.)  Of groups so small that the factor would be past the range, 2^100 times
// the values are coded.
template <typename Code, int N>
__device__ __forceinline__ void encode_fast(const float (&values)[N], const GroupScale& group, uint32_t (&w)[N / 4])
{
    GroupScale g = group;
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = values[i];
    if (g.factor > 1e30f) {
        constexpr float kLift = 1.267650600e+30f;
        g = GroupScale::of<Code>(abs_bits(g.most * kLift));
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] *= kLift;
    }
    const uint32_t mask = g.factor > 0.0f ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        float t[4];
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const Pair v = pair(x[4 * i + k], x[4 * i + k + 1]), by = pair(g.factor);
            const Pair u = Code::kLargest == CodeI8::kLargest ? fma2(v, by, pair(CodeI8::kRound)) : v * by;
            t[k] = u.v.x, t[k + 1] = u.v.y;
        }
        w[i] = (Code::kLargest == CodeI8::kLargest ? CodeI8::last_bytes(t) : CodeE4M3::encode4(t)) & mask;
    }
}

// The code by the definition, from the quotient in 64 bits.  Out of line: few values come here.
template <typename Code>
__device__ __noinline__ uint32_t code_of_quotient(float v, float most)
{
    return Code::encode_exact(static_cast<double>(v) * Code::kLargest / static_cast<double>(most)) & 0xFFu;
}

// The codes by the definition, for values of type T.
//
// A quotient of bf16 values, L m 2^e / n with m and n of eight bits, often lies on a border between codes (one value in a thousand is
// half of its group's largest); if not, it is at least 2^-17 of itself away (|2 L m 2^i - b n| >= 1 for a border of b, of eight bits).
// So the product with `factor`, rounded to 18 bits (by a splitting product, after Dekker), is on the border where the quotient is, and on
// its side of it elsewhere.  Quotients of fp32 values come as near as 2^-33: the few whose product is in doubt are done again.  So is
// all of a group so small that `factor` overflows, or (fp32) so large that the reciprocal in it has lost bits.
template <typename T, typename Code, int N>
__device__ __forceinline__ void encode_exactly(const float (&x)[N], const GroupScale& g, uint32_t (&w)[N / 4])
{
    constexpr bool kI8 = Code::kLargest == CodeI8::kLargest;
    const bool all = g.factor > 1e30f || (sizeof(T) == 4 && g.most > 8e37f);
    bool doubt = all;
    if constexpr (sizeof(T) == 2) {
        const uint32_t mask = g.factor > 0.0f ? 0xFFFFFFFFu : 0u;
        const Pair by = pair(g.factor), split = pair(65.0f), minus = pair(-1.0f);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            float t[4];
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
                const Pair u = pair(x[4 * i + k], x[4 * i + k + 1]) * by, far = u * split;
                Pair v = fma2(fma2(u, minus, far), minus, far);    // far - (far - u)
                if (kI8) v = v + pair(CodeI8::kRound);
                t[k] = v.v.x, t[k + 1] = v.v.y;
            }
            w[i] = (kI8 ? CodeI8::last_bytes(t) : CodeE4M3::encode4(t)) & mask;
        }
    } else {
        encode_fast<Code>(x, g, w);
        if (kI8) {
            float far = 0.0f;                                      // the largest distance from the nearest integer
            const Pair by = pair(g.factor), round = pair(CodeI8::kRound), minus = pair(-1.0f);
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const Pair v = pair(x[i], x[i + 1]), off = fma2(v, by, fma2(fma2(v, by, round), minus, round));
                far = fmaxf(far, fmaxf(fabsf(off.v.x), fabsf(off.v.y)));
            }
            doubt |= far > 0.49996f;
        } else {
            uint32_t border = 0xFFFFFFFFu, small = 0xFFFFFFFFu;    // (any value below 2^-6 that is not 0 is looked at)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t t = __float_as_uint(x[i] * g.factor);
                border = min(border, (t + 8u - 0x80000u) & 0xFFFFFu);
                small = min(small, (t & 0x7FFFFFFFu) - 1u);
            }
            doubt |= border < 16u || small < 0x3C800000u - 1u;
        }
    }
    if (doubt && g.factor > 0.0f) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (all || (kI8 ? near_border_i8(x[i], g.factor) : near_border_e4m3(x[i] * g.factor))) {
                const int shift = 8 * (i % 4);
                w[i / 4] = (w[i / 4] & ~(0xFFu << shift)) | (code_of_quotient<Code>(x[i], g.most) << shift);
            }
        }
    }
}

// The largest absolute value of a 16-byte vector, as bits of an fp32 value, and `most`.
template <typename T>
__device__ __forceinline__ uint32_t abs_max16(uint32_t most, const uint4& v)
{
    const uint32_t w[4] = {v.x & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu), v.y & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu),
                           v.z & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu), v.w & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu)};
    if constexpr (sizeof(T) == 2) {
        uint32_t a, b;
        asm("max.u16x2 %0, %1, %2;" : "=r"(a) : "r"(w[0]), "r"(w[1]));
        asm("max.u16x2 %0, %1, %2;" : "=r"(b) : "r"(w[2]), "r"(w[3]));
        asm("max.u16x2 %0, %1, %2;" : "=r"(a) : "r"(a), "r"(b));
        return max(most, max(a << 16, a & 0xFFFF0000u));
    } else {
        return max(max(max(most, w[0]), max(w[1], w[2])), w[3]);
    }
}

#endif  // __CUDACC__

}  // namespace cobalt
