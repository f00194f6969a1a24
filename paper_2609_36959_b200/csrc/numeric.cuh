// Element types of the dense operators (layer norm, gate, dropout, expert feed-forward): 16-byte vectors of
// bf16 or fp32 values, unpacked to fp32 registers.
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace cobalt {

#ifdef __CUDACC__

template <typename T>
struct Vec16;

template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int kElems = 8;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[8])
    {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&p);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <>
struct Vec16<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};

// Two fp32 values in a register pair: sm_100 adds, multiplies and fuses both with one instruction (PTX .f32x2).
struct Pair {
    float2 v;
};

__device__ __forceinline__ Pair pair(float a, float b) { return Pair{make_float2(a, b)}; }
__device__ __forceinline__ Pair pair(float a) { return Pair{make_float2(a, a)}; }
__device__ __forceinline__ uint64_t pair_bits(const Pair& p)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(p.v.x), "f"(p.v.y));
    return r;
}
__device__ __forceinline__ Pair bits_pair(uint64_t b)
{
    Pair r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.v.x), "=f"(r.v.y) : "l"(b));
    return r;
}
__device__ __forceinline__ Pair operator+(const Pair& a, const Pair& b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return bits_pair(r);
}
__device__ __forceinline__ Pair operator*(const Pair& a, const Pair& b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)));
    return bits_pair(r);
}
__device__ __forceinline__ Pair fma2(const Pair& a, const Pair& b, const Pair& c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(pair_bits(a)), "l"(pair_bits(b)), "l"(pair_bits(c)));
    return bits_pair(r);
}

// A 16-byte vector as pairs of neighbouring values.
template <typename T>
__device__ __forceinline__ void unpack_pairs(const uint4& v, Pair (&f)[Vec16<T>::kElems / 2])
{
    float e[Vec16<T>::kElems];
    Vec16<T>::unpack(v, e);
#pragma unroll
    for (int i = 0; i < Vec16<T>::kElems / 2; ++i) f[i] = pair(e[2 * i], e[2 * i + 1]);
}

template <typename T>
__device__ __forceinline__ uint4 pack_pairs(const Pair (&f)[Vec16<T>::kElems / 2])
{
    float e[Vec16<T>::kElems];
#pragma unroll
    for (int i = 0; i < Vec16<T>::kElems / 2; ++i) {
        e[2 * i] = f[i].v.x;
        e[2 * i + 1] = f[i].v.y;
    }
    return Vec16<T>::pack(e);
}

// A 16-byte load of data that the same thread may overwrite later (in-place calls): like ld_stream16 without the
// read-only path, and kept in program order with st_stream16.
__device__ __forceinline__ uint4 ld_once16(const void* p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
    return v;
}

#endif  // __CUDACC__

}  // namespace cobalt
