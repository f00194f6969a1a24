// Dropout from a counter-based generator, added to the residual stream, and its backward pass.
//
//   out[i] = residual[i] + keep(i) ? x[i] * scale : 0        grad_x[i] = keep(i) ? grad_out[i] * scale : 0
//
// keep(i) is a pure function of (seed, i), so the backward pass draws the same mask again and nothing is stored.
// The generator is Philox-4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011): block b = i / 8 is the counter (b, 0) under the key `seed`, and its four words are eight
// half-words, one an element, compared with round(p * 2^16).  scale = 2^16 / (2^16 - threshold) belongs to the
// rounded probability, so the expectation is exact.
//
// A thread owns one block of eight elements: the generator's 40 multiplications serve eight elements (16 bits each
// decide to 1/65536, finer than any rate in use; a word an element would double them).
#include <math.h>

#include "numeric.cuh"

namespace cobalt {

constexpr int kDropoutThreads = 256;
constexpr int kDropoutBlock = 8;         // elements of one counter

__device__ __forceinline__ uint4 philox_4x32_10(uint32_t c0, uint32_t c1, uint32_t k0, uint32_t k1)
{
    uint32_t c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint32_t h0 = __umulhi(c0, 0xD2511F53u), l0 = c0 * 0xD2511F53u;
        const uint32_t h1 = __umulhi(c2, 0xCD9E8D57u), l1 = c2 * 0xCD9E8D57u;
        c0 = h1 ^ c1 ^ k0;
        c1 = l1;
        c2 = h0 ^ c3 ^ k1;
        c3 = l0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// One block of up to eight elements; `add` is the residual (may be null).
template <typename T, bool kWhole>
__device__ __forceinline__ void dropout_block(const T* x, const T* add, T* out, int64_t first, int count, uint4 rnd,
                                              uint32_t threshold, float scale)
{
    constexpr int kVecs = kDropoutBlock / Vec16<T>::kElems;
    const uint32_t w[4] = {rnd.x, rnd.y, rnd.z, rnd.w};
    if (kWhole) {
        uint4 xv[kVecs], av[kVecs];
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            xv[v] = ld_once16(x + first + v * Vec16<T>::kElems);
            if (add) av[v] = ld_once16(add + first + v * Vec16<T>::kElems);
        }
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            float f[Vec16<T>::kElems], a[Vec16<T>::kElems];
            Vec16<T>::unpack(xv[v], f);
            if (add) Vec16<T>::unpack(av[v], a);
#pragma unroll
            for (int i = 0; i < Vec16<T>::kElems; ++i) {
                const int e = v * Vec16<T>::kElems + i;
                const uint32_t half = (e & 1) ? (w[e >> 1] >> 16) : (w[e >> 1] & 0xFFFFu);
                const float kept = half >= threshold ? f[i] * scale : 0.0f;   // a select: a dropped infinity is 0 too
                f[i] = add ? a[i] + kept : kept;
            }
            st_stream16(out + first + v * Vec16<T>::kElems, Vec16<T>::pack(f));
        }
    } else {
#pragma unroll
        for (int e = 0; e < kDropoutBlock; ++e) {
            if (e < count) {
                const uint32_t half = (e & 1) ? (w[e >> 1] >> 16) : (w[e >> 1] & 0xFFFFu);
                const float kept = half >= threshold ? static_cast<float>(x[first + e]) * scale : 0.0f;
                out[first + e] = static_cast<T>(add ? static_cast<float>(add[first + e]) + kept : kept);
            }
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kDropoutThreads)
dropout_kernel(const T* x, const T* add, T* out, int64_t n, uint64_t seed, const uint64_t* seed_ptr, uint32_t threshold,
               float scale)
{
    if (seed_ptr) seed = *seed_ptr;
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const int64_t blocks = (n + kDropoutBlock - 1) / kDropoutBlock;
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kDropoutThreads;
    for (int64_t b = static_cast<int64_t>(blockIdx.x) * kDropoutThreads + threadIdx.x; b < blocks; b += stride) {
        const uint4 rnd = philox_4x32_10(static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32), k0, k1);
        const int64_t first = b * kDropoutBlock;
        if (first + kDropoutBlock <= n)
            dropout_block<T, true>(x, add, out, first, kDropoutBlock, rnd, threshold, scale);
        else
            dropout_block<T, false>(x, add, out, first, static_cast<int>(n - first), rnd, threshold, scale);
    }
}

static int launch_dropout(const void* x, const void* add, int64_t n, int32_t dtype, double p, uint64_t seed, void* out,
                          uint32_t flags, cobalt_stream_t stream)
{
    if (n < 0 || !(p >= 0.0 && p <= 1.0) || (dtype != COBALT_BF16 && dtype != COBALT_F32) ||
        (flags & ~COBALT_SEED_ON_DEVICE))
        return COBALT_ERR_INVALID_ARG;
    if (n == 0) return COBALT_OK;
    if (!x || !out || !aligned16(x) || !aligned16(add) || !aligned16(out)) return COBALT_ERR_INVALID_ARG;
    const uint64_t* seed_ptr = nullptr;
    if (flags & COBALT_SEED_ON_DEVICE) {
        if (seed == 0 || seed % 8 != 0) return COBALT_ERR_INVALID_ARG;
        seed_ptr = reinterpret_cast<const uint64_t*>(static_cast<uintptr_t>(seed));
    }
    const uint32_t threshold = static_cast<uint32_t>(floor(p * 65536.0 + 0.5));   // 65536: everything is dropped
    const float scale = threshold < 65536u ? static_cast<float>(65536.0 / (65536.0 - threshold)) : 0.0f;
    const int64_t ctas = ((n + kDropoutBlock - 1) / kDropoutBlock + kDropoutThreads - 1) / kDropoutThreads;
    const unsigned grid = static_cast<unsigned>(ctas < 0x7FFFFFFFll ? ctas : 0x7FFFFFFFll);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16)
        dropout_kernel<__nv_bfloat16><<<grid, kDropoutThreads, 0, s>>>(
            static_cast<const __nv_bfloat16*>(x), static_cast<const __nv_bfloat16*>(add),
            static_cast<__nv_bfloat16*>(out), n, seed, seed_ptr, threshold, scale);
    else
        dropout_kernel<float><<<grid, kDropoutThreads, 0, s>>>(static_cast<const float*>(x), static_cast<const float*>(add),
                                                               static_cast<float*>(out), n, seed, seed_ptr, threshold,
                                                               scale);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_dropout_add(const void* x, const void* residual, int64_t n, int32_t dtype, double p, uint64_t seed, void* out,
                       uint32_t flags, cobalt_stream_t stream)
{
    return launch_dropout(x, residual, n, dtype, p, seed, out, flags, stream);
}

int cobalt_dropout_add_backward(const void* grad_out, int64_t n, int32_t dtype, double p, uint64_t seed, void* grad_x,
                                uint32_t flags, cobalt_stream_t stream)
{
    // the adjoint of x -> keep * scale * x is itself; the residual's gradient is grad_out
    return launch_dropout(grad_out, nullptr, n, dtype, p, seed, grad_x, flags, stream);
}

}  // extern "C"
