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
// A thread owns blocks of eight elements: the generator's 20 wide multiplications serve eight elements (16 bits each
// decide to 1/65536, finer than any rate in use; a word an element would double them).
#include <math.h>

#include "numeric.cuh"

namespace cobalt {

constexpr int kDropoutThreads = 256;
constexpr int kDropoutBlock = 8;         // elements of one counter
constexpr int kDropoutUnroll = 1;        // blocks a thread has in flight

__device__ __forceinline__ uint4 philox_4x32_10(uint32_t c0, uint32_t c1, uint32_t k0, uint32_t k1)
{
    uint32_t c2 = 0, c3 = 0;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
        c1 = static_cast<uint32_t>(b);
        c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
        c3 = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// The threshold in the upper half of a word, to which whole words compare: the high half-word decides there alone, and
// the low one after a shift.  `any` is false when the threshold is 2^16, which no word reaches.
struct DropoutRule {
    uint32_t limit;
    bool any;
    float scale;
};

__device__ __forceinline__ float dropout_value(float v, uint32_t word, int e, const DropoutRule& rule)
{
    const uint32_t w = (e & 1) ? word : word << 16;
    return (w >= rule.limit && rule.any) ? v * rule.scale : 0.0f;      // a select: a dropped infinity is 0 too
}

template <typename T>
__global__ void __launch_bounds__(kDropoutThreads)
dropout_kernel(const T* x, const T* add, T* out, int64_t n, uint64_t seed, const uint64_t* seed_ptr, DropoutRule rule)
{
    constexpr int N = Vec16<T>::kElems, kVecs = kDropoutBlock / N;
    if (seed_ptr) seed = *seed_ptr;
    const uint32_t k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
    const int64_t whole = n / kDropoutBlock, stride = static_cast<int64_t>(gridDim.x) * kDropoutThreads * kDropoutUnroll;
    for (int64_t base = static_cast<int64_t>(blockIdx.x) * kDropoutThreads * kDropoutUnroll + threadIdx.x; base < whole; base += stride) {
        uint4 xv[kDropoutUnroll][kVecs], av[kDropoutUnroll][kVecs];
#pragma unroll
        for (int u = 0; u < kDropoutUnroll; ++u) {
            const int64_t b = base + u * kDropoutThreads;
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                if (b < whole) {
                    xv[u][v] = ld_once16(x + b * kDropoutBlock + v * N);
                    if (add) av[u][v] = ld_once16(add + b * kDropoutBlock + v * N);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kDropoutUnroll; ++u) {
            const int64_t b = base + u * kDropoutThreads;
            if (b >= whole) break;
            const uint4 rnd = philox_4x32_10(static_cast<uint32_t>(b), static_cast<uint32_t>(b >> 32), k0, k1);
            const uint32_t w[4] = {rnd.x, rnd.y, rnd.z, rnd.w};
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
                float f[N], a[N];
                Vec16<T>::unpack(xv[u][v], f);
                if (add) Vec16<T>::unpack(av[u][v], a);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int e = v * N + i;
                    const float kept = dropout_value(f[i], w[e >> 1], e, rule);
                    f[i] = add ? a[i] + kept : kept;
                }
                st_stream16(out + b * kDropoutBlock + v * N, Vec16<T>::pack(f));
            }
        }
    }
    // the last n % 8 elements
    if (blockIdx.x == 0 && threadIdx.x < n % kDropoutBlock) {
        const uint4 rnd = philox_4x32_10(static_cast<uint32_t>(whole), static_cast<uint32_t>(whole >> 32), k0, k1);
        const uint32_t w[4] = {rnd.x, rnd.y, rnd.z, rnd.w};
        const int64_t at = whole * kDropoutBlock + threadIdx.x;
#pragma unroll
        for (int e = 0; e < kDropoutBlock; ++e) {
            if (e == static_cast<int>(threadIdx.x)) {
                const float kept = dropout_value(static_cast<float>(x[at]), w[e >> 1], e, rule);
                out[at] = static_cast<T>(add ? static_cast<float>(add[at]) + kept : kept);
            }
        }
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
    DropoutRule rule;
    rule.limit = threshold << 16;
    rule.any = threshold < 65536u;
    rule.scale = rule.any ? static_cast<float>(65536.0 / (65536.0 - threshold)) : 0.0f;
    const int64_t per_cta = static_cast<int64_t>(kDropoutThreads) * kDropoutUnroll * kDropoutBlock;
    const int64_t ctas = (n + per_cta - 1) / per_cta;
    const unsigned grid = static_cast<unsigned>(ctas < 0x7FFFFFFFll ? ctas : 0x7FFFFFFFll);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16)
        dropout_kernel<__nv_bfloat16><<<grid, kDropoutThreads, 0, s>>>(static_cast<const __nv_bfloat16*>(x),
                                                                       static_cast<const __nv_bfloat16*>(add),
                                                                       static_cast<__nv_bfloat16*>(out), n, seed, seed_ptr, rule);
    else
        dropout_kernel<float><<<grid, kDropoutThreads, 0, s>>>(static_cast<const float*>(x), static_cast<const float*>(add),
                                                               static_cast<float*>(out), n, seed, seed_ptr, rule);
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
