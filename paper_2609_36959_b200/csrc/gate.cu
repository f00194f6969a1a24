// Gate: the K largest logits of every token, their normalised weights, and the gradient of the logits.
//
//   ids[t]  = the K largest logits of token t in descending order, equal ones by ascending expert id
//   w[t][k] = exp(l_k - l_0) / sum_j exp(l_j - l_0)               softmax over the chosen
//           = s_k / sum_j s_j,  s = 1 / (1 + exp(-l))             sigmoid, renormalised over the chosen
//   dl_k    = w_k (g_k - sum_j g_j w_j)  [ * (1 - s_k) with sigmoid ], 0 for the experts that were not chosen
//
// L = 8, 16 or 32 lanes take a token, its E logits in their registers; L is at least K, and a warp holds 32 / L tokens.
// Each lane keeps the maxima of four parts of its logits; the K-th largest of these 4L maxima is a bound that K logits
// reach at least, and few more do (about 10 of 256 for K = 8).  Those go to shared memory, and their rank is the number
// of larger ones.  A token with NaNs, or with more candidates than the list holds (many equal logits), takes K rounds
// over all its logits instead.  Bound by instructions, which several tokens a warp share, then by the 4E bytes that a
// token reads.  131072 x 256 fp32, K = 8: 35 us (the reads alone 21), the gradient 27 us, with sigmoid 41 us: its 2^20
// gathered logits are as many DRAM bursts of 64 bytes (10 us).
#include "numeric.cuh"

namespace cobalt {

constexpr int kGateThreads = 256;
constexpr int kGateWarps = kGateThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;

constexpr int kGateList = 64;                               // candidates of a token that are ranked directly

// Unsigned integers in the order of the values: -inf < ... < -0 = +0 < ... < +inf (0xFF800000) < NaN (a NaN is chosen first
// and shows in the weights).  The smallest key of a value is 0x007FFFFF (-inf), so 0 marks "taken or absent"; the largest
// word is left free for "above every candidate".
constexpr uint32_t kNanKey = 0xFFFFFFFEu;

__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return kNanKey;
    const uint32_t b = __float_as_uint(v + 0.0f);          // -0 + 0 = +0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The larger and the lesser of two values, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ float key_value(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
}

__device__ __forceinline__ float load_logit(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_logit(const __nv_bfloat16* p)
{
    return __uint_as_float(static_cast<uint32_t>(__ldg(reinterpret_cast<const unsigned short*>(p))) << 16);
}

// Weights of the chosen logits among L lanes: lane k < K of them holds value v, the first one the largest.
template <int L>
__device__ __forceinline__ float chosen_weight(float v, int K, int k, bool sigmoid)
{
    const float top = __shfl_sync(kAll, v, 0, L);
    float score = 0.0f;
    if (k < K) {
        if (sigmoid) {
            // s_k up to the common factor exp(min(top, 0)): the ratio survives where s itself underflows
            const float m = fminf(top, 0.0f);
            score = v <= 0.0f ? expf(v - m) / (1.0f + expf(v)) : 1.0f / (1.0f + expf(-v));
        } else {
            score = expf(v - top);
        }
    }
    float sum = score;
#pragma unroll
    for (int off = 1; off < L; off <<= 1) sum += __shfl_xor_sync(kAll, sum, off);
    return top == -INFINITY ? 0.0f : score / sum;          // every expert masked: no weight, and no NaN
}

// Where logit j of a lane stands in the row: chunks of kChunk neighbouring logits (one 16-byte load) go to the L lanes in
// turn; kChunk = 1 for rows that are no whole vectors.
template <int L, int kChunk>
__device__ __forceinline__ int logit_place(int j, int sub)
{
    return (j / kChunk * L + sub) * kChunk + j % kChunk;
}

// The lane's logits; -inf behind the row's end.
template <int L, int VPL, int kChunk, typename T>
__device__ __forceinline__ void load_logits(const T* row, int E, int sub, float (&v)[VPL])
{
#pragma unroll
    for (int j = 0; j < VPL; j += kChunk) {
        const int e = logit_place<L, kChunk>(j, sub);
        if constexpr (kChunk == 1) {
            v[j] = e < E ? load_logit(row + e) : -INFINITY;
        } else {
            float f[kChunk];
#pragma unroll
            for (int k = 0; k < kChunk; ++k) f[k] = -INFINITY;
            if (e < E) Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(row + e)), f);
#pragma unroll
            for (int k = 0; k < kChunk; ++k) v[j + k] = f[k];
        }
    }
}

// A candidate as one integer, larger ones first: the value's order, then the lower id.
__device__ __forceinline__ unsigned long long candidate(float v, int id)
{
    return (static_cast<unsigned long long>(order_key(v)) << 32) | ~static_cast<uint32_t>(id);
}

// K rounds over all logits of the token, read again each time; lane k gets the k-th candidate.
template <int L, typename T>
__device__ __noinline__ unsigned long long choose_by_rounds(const T* row, int E, int K, int sub)
{
    unsigned long long mine = 0, last = ~0ull;               // above every candidate
    for (int k = 0; k < K; ++k) {
        unsigned long long best = 0;                        // the largest below the one before
        for (int e = sub; e < E; e += L) {
            const unsigned long long c = candidate(load_logit(row + e), e);
            if (c < last && c > best) best = c;
        }
        for (int off = 1; off < L; off <<= 1) {
            const unsigned long long o = __shfl_xor_sync(kAll, best, off);
            best = o > best ? o : best;
        }
        last = best;
        if (sub == k) mine = best;
    }
    return mine;
}

__device__ __forceinline__ void order_pair(float& a, float& b)
{
    const float hi = max_nan(a, b), lo = min_nan(a, b);
    a = hi;
    b = lo;
}

// VPL: logits a lane holds (E <= L * VPL).
template <typename T, int L, int VPL, int kChunk>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_kernel(const T* __restrict__ logits, int64_t T_, int E, int K, bool sigmoid, int32_t* __restrict__ ids,
                 float* __restrict__ weights)
{
    constexpr int kTokens = 32 / L;                         // of a warp
    __shared__ unsigned long long list[kGateWarps][kTokens][kGateList];
    __shared__ unsigned long long chosen[kGateWarps][kTokens][COBALT_MAX_TOPK];
    __shared__ int listed[kGateWarps][kTokens];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % L, own = lane / L;
    const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * kGateWarps + warp) * kTokens, t = t0 + own;
    if (t0 >= T_) return;
    const T* row = logits + (t < T_ ? t : T_ - 1) * E;
    float v[VPL];
    load_logits<L, VPL, kChunk>(row, E, sub, v);
    if (sub == 0) listed[warp][own] = 0;
    // (a NaN stays a NaN through all of this, and every comparison with the bound is then false: no candidates)
    float part[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        part[q] = v[q * (VPL / 4)];
#pragma unroll
        for (int j = 1; j < VPL / 4; ++j) part[q] = max_nan(part[q], v[q * (VPL / 4) + j]);
    }
    order_pair(part[0], part[1]);
    order_pair(part[2], part[3]);
    order_pair(part[0], part[2]);
    order_pair(part[1], part[3]);
    order_pair(part[1], part[2]);
    float least = 0.0f;
    for (int k = 0; k < K; ++k) {                           // equal maxima of several lanes leave together
        least = part[0];
#pragma unroll
        for (int off = 1; off < L; off <<= 1) least = max_nan(least, __shfl_xor_sync(kAll, least, off));
        if (part[0] == least) {
            part[0] = part[1];
            part[1] = part[2];
            part[2] = part[3];
            part[3] = -INFINITY;
        }
    }
    uint32_t mask = 0;
    if (E == L * VPL) {
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (v[j] >= least) mask |= 1u << j;
    } else {
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (v[j] >= least && logit_place<L, kChunk>(j, sub) < E) mask |= 1u << j;
    }
    __syncwarp();
    // places in the list are dealt in any order: the ranks do not depend on it
    int at = 0;
    if (mask != 0) at = atomicAdd(&listed[warp][own], __popc(mask));
    __syncwarp();
    const int n = listed[warp][own];
    const bool ranked = n >= K && n <= kGateList;
    if (ranked) {
        while (mask != 0) {                                 // one or two a lane: read again, the registers cannot be indexed
            const int e = logit_place<L, kChunk>(__ffs(mask) - 1, sub);
            mask &= mask - 1;
            list[warp][own][at++] = candidate(load_logit(row + e), e);
        }
    }
    __syncwarp();
    if (ranked)
        for (int i = sub; i < n; i += L) {
            const unsigned long long a = list[warp][own][i];
            int rank = 0;
#pragma unroll 4
            for (int c = 0; c < n; ++c) rank += list[warp][own][c] > a;
            if (rank < K) chosen[warp][own][rank] = a;
        }
    __syncwarp();
    unsigned long long mine = ranked && sub < K ? chosen[warp][own][sub] : 0;
    if (!__all_sync(kAll, ranked)) {
        const unsigned long long slow = choose_by_rounds<L>(row, E, K, sub);
        if (!ranked) mine = slow;
    }
    const uint32_t key = static_cast<uint32_t>(mine >> 32);
    const float value = key == kNanKey ? __int_as_float(0x7FC00000) : key_value(key);
    const float w = chosen_weight<L>(value, K, sub, sigmoid);
    if (sub < K && t < T_) {
        ids[t * K + sub] = static_cast<int>(~static_cast<uint32_t>(mine));
        weights[t * K + sub] = w;
    }
}

__device__ __forceinline__ void store_grad(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_grad(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// A warp takes 32 / lanes tokens, `lanes` (K or the next power of two) lanes each for the chosen, all lanes for the zeros.
// The sigmoid's 1 - s_k is 1 / (1 + exp(l_k)) of the lane's own logit, gathered while the zeros are stored: formed as a
// difference from the rounded weights it loses all its digits where s_k is near one.
template <typename T, bool kVector>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_backward_kernel(const float* __restrict__ grad_w, const T* __restrict__ logits, const int32_t* __restrict__ ids,
                          const float* __restrict__ weights, int64_t T_, int E, int K, int lanes, bool sigmoid,
                          T* __restrict__ grad_logits, uint32_t* __restrict__ err_word)
{
    const int lane = threadIdx.x & 31, tokens = 32 / lanes;
    const int64_t t0 = (static_cast<int64_t>(blockIdx.x) * kGateWarps + (threadIdx.x >> 5)) * tokens;
    if (t0 >= T_) return;
    const int k = lane & (lanes - 1);
    const int64_t t = t0 + lane / lanes;
    int id = -1;
    float g = 0.0f, w = 0.0f;
    if (k < K && t < T_) {
        id = ids[t * K + k];
        g = grad_w[t * K + k];
        w = weights[t * K + k];
        if (id < 0 || id >= E) {
            flag_error(err_word, COBALT_DEVERR_BAD_EXPERT_ID);
            id = -1;
        }
    }
    float logit = 0.0f;
    if (sigmoid && id >= 0) logit = load_logit(logits + t * E + id);
    // the zeros of the warp's rows, which lie one after another
    const int64_t count = (T_ - t0 < tokens ? T_ - t0 : tokens) * E;
    T* rows = grad_logits + t0 * E;
    if (kVector) {                                          // rows are whole 16-byte vectors
        for (int64_t e = lane * Vec16<T>::kElems; e < count; e += 32 * Vec16<T>::kElems)
            *reinterpret_cast<uint4*>(rows + e) = make_uint4(0, 0, 0, 0);
    } else {
        for (int64_t e = lane; e < count; e += 32) store_grad(rows + e, 0.0f);
    }
    float dot = g * w;
    for (int off = 1; off < lanes; off <<= 1) dot += __shfl_xor_sync(kAll, dot, off);
    float d = w * (g - dot);
    if (sigmoid) d *= 1.0f / (1.0f + expf(logit));
    __syncwarp();                                           // the zeros of other lanes come before the chosen values
    if (id >= 0) store_grad(grad_logits + t * E + id, d);
}

static int check_gate(int64_t T, int32_t E, int32_t K, int32_t dtype, uint32_t flags)
{
    if (T < 0 || E < 1 || K < 1 || K > E || (dtype != COBALT_BF16 && dtype != COBALT_F32) || (flags & ~COBALT_GATE_SIGMOID))
        return COBALT_ERR_INVALID_ARG;
    if (E > COBALT_MAX_EXPERTS || K > COBALT_MAX_TOPK || T * static_cast<int64_t>(K) >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

static int power_of_two(int k)
{
    int n = 1;
    while (n < k) n *= 2;
    return n;
}

template <typename T, int kChunk, int L>
static bool launch_gate_lanes(const T* l, int64_t T_, int E, int K, bool sigmoid, int32_t* ids, float* w, cudaStream_t s)
{
    const int64_t per_cta = static_cast<int64_t>(kGateWarps) * (32 / L);
    const unsigned grid = static_cast<unsigned>((T_ + per_cta - 1) / per_cta);
#define COBALT_GATE(VPL)                                                                                          \
    do {                                                                                                          \
        gate_topk_kernel<T, L, VPL, kChunk><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);          \
        return true;                                                                                              \
    } while (0)
    if constexpr (L < 32) {                                 // 32 lanes only take what is too long for 16
        if constexpr (kChunk <= 4)
            if (E <= 4 * L) COBALT_GATE(4);
        if (E <= 8 * L) COBALT_GATE(8);
        if (E <= 16 * L) COBALT_GATE(16);
    }
    if (E <= 32 * L) COBALT_GATE(32);
#undef COBALT_GATE
    return false;
}

// As few lanes a token as hold its K chosen and, at 32 logits a lane, its row.
template <typename T, int kChunk>
static void launch_gate_chunk(const T* l, int64_t T_, int E, int K, bool sigmoid, int32_t* ids, float* w, cudaStream_t s)
{
    if (K <= 8 && launch_gate_lanes<T, kChunk, 8>(l, T_, E, K, sigmoid, ids, w, s)) return;
    if (launch_gate_lanes<T, kChunk, 16>(l, T_, E, K, sigmoid, ids, w, s)) return;
    (void)launch_gate_lanes<T, kChunk, 32>(l, T_, E, K, sigmoid, ids, w, s);
}

template <typename T>
static void launch_gate(const void* logits, int64_t T_, int E, int K, bool sigmoid, int32_t* ids, float* w, cudaStream_t s)
{
    const T* l = static_cast<const T*>(logits);
    if (E % Vec16<T>::kElems == 0) launch_gate_chunk<T, Vec16<T>::kElems>(l, T_, E, K, sigmoid, ids, w, s);
    else launch_gate_chunk<T, 1>(l, T_, E, K, sigmoid, ids, w, s);
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_gate_topk(const void* logits, int64_t T, int32_t E, int32_t K, int32_t dtype, int32_t* topk_ids,
                     float* gate_w, uint32_t flags, cobalt_stream_t stream)
{
    const int rc = check_gate(T, E, K, dtype, flags);
    if (rc != COBALT_OK) return rc;
    if (T == 0) return COBALT_OK;
    if (!logits || !topk_ids || !gate_w || !aligned16(logits) || !aligned16(topk_ids) || !aligned16(gate_w))
        return COBALT_ERR_INVALID_ARG;
    const bool sigmoid = (flags & COBALT_GATE_SIGMOID) != 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16) launch_gate<__nv_bfloat16>(logits, T, E, K, sigmoid, topk_ids, gate_w, s);
    else launch_gate<float>(logits, T, E, K, sigmoid, topk_ids, gate_w, s);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

int cobalt_gate_topk_backward(const float* grad_gate_w, const void* logits, const int32_t* topk_ids, const float* gate_w,
                              int64_t T, int32_t E, int32_t K, int32_t dtype, void* grad_logits, uint32_t flags,
                              cobalt_stream_t stream)
{
    int rc = check_gate(T, E, K, dtype, flags);
    if (rc != COBALT_OK) return rc;
    if (T == 0) return COBALT_OK;
    const bool sigmoid = (flags & COBALT_GATE_SIGMOID) != 0;
    if (!grad_gate_w || !topk_ids || !gate_w || !grad_logits || (sigmoid && !logits)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_gate_w) || !aligned16(logits) || !aligned16(topk_ids) || !aligned16(gate_w) || !aligned16(grad_logits))
        return COBALT_ERR_INVALID_ARG;
    uint32_t* err_word = nullptr;
    rc = device_error_word(&err_word);
    if (rc != COBALT_OK) return rc;
    const int lanes = power_of_two(K);
    const int64_t per_cta = static_cast<int64_t>(kGateWarps) * (32 / lanes);
    const unsigned grid = static_cast<unsigned>((T + per_cta - 1) / per_cta);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool vector = E % (dtype == COBALT_BF16 ? 8 : 4) == 0;
#define COBALT_GATE_BACKWARD(TT, VECTOR)                                                                                      \
    gate_topk_backward_kernel<TT, VECTOR><<<grid, kGateThreads, 0, s>>>(grad_gate_w, static_cast<const TT*>(logits), topk_ids, gate_w, \
                                                                        T, E, K, lanes, sigmoid, static_cast<TT*>(grad_logits), err_word)
    if (dtype == COBALT_BF16) {
        if (vector) COBALT_GATE_BACKWARD(__nv_bfloat16, true);
        else COBALT_GATE_BACKWARD(__nv_bfloat16, false);
    } else {
        if (vector) COBALT_GATE_BACKWARD(float, true);
        else COBALT_GATE_BACKWARD(float, false);
    }
#undef COBALT_GATE_BACKWARD
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // extern "C"
