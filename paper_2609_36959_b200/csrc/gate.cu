// Gate: the K largest logits of every token, their normalised weights, and the gradient of the logits.
//
//   ids[t]  = the K largest logits of token t in descending order, equal ones by ascending expert id
//   w[t][k] = exp(l_k - l_0) / sum_j exp(l_j - l_0)               softmax over the chosen
//           = s_k / sum_j s_j,  s = 1 / (1 + exp(-l))             sigmoid, renormalised over the chosen
//   dl_k    = w_k (g_k - sum_j g_j w_j)  [ * (1 - s_k) with sigmoid ], 0 for the experts that were not chosen
//
// One warp a token, its E logits in registers (element e in lane e % 32).  The K-th largest of the 32 lane maxima is a
// bound that at least K logits reach, and few more do (about 10 of 256 for K = 8).  Those go to shared memory, and
// their rank is the number of larger ones.  A token with NaNs, or with more candidates than the list holds (many equal
// logits), takes K rounds over all its logits instead: largest key by an integer reduction of the warp, lowest id among
// equal keys by a second one.  Bound by instructions (about 200 a token against 480 for the rounds alone at E = 256,
// K = 8), then by the 4E bytes that a token reads.
#include "numeric.cuh"

namespace cobalt {

constexpr int kGateThreads = 256;
constexpr int kGateWarps = kGateThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;

constexpr int kGateList = 64;                               // candidates of a token that are ranked directly

// Unsigned integers in the order of the values: -inf < ... < -0 = +0 < ... < +inf < NaN (a NaN is chosen first and
// shows in the weights).  The smallest key of a value is 0x007FFFFF (-inf), so 0 marks "taken or absent".
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(v + 0.0f);          // -0 + 0 = +0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// The larger of two values, NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
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

// Weights of the chosen logits: lane k < K holds value v.
__device__ __forceinline__ float chosen_weight(float v, int K, int lane, bool sigmoid)
{
    const float top = __shfl_sync(kAll, v, 0);
    if (top == -INFINITY) return 0.0f;                     // every expert masked: no weight, and no NaN
    float score = 0.0f;
    if (lane < K) {
        if (sigmoid) {
            // s_k up to the common factor exp(min(top, 0)): the ratio survives where s itself underflows
            const float m = fminf(top, 0.0f);
            score = v <= 0.0f ? expf(v - m) / (1.0f + expf(v)) : 1.0f / (1.0f + expf(-v));
        } else {
            score = expf(v - top);
        }
    }
    const float sum = warp_sum(score);
    return score / sum;
}

// K rounds over all logits of the token; lane k gets the k-th.
template <int VPL>
__device__ void choose_by_rounds(const float (&v)[VPL], int E, int K, int lane, uint32_t* my_key, int* my_id)
{
    uint32_t key[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) key[j] = j * 32 + lane < E ? order_key(v[j]) : 0u;
    for (int k = 0; k < K; ++k) {
        uint32_t best = 0;
        int at = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (key[j] > best) {                            // strictly larger: the lowest id of a lane stays
                best = key[j];
                at = j;
            }
        const uint32_t top = __reduce_max_sync(kAll, best);
        const int id = __reduce_min_sync(kAll, best == top ? at * 32 + lane : 0x7FFFFFFF);
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (j * 32 + lane == id) key[j] = 0;
        if (lane == k) {
            *my_key = top;
            *my_id = id;
        }
    }
}

// VPL: logits a lane holds (E <= 32 * VPL).
template <typename T, int VPL>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_kernel(const T* __restrict__ logits, int64_t T_, int E, int K, bool sigmoid, int32_t* __restrict__ ids,
                 float* __restrict__ weights)
{
    // a candidate: its key, then the complement of its id, so that a larger word comes first
    __shared__ unsigned long long list[kGateWarps][kGateList];
    __shared__ unsigned long long chosen[kGateWarps][COBALT_MAX_TOPK];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + warp;
    if (t >= T_) return;
    const T* row = logits + t * E;
    float v[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) v[j] = j * 32 + lane < E ? load_logit(row + j * 32 + lane) : -INFINITY;
    uint32_t my_key = 0;
    int my_id = 0;
    bool ranked = false;
    if (VPL > 1) {
        float best = v[0];
#pragma unroll
        for (int j = 1; j < VPL; ++j) best = max_nan(best, v[j]);
        uint32_t key = order_key(best), bound = 0;
        const bool any_nan = __any_sync(kAll, best != best);
        for (int k = 0; k < K; ++k) {                       // equal maxima leave together: the bound is then lower still
            bound = __reduce_max_sync(kAll, key);
            if (key == bound) key = 0;
        }
        // (all lanes gone: fewer than K different maxima, take every logit)
        const float least = bound == 0 ? -INFINITY : key_value(bound);
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (v[j] >= least && j * 32 + lane < E) mask |= 1u << j;
        const int count = __popc(mask);
        int at = count;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(kAll, at, off);
            if (lane >= off) at += o;
        }
        const int n = __shfl_sync(kAll, at, 31);
        at -= count;
        if (n <= kGateList && !any_nan) {
            ranked = true;
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if ((mask >> j) & 1u)
                    list[warp][at++] = (static_cast<unsigned long long>(order_key(v[j])) << 32) | ~static_cast<uint32_t>(j * 32 + lane);
            __syncwarp();
            for (int i = lane; i < n; i += 32) {
                const unsigned long long mine = list[warp][i];
                int rank = 0;
                for (int c = 0; c < n; ++c) rank += list[warp][c] > mine;
                if (rank < K) chosen[warp][rank] = mine;
            }
            __syncwarp();
            if (lane < K) {
                const unsigned long long c = chosen[warp][lane];
                my_key = static_cast<uint32_t>(c >> 32);
                my_id = static_cast<int>(~static_cast<uint32_t>(c));
            }
        }
    }
    if (!ranked) choose_by_rounds<VPL>(v, E, K, lane, &my_key, &my_id);
    const float value = my_key == 0xFFFFFFFFu ? __int_as_float(0x7FC00000) : key_value(my_key);
    const float w = chosen_weight(value, K, lane, sigmoid);
    if (lane < K) {
        ids[t * K + lane] = my_id;
        weights[t * K + lane] = w;
    }
}

__device__ __forceinline__ void store_grad(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_grad(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The sigmoid's 1 - s_k needs the sum S of the chosen sigmoids, s_k = w_k S: S = s_0 / w_0 from the first logit alone,
// one gathered sector a token instead of K (41 to 33 us at T = 131072, E = 256, K = 8).
template <typename T, bool kVector>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_backward_kernel(const float* __restrict__ grad_w, const T* __restrict__ logits, const int32_t* __restrict__ ids,
                          const float* __restrict__ weights, int64_t T_, int E, int K, bool sigmoid,
                          T* __restrict__ grad_logits, uint32_t* __restrict__ err_word)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + (threadIdx.x >> 5);
    if (t >= T_) return;
    T* row = grad_logits + t * E;
    if (kVector) {                                          // rows are whole 16-byte vectors
        for (int e = lane * Vec16<T>::kElems; e < E; e += 32 * Vec16<T>::kElems)
            *reinterpret_cast<uint4*>(row + e) = make_uint4(0, 0, 0, 0);
    } else {
        for (int e = lane; e < E; e += 32) store_grad(row + e, 0.0f);
    }
    int id = -1;
    float g = 0.0f, w = 0.0f;
    if (lane < K) {
        id = ids[t * K + lane];
        g = grad_w[t * K + lane];
        w = weights[t * K + lane];
        if (id < 0 || id >= E) {
            flag_error(err_word, COBALT_DEVERR_BAD_EXPERT_ID);
            id = -1;
        }
    }
    const float dot = warp_sum(g * w);
    float d = w * (g - dot);
    if (sigmoid) {
        float total = 0.0f;
        if (lane == 0 && id >= 0 && w > 0.0f) total = 1.0f / (1.0f + expf(-load_logit(logits + t * E + id))) / w;
        total = __shfl_sync(kAll, total, 0);
        d *= 1.0f - w * total;
    }
    __syncwarp();                                           // the zeros of other lanes come before the chosen values
    if (id >= 0) store_grad(row + id, d);
}

static int check_gate(int64_t T, int32_t E, int32_t K, int32_t dtype, uint32_t flags)
{
    if (T < 0 || E < 1 || K < 1 || K > E || (dtype != COBALT_BF16 && dtype != COBALT_F32) || (flags & ~COBALT_GATE_SIGMOID))
        return COBALT_ERR_INVALID_ARG;
    if (E > COBALT_MAX_EXPERTS || K > COBALT_MAX_TOPK || T * static_cast<int64_t>(K) >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

template <typename T>
static void launch_gate(const void* logits, int64_t T_, int E, int K, bool sigmoid, int32_t* ids, float* w, cudaStream_t s)
{
    const unsigned grid = static_cast<unsigned>((T_ + kGateWarps - 1) / kGateWarps);
    const T* l = static_cast<const T*>(logits);
    if (E <= 32) gate_topk_kernel<T, 1><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
    else if (E <= 64) gate_topk_kernel<T, 2><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
    else if (E <= 128) gate_topk_kernel<T, 4><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
    else if (E <= 256) gate_topk_kernel<T, 8><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
    else if (E <= 512) gate_topk_kernel<T, 16><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
    else gate_topk_kernel<T, 32><<<grid, kGateThreads, 0, s>>>(l, T_, E, K, sigmoid, ids, w);
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
    const unsigned grid = static_cast<unsigned>((T + kGateWarps - 1) / kGateWarps);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool vector = E % (dtype == COBALT_BF16 ? 8 : 4) == 0;
#define COBALT_GATE_BACKWARD(TT, VECTOR)                                                                                      \
    gate_topk_backward_kernel<TT, VECTOR><<<grid, kGateThreads, 0, s>>>(grad_gate_w, static_cast<const TT*>(logits), topk_ids, gate_w, \
                                                                        T, E, K, sigmoid, static_cast<TT*>(grad_logits), err_word)
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
