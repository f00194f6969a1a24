// Gate: the K largest logits of every token, their normalised weights, and the gradient of the logits.
//
//   ids[t]  = the K largest logits of token t in descending order, equal ones by ascending expert id
//   w[t][k] = exp(l_k - l_0) / sum_j exp(l_j - l_0)               softmax over the chosen
//           = s_k / sum_j s_j,  s = 1 / (1 + exp(-l))             sigmoid, renormalised over the chosen
//   dl_k    = w_k (g_k - sum_j g_j w_j)  [ * (1 - s_k) with sigmoid ], 0 for the experts that were not chosen
//
// One warp a token, its E logits in registers (element e in lane e % 32).  A round takes the largest key of the warp
// with one integer reduction and the lowest id among equal keys with a second one.  Bound by the instructions of the
// K rounds, not by the 4E bytes that a token reads.
#include "numeric.cuh"

namespace cobalt {

constexpr int kGateThreads = 256;
constexpr int kGateWarps = kGateThreads / 32;
constexpr uint32_t kAll = 0xFFFFFFFFu;

// Unsigned integers in the order of the values: -inf < ... < -0 = +0 < ... < +inf < NaN (a NaN is chosen first and
// shows in the weights).  The smallest key of a value is 0x007FFFFF (-inf), so 0 marks "taken or absent".
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(v + 0.0f);          // -0 + 0 = +0
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
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

// VPL: logits a lane holds (E <= 32 * VPL).
template <typename T, int VPL>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_kernel(const T* __restrict__ logits, int64_t T_, int E, int K, bool sigmoid, int32_t* __restrict__ ids,
                 float* __restrict__ weights)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + (threadIdx.x >> 5);
    if (t >= T_) return;
    const T* row = logits + t * E;
    uint32_t key[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int e = j * 32 + lane;
        key[j] = e < E ? order_key(load_logit(row + e)) : 0u;
    }
    uint32_t my_key = 0;
    int my_id = 0;
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
        if (lane == (id & 31)) {
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if (j == (id >> 5)) key[j] = 0;
        }
        if (lane == k) {
            my_key = top;
            my_id = id;
        }
    }
    const float v = my_key == 0xFFFFFFFFu ? __int_as_float(0x7FC00000) : key_value(my_key);
    const float w = chosen_weight(v, K, lane, sigmoid);
    if (lane < K) {
        ids[t * K + lane] = my_id;
        weights[t * K + lane] = w;
    }
}

__device__ __forceinline__ void store_grad(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_grad(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <typename T>
__global__ void __launch_bounds__(kGateThreads)
gate_topk_backward_kernel(const float* __restrict__ grad_w, const T* __restrict__ logits, const int32_t* __restrict__ ids,
                          const float* __restrict__ weights, int64_t T_, int E, int K, bool sigmoid,
                          T* __restrict__ grad_logits, uint32_t* __restrict__ err_word)
{
    const int lane = threadIdx.x & 31;
    const int64_t t = static_cast<int64_t>(blockIdx.x) * kGateWarps + (threadIdx.x >> 5);
    if (t >= T_) return;
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
    T* row = grad_logits + t * E;
    for (int e = lane; e < E; e += 32) store_grad(row + e, 0.0f);
    __syncwarp();                                           // the zeros of other lanes come before the chosen values
    if (id >= 0) {
        float d = w * (g - dot);
        if (sigmoid) d *= 1.0f / (1.0f + expf(load_logit(logits + t * E + id)));   // 1 - s
        store_grad(row + id, d);
    }
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
    if (dtype == COBALT_BF16)
        gate_topk_backward_kernel<__nv_bfloat16><<<grid, kGateThreads, 0, s>>>(
            grad_gate_w, static_cast<const __nv_bfloat16*>(logits), topk_ids, gate_w, T, E, K, sigmoid,
            static_cast<__nv_bfloat16*>(grad_logits), err_word);
    else
        gate_topk_backward_kernel<float><<<grid, kGateThreads, 0, s>>>(grad_gate_w, static_cast<const float*>(logits), topk_ids,
                                                                       gate_w, T, E, K, sigmoid,
                                                                       static_cast<float*>(grad_logits), err_word);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // extern "C"
