// A dense product with its elementwise part, and its gradients.
//
//   pre = x W^T + b      out = act(pre) + residual            x [T, K], W [N, K], bf16, or e4m3 with a scale for each row
//   d = dout act'(pre)   dx = d W   dW = d^T x   db = sum_t d
//
// Three products, one kernel template (tcgen05, fp32 accumulators in tensor memory).  All of them have the form
//   D[j][i] = sum_k A(i, k) B(j, k)     with i contiguous in the result:
//   forward  i = feature, j = token, k over K      A = W, B = x
//   dx       i = column of x, j = token, k over N  A = W transposed, B = d
//   dW       i = column of x, j = feature, k over T   A = x transposed, B = d transposed
//
//   - A CTA pair computes 256 of i (M, 128 a CTA) by n of j (N, a multiple of 32 up to 256).  Warp 0 of each CTA feeds a ring of
//     128-byte deep blocks by tensor-map loads, warp 1 of the leading CTA issues the products, warps 2 to 9 run the epilogue
//     under the products of the next tile (two accumulators).
//   - Persistent pairs deal the tiles round robin.  Where a product has fewer tiles than there are pairs, k is split; the parts
//     go to the workspace in fp32 and a second kernel adds them in order and runs the epilogue.
//   - Where k is short (four blocks) and i long, a router's dx, a pair keeps its j's operand in shared memory for all tiles of i and only
//     the other one streams: half of what went through L2, which bounded that product (11 TB/s).
//   - Epilogue: bias, scales and activation are applied to the accumulators as they are read, and bf16 results leave through shared
//     memory by tensor-map stores.  With a residual, a saved pre-activation or kLong the accumulators pass through shared memory in
//     fp32 instead, 32 columns of j at a time, so that a thread has eight neighbouring i of one j: everything moves in 16-byte vectors, and
//     the 128 i that share a scale when pre is kept in 8 bits are sixteen neighbouring lanes.
//   - One token, or a few and a small W: the fp32 units, W's rows streamed by warps.
//
// Large products are bound by the tensor pipe, and back to back by the 1000 W cap: 8192 tokens, 4096 to 2816, alone: forward (silu, residual,
// 8-bit pre) 133 us, dx 119 us (1590 TFLOP/s), dW 131 us (pipe 86, 94 and 91 % active).  A router's products move 1.9 GB of x or dx for 256
// features: logits 390 us (L2 to the SMs, 9.6 TB/s), dx 431 us (writes: torch's fill of the same 1.9 GB takes 487), dW 335 us.  Small
// calls are bound by their launch and the first loads (64 x 256 to 256: 3.9 us in a graph).
//
// Every wait is bounded: when one runs out the kernel sets COBALT_DEVERR_WAIT_TIMEOUT, drains its copies, frees its tensor
// memory and returns.
#include "linear_plan.h"
#include "packed.cuh"
#include "tcgen05.cuh"
#include "tensor_map.cuh"

namespace cobalt {

typedef __nv_bfloat16 bf16;

constexpr int kHalfBytes = 128 * kDeepBytes;
constexpr int kSlotBytes = 2 * kHalfBytes;
constexpr int kBoxBytes = 64 * kDeepBytes;       // MN-major box: 64 values of M or N x 64 of k
constexpr int kRing = 6;
constexpr int kStayBlocks = 4;           // blocks of k that stay: beside them the ring has eight slots of the other operand
constexpr int kStayRing = (kRing * kSlotBytes - kStayBlocks * kHalfBytes) / kHalfBytes;
// Epilogue staging of 128 values of i, two buffers for each of two groups of four warps: 32 j in bf16, as two boxes of 64 values with the
// 128-byte swizzle, or 16 j in fp32, an odd number of 16-byte units each.
constexpr int kBox16 = 32 * 128, kBuffer16 = 2 * kBox16;
constexpr int kPitch32 = 528, kBuffer32 = 16 * kPitch32;
constexpr int kStaging = 4 * (kBuffer16 > kBuffer32 ? kBuffer16 : kBuffer32);
constexpr int kLinearSmem = kRing * kSlotBytes + kStaging + 256;
constexpr int kLinearThreads = 320;
// Blocks of k that the tensor cores add up before fp32 registers take over (kLong): 512 bf16 values or 1024 e4m3 ones of an fp32 result,
// 8192 tokens of the weights' gradient.
constexpr int kResultBlocks = 8, kTokenBlocks = 128;
constexpr int kBand = 8;                 // tiles of j that run together for every tile of i

enum Product { kForward, kForwardE4M3, kGradRows, kGradWeights };

// kPlain: bf16 results of bias, scales and activation alone.  kFull: any.  kLong: long sums.  The tensor cores cut every addition, 16 bf16
// products each: a sum of 7168 of either sign is 7.9e-6 off, a sum of 8192 of one sign 3.0e-5 too small, of 131072 7.7e-4 and of a million
// 6.6e-3, more than half a step of bf16.  So a part is added there and the sums of the parts, rounded, in registers: for fp32 results 512
// values at a time (4.8e-7), for the weights' gradient, where a split has more than 8192 tokens, 8192 at a time (2.3 ms at 131072 tokens,
// 4096 x 2560, as in one go).  bf16 results of sums over K or N, at most 65536 values, are added in one go: a tenth of a half step.
enum Form { kPlain, kFull, kLong };

// The elementwise part of the forward call.
struct Finish {
    const bf16* bias;                    // or null
    const void* residual;                // or null, of the result's type
    const float* x_scales;               // e4m3 only
    const float* w_scales;
    int act;
    int f32;                             // the result's type
    void* pre;                           // or null
    float* pre_scales;                   // pre in 8 bits
};

struct LinearArgs {
    int I, J;
    int n, m_tiles, j_tiles, splits, blocks, per_split;      // blocks of k: all, and those of a split
    void* out;
    float* partial;                      // [splits][J][I] where splits > 1
    Finish finish;
    uint32_t* err_word;
};

// 2^x and 1 / x by the special function unit, good to two units; results below 2^-126 are 0.
__device__ __forceinline__ float fast_exp2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_inverse(float x)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr float kLog2E = 1.44269504088896341f;

__device__ __forceinline__ float fast_sigmoid(float v) { return fast_inverse(1.0f + fast_exp2(-kLog2E * v)); }

// The tail T(a) of the normal distribution, 1 - Phi(a), for a >= 0: exp(-a^2 / 2) t Q(t) with t = 1 / (1 + 0.305 a), the form of 7.1.26 in
// Abramowitz and Stegun's Handbook.  Q, of degree 7, was fitted to the least relative error (weighted least squares, the weights times the
// error until it is level, after Lawson): 9.7e-8 for a up to 14.5, beyond which the exponential is 0.  The error has to be relative: the tail
// is all there is of gelu below 0.  (A rational power good to 3e-7 absolutely was 0.6 us of 18 faster at 4999 x 2048 to 1408, and 0.4 % off
// at -4, 5 % at -5.)  Rounding adds 1.5 a^2 + 22 units of 2^-24.
__device__ __forceinline__ Pair normal_tail(const Pair& a)
{
    const Pair arg = a * a * pair(-0.5f * kLog2E), d = fma2(a, pair(0.305f), pair(1.0f));
    const Pair t = pair(fast_inverse(d.v.x), fast_inverse(d.v.y));
    const Pair e = pair(fast_exp2(arg.v.x), fast_exp2(arg.v.y));
    Pair q = fma2(t, pair(3.663886949e-02f), pair(-1.527460937e-01f));
    q = fma2(t, q, pair(1.853149138e-01f));
    q = fma2(t, q, pair(-3.762067665e-02f));
    q = fma2(t, q, pair(1.208403976e-01f));
    q = fma2(t, q, pair(1.034736942e-01f));
    q = fma2(t, q, pair(1.224586845e-01f));
    q = fma2(t, q, pair(1.216402452e-01f));
    return q * t * e;
}

// The activations, of whole arrays: the switch stands outside the loops (inside, it took as long as the rest of the epilogue), and the
// arithmetic is on pairs, since the epilogue is bound by instructions.  gelu(v) = max(v, 0) - |v| T(|v|), without branches.
template <int N>
__device__ __forceinline__ void apply_act(int act, float (&v)[N])
{
    if (act == COBALT_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];              // a NaN stays
    } else if (act == COBALT_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= fast_sigmoid(v[i]);
    } else if (act == COBALT_ACT_GELU) {
        constexpr int kStep = N > 1 ? 2 : 1;
#pragma unroll
        for (int i = 0; i < N; i += kStep) {
            // (|v| held finite: infinity times 0 below)
            const Pair a = pair(fminf(fabsf(v[i]), 1e4f), fminf(fabsf(v[i + kStep - 1]), 1e4f));
            const Pair r = fma2(a * pair(-1.0f), normal_tail(a),
                                pair(v[i] < 0.0f ? 0.0f : v[i], v[i + kStep - 1] < 0.0f ? 0.0f : v[i + kStep - 1]));
            v[i] = r.v.x;
            v[i + kStep - 1] = r.v.y;
        }
    }
}

// d times the activation's slope at v, for a bf16 result.  gelu's slope is Phi(v) + v phi(v), Phi by 7.1.26 of the same Handbook with its own
// coefficients (t's is that of |v| here): good to 7.5e-8, and in the tail, where v phi(v) is nearly all of it, to 2.2e-4 of the slope, a
// twentieth of bf16's half step.
template <int N>
__device__ __forceinline__ void apply_slope(int act, const float (&v)[N], float (&d)[N])
{
    if (act == COBALT_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) d[i] *= v[i] > 0.0f ? 1.0f : 0.0f;
    } else if (act == COBALT_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = fast_sigmoid(v[i]);
            d[i] *= s * fmaf(v[i], 1.0f - s, 1.0f);
        }
    } else if (act == COBALT_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float t = fast_inverse(fmaf(0.3275911f * 0.70710678118654752f, fabsf(v[i]), 1.0f)), e = fast_exp2(-0.5f * kLog2E * v[i] * v[i]);
            float q = fmaf(t, 1.061405429f, -1.453152027f);
            q = fmaf(t, q, 1.421413741f);
            q = fmaf(t, q, -0.284496736f);
            q = fmaf(t, q, 0.254829592f);
            q *= 0.5f * t * e;
            d[i] *= fmaf(v[i] * 0.39894228040143268f, e, v[i] > 0.0f ? 1.0f - q : q);
        }
    }
}

// Eight neighbouring values to bf16 or fp32 memory.
__device__ __forceinline__ void store8(void* p, int64_t at, bool f32, const float (&v)[8])
{
    if (f32) {
        const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
        *reinterpret_cast<uint4*>(static_cast<float*>(p) + at) = Vec16<float>::pack(a);
        *reinterpret_cast<uint4*>(static_cast<float*>(p) + at + 4) = Vec16<float>::pack(b);
    } else {
        *reinterpret_cast<uint4*>(static_cast<bf16*>(p) + at) = Vec16<bf16>::pack(v);
    }
}

// What the epilogue needs of eight features, whatever the token.
struct FeatureConstants {
    float bias[8], scale[8];
    __device__ __forceinline__ void load(const Finish& f, int i0, bool mine)
    {
#pragma unroll
        for (int k = 0; k < 8; ++k) bias[k] = 0.0f, scale[k] = 1.0f;
        if (mine && f.bias) Vec16<bf16>::unpack(__ldg(reinterpret_cast<const uint4*>(f.bias + i0)), bias);
        if (mine && f.w_scales) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(f.w_scales + i0)), b = __ldg(reinterpret_cast<const float4*>(f.w_scales + i0 + 4));
            scale[0] = a.x, scale[1] = a.y, scale[2] = a.z, scale[3] = a.w;
            scale[4] = b.x, scale[5] = b.y, scale[6] = b.z, scale[7] = b.w;
        }
    }
};

// The residual of eight features, fetched ahead of their sums.
struct Residual8 {
    uint4 a, b;
    __device__ __forceinline__ void load(const LinearArgs& p, int64_t j, int i0, bool mine)
    {
        a = b = make_uint4(0, 0, 0, 0);
        if (!mine || !p.finish.residual) return;
        const int64_t at = j * p.I + i0;
        a = ld_once16(static_cast<const uint8_t*>(p.finish.residual) + at * (p.finish.f32 ? 4 : 2));
        if (p.finish.f32) b = ld_once16(static_cast<const float*>(p.finish.residual) + at + 4);
    }
    __device__ __forceinline__ void add_to(const LinearArgs& p, float (&v)[8]) const
    {
        if (!p.finish.residual) return;
        float r[8];
        if (p.finish.f32) {
            float x[4], y[4];
            Vec16<float>::unpack(a, x);
            Vec16<float>::unpack(b, y);
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] = x[k], r[4 + k] = y[k];
        } else {
            Vec16<bf16>::unpack(a, r);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += r[k];
    }
};

// The result for features i0 .. i0 + 7 of token j from their sums.  All sixteen lanes of 128 features are here together
// (`mine` says which of them have a result).
template <int kProduct>
__device__ __forceinline__ void finish8(const LinearArgs& p, int64_t j, int i0, bool mine, const FeatureConstants& c, const Residual8& residual, float (&v)[8])
{
    const Finish& f = p.finish;
    const int64_t at = j * p.I + i0;
    if (kProduct == kForward || kProduct == kForwardE4M3) {
        if (kProduct == kForwardE4M3) {
            const float sx = mine ? __ldg(f.x_scales + j) : 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= sx * c.scale[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] += c.bias[k];
        if (f.pre_scales) {
            uint32_t most = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) most = abs_max(most, v[k]);
            if (!mine) most = 0;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, off));
            const GroupScale g = GroupScale::of<CodeI8>(most);
            if (mine) {
                uint32_t codes[2];
                encode_fast<CodeI8>(v, g, codes);            // pre is itself a rounded sum: a code at a border may go either way
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(f.pre) + at) = make_uint2(codes[0], codes[1]);
                if (i0 % kPackGroup == 0) f.pre_scales[j * ((p.I + kPackGroup - 1) / kPackGroup) + i0 / kPackGroup] = g.scale;
            }
        } else if (f.pre && mine) {
            store8(f.pre, at, false, v);
        }
        apply_act(f.act, v);
        residual.add_to(p, v);
        if (mine) store8(p.out, at, f.f32, v);
    } else if (mine) {
        store8(p.out, at, false, v);
    }
}

struct LinearTile {
    int i0, j0, split, first, blocks;    // first block of k, and how many
};

template <bool kStay>
__device__ __forceinline__ LinearTile linear_tile(const LinearArgs& p, int t)
{
    LinearTile r;
    if (kStay) {                         // all tiles of i for one j
        r.split = r.first = 0;
        r.j0 = t / p.m_tiles * p.n;
        r.i0 = t % p.m_tiles * kTileM;
        r.blocks = p.blocks;
        return r;
    }
    const int each = p.m_tiles * p.j_tiles;
    r.split = t / each;
    const int in = t - r.split * each, band = in / (kBand * p.m_tiles), high = min(kBand, p.j_tiles - band * kBand), at = in - band * kBand * p.m_tiles;
    r.j0 = (band * kBand + at % high) * p.n;
    r.i0 = at / high * kTileM;
    r.first = r.split * p.per_split;
    r.blocks = min(p.per_split, p.blocks - r.first);
    return r;
}

template <int kProduct, int kForm, bool kStay>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLinearThreads, 1)
linear_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
              const __grid_constant__ LinearArgs p)
{
    constexpr bool kAMn = kProduct == kGradRows || kProduct == kGradWeights, kBMn = kProduct == kGradWeights;
    constexpr int kStepK = kProduct == kForwardE4M3 ? kDeepBytes : kDeep;                // values of k in a block
    constexpr int kLongBlocks = kProduct == kGradWeights ? kTokenBlocks : kResultBlocks;
    extern __shared__ __align__(1024) uint8_t smem[];                    // the swizzle counts from 1024-byte boundaries
    const uint32_t base = smem_u32(smem), staging = base + kRing * kSlotBytes, bars = staging + kStaging;
    constexpr int kSlots = kStay ? kStayRing : kRing, kStride = kStay ? kHalfBytes : kSlotBytes;
    const uint32_t stay = base + kSlots * kStride;                       // kStay: the blocks of j's operand
    const uint32_t ready = bars, empty = bars + 8 * kSlots, acc_full = bars + 16 * kSlots, acc_empty = acc_full + 16, drain = acc_full + 32,
                   tmem_slot = acc_full + 40, stay_ready = acc_full + 48, stay_empty = acc_full + 56;
    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int i = 0; i < kSlots; ++i) {
            barrier_init(ready + 8 * i, 2);      // leading CTA: both CTAs' loads of the slot
            barrier_init(empty + 8 * i, 1);      // the products that read the slot are done
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(acc_full + 8 * i, 1);
            barrier_init(acc_empty + 8 * i, 16);  // leading CTA: eight epilogue warps of each CTA
        }
        barrier_init(drain, 1);
        barrier_init(stay_ready, 2);
        barrier_init(stay_empty, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_a);
        prefetch_map(&map_b);
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot, 512);
    tmem_fence_before();
    cluster_sync();
    tmem_fence_after();
    wait_for_prior_kernel();
    launch_dependents();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot) : "memory");

    // the tiles (kStay: all those of a j) are dealt round robin
    const int tiles = p.m_tiles * p.j_tiles * p.splits, pairs = gridDim.x >> 1, unit = kStay ? p.m_tiles : 1, first = (blockIdx.x >> 1) * unit;
    auto next = [&](int t) { return (t + 1) % unit != 0 ? t + 1 : t + 1 + (pairs - 1) * unit; };
    bool ok = true;                              // no wait has run out

    if (warp == 0) {
        // ---- loads of this CTA's halves --------------------------------------------------------------------
        const uint32_t pair_ready = peer_address(ready, 0);
        const uint64_t policy = policy_normal();
        const int half = p.n / 2;
        Ring ring;
        int64_t issued = 0;
        int changes = 0;                         // kStay: how often the operand that stays was loaded
        for (int t = first; t < tiles && ok; t = next(t)) {
            const LinearTile w = linear_tile<kStay>(p, t);
            // boxes wholly outside their tensor are left out: what is in the slot then only reaches results that are not stored
            const int i0 = w.i0 + static_cast<int>(rank) * 128, j0 = w.j0 + static_cast<int>(rank) * half;
            const int boxes_a = i0 >= p.I ? 0 : !kAMn || i0 + 64 >= p.I ? 1 : 2;
            const int boxes_b = j0 >= p.J ? 0 : kBMn ? min((half + 63) / 64, (p.J - j0 + 63) / 64) : 1;
            const uint32_t bytes_b = boxes_b * (kBMn ? kBoxBytes : half * kDeepBytes), bytes = boxes_a * (kAMn ? kBoxBytes : kHalfBytes) + (kStay ? 0 : bytes_b);
            if (kStay && t % unit == 0) {
                if (!(ok = barrier_wait(stay_empty, (changes & 1) ^ 1))) break;
                if (elect_one()) {
                    const uint32_t bar = peer_address(stay_ready, 0);
                    barrier_expect_cluster(bar, w.blocks * bytes_b);
                    for (int k = 0; k < w.blocks && boxes_b > 0; ++k) tma_load_2d(stay + k * kHalfBytes, &map_b, bar, policy, k * kStepK, j0);
                }
                __syncwarp();
                ++changes;
            }
            for (int k = w.first; k < w.first + w.blocks; ++k) {
                if (!(ok = barrier_wait(empty + 8 * ring.slot, ring.phase ^ 1))) break;
                const uint32_t bar = pair_ready + 8 * ring.slot, a = base + ring.slot * kStride, b = a + kHalfBytes;
                if (elect_one()) {
                    barrier_expect_cluster(bar, bytes);
                    if (kAMn) {
                        if (boxes_a > 0) tma_load_2d(a, &map_a, bar, policy, i0, k * kStepK);
                        if (boxes_a > 1) tma_load_2d(a + kBoxBytes, &map_a, bar, policy, i0 + 64, k * kStepK);
                    } else if (boxes_a > 0) {
                        tma_load_2d(a, &map_a, bar, policy, k * kStepK, i0);
                    }
                    if (kStay) {
                    } else if (kBMn) {
                        if (boxes_b > 0) tma_load_2d(b, &map_b, bar, policy, j0, k * kStepK);
                        if (boxes_b > 1) tma_load_2d(b + kBoxBytes, &map_b, bar, policy, j0 + 64, k * kStepK);
                    } else if (boxes_b > 0) {
                        tma_load_2d(b, &map_b, bar, policy, k * kStepK, j0);
                    }
                }
                __syncwarp();
                ring.next<kSlots>();
                ++issued;
            }
        }
        if (!ok) {
            // the copies in flight have to land before the pair's shared memory is given back: the leading CTA waits for
            // its last blocks, which the other CTA's copies count on too, and once more for a block that will not be
            // complete, for those of the other CTA that are further ahead
            if (lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
            if (rank == 0)
                for (int64_t i = issued > kSlots ? issued - kSlots : 0; i <= issued; ++i)
                    (void)barrier_wait(ready + 8 * static_cast<int>(i % kSlots), static_cast<uint32_t>(i / kSlots) & 1);
            if (kStay && rank == 0 && changes > 0) (void)barrier_wait(stay_ready, (changes - 1) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- products (leading CTA) ------------------------------------------------------------------------------
        Ring ring;
        int turn = 0;                            // accumulators used so far
        int changes = 0;
        const uint32_t idesc = kProduct == kForwardE4M3 ? instruction_descriptor_e4m3(p.n) : instruction_descriptor(p.n, kAMn, kBMn);
        for (int t = first; t < tiles && ok && rank == 0; t = next(t)) {
            const LinearTile w = linear_tile<kStay>(p, t);
            if (kStay && t % unit == 0) {
                if (!(ok = barrier_wait(stay_ready, changes & 1))) break;
                ++changes;
            }
            for (int k = 0; k < w.blocks && ok; ++turn) {
                const uint32_t acc = turn & 1, d = tmem + acc * 256;
                const int first_k = k, end = kForm == kLong ? min(w.blocks, k + kLongBlocks) : w.blocks;
                if (!(ok = barrier_wait(acc_empty + 8 * acc, ((turn >> 1) & 1) ^ 1))) break;
                tmem_fence_after();
                for (; k < end; ++k) {
                    const uint32_t a = base + ring.slot * kStride;
                    if (!(ok = barrier_wait(ready + 8 * ring.slot, ring.phase))) break;
                    tmem_fence_after();
                    if (elect_one()) {
                        // K-major: 32 bytes further in the swizzled row; MN-major: two 8-row groups
                        const uint64_t da = matrix_descriptor(a, kAMn ? kBoxBytes : 16, 1024), db = matrix_descriptor(kStay ? stay + k * kHalfBytes : a + kHalfBytes, kBMn ? kBoxBytes : 16, 1024);
                        constexpr uint32_t step_a = (kAMn ? 2048 : 32) >> 4, step_b = (kBMn ? 2048 : 32) >> 4;
#pragma unroll
                        for (uint32_t i = 0; i < 4; ++i) {
                            if (kProduct == kForwardE4M3) mma_pair_e4m3(d, da + i * step_a, db + i * step_b, idesc, k > first_k || i > 0);
                            else mma_pair(d, da + i * step_a, db + i * step_b, idesc, k > first_k || i > 0);
                        }
                        mma_commit_pair(empty + 8 * ring.slot);
                    }
                    __syncwarp();
                    ring.next<kSlots>();
                }
                if (ok) {
                    if (elect_one()) {
                        mma_commit_pair(acc_full + 8 * acc);
                        if (kStay && (t + 1) % unit == 0) mma_commit_pair(stay_empty);         // the last tile of this j
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok) {
            if (lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
            if (elect_one()) mma_commit_pair(drain);     // products in flight end before the tensor memory is freed
            (void)barrier_wait(drain, 0);
        }
        __syncwarp();
    } else {
        // ---- epilogue: two groups of four warps, each a quarter of the tensor memory lanes a warp, take 32 columns in turn ----------
        const int quarter = warp & 3, group = (warp - 2) >> 2, tid = (threadIdx.x - 64) & 127;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * quarter) << 16);
        int turn = 0, stored = 0;                // accumulators, and (kPlain) staging buffers of this group, used so far
        // one verdict for the eight warps: none is left alone at the barriers below
        auto accumulator = [&]() {
            ok = named_barrier_and(1, 256, barrier_wait(acc_full + 8 * (turn & 1), (turn >> 1) & 1));
            if (ok) tmem_fence_after();
            return ok;
        };
        auto release = [&]() {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_tmem(peer_address(acc_empty + 8 * (turn & 1), 0));
            ++turn;
        };
        for (int t = first; t < tiles; t = next(t)) {
            const LinearTile w = linear_tile<kStay>(p, t);
            const int i_cta = w.i0 + static_cast<int>(rank) * 128, i8 = i_cta + 8 * (tid & 15), columns = min(p.n, p.J - w.j0);
            const bool split = p.splits > 1;
            // 32 sums of one i: a split's part
            auto store_part = [&](int c, const float (&r)[32]) {
                const int i = i_cta + 32 * quarter + lane;
                if (i >= p.I) return;
                float* out = p.partial + (static_cast<int64_t>(w.split) * p.J + w.j0 + c) * p.I + i;
#pragma unroll
                for (int k = 0; k < 32; ++k)
                    if (c + k < columns) out[static_cast<int64_t>(k) * p.I] = r[k];
            };
            FeatureConstants constants;
            Residual8 residual[4];
            auto fetch_residual = [&](int c) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = c + 8 * i + (tid >> 4);
                    residual[i].load(p, w.j0 + j, i8, j < columns && i8 < p.I);
                }
            };
            auto finish = [&](int c, const float (&r)[32]) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t buf = staging + (2 * group + h) * kBuffer32, at = buf + (32 * quarter + lane) * 4;
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(at + k * kPitch32), "f"(r[16 * h + k]) : "memory");
                    named_barrier(2 + group, 128);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int col = 8 * i + (tid >> 4);
                        const uint4 lo = load_shared16(buf + col * kPitch32 + (tid & 15) * 32), hi = load_shared16(buf + col * kPitch32 + (tid & 15) * 32 + 16);
                        float v[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                                      __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
                        const int j = c + 16 * h + col;
                        finish8<kProduct>(p, w.j0 + j, i8, j < columns && i8 < p.I, constants, residual[2 * h + i], v);
                    }
                }
            };
            if constexpr (kForm == kLong) {
                float sum[4][32] = {};
                for (int k = 0; k < w.blocks; k += kLongBlocks) {
                    if (!accumulator()) break;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = 64 * q + 32 * group;
                        if (c >= columns) break;
                        uint32_t r[32];
                        tmem_fetch_32x32(lanes + (turn & 1) * 256 + c, r);
                        tmem_wait(r);
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[q][i] += __uint_as_float(r[i]);
                    }
                    release();
                }
                if (!ok) break;
                if (!split) constants.load(p.finish, i8, i8 < p.I);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = 64 * q + 32 * group;
                    if (c >= columns) break;
                    if (split) {
                        store_part(c, sum[q]);
                    } else {
                        fetch_residual(c);
                        finish(c, sum[q]);
                    }
                }
            } else if (kForm == kFull || split) {
                if (!split) {
                    constants.load(p.finish, i8, i8 < p.I);
                    fetch_residual(32 * group);
                }
                if (!accumulator()) break;
                for (int c = 32 * group; c < columns; c += 64) {
                    uint32_t raw[32];
                    float r[32];
                    tmem_fetch_32x32(lanes + (turn & 1) * 256 + c, raw);
                    tmem_wait(raw);
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = __uint_as_float(raw[i]);
                    if (split) {
                        store_part(c, r);
                    } else if (kForm == kFull) {
                        finish(c, r);
                        fetch_residual(c + 64);
                    }
                }
                release();
            } else {
                // the elementwise part on the accumulators where they are, and the result leaves by tensor-map stores (stores by the threads
                // took half of the epilogue's time): a lane has four i (16 hl + 8 o + lane / 4) and pairs of j
                constexpr bool kElementwise = kProduct == kForward || kProduct == kForwardE4M3;
                float bias[4] = {}, scale[4] = {1.0f, 1.0f, 1.0f, 1.0f};
                if (kElementwise) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int i = i_cta + 32 * quarter + 8 * q + (lane >> 2);
                        if (p.finish.bias && i < p.I) bias[q] = __bfloat162float(p.finish.bias[i]);
                        if (kProduct == kForwardE4M3 && i < p.I) scale[q] = __ldg(p.finish.w_scales + i);
                    }
                }
                float sx[8];
                auto token_scales = [&](int c) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = c + 8 * (i >> 1) + 2 * (lane & 3) + (i & 1);
                        sx[i] = j < columns ? __ldg(p.finish.x_scales + w.j0 + j) : 0.0f;
                    }
                };
                if (kProduct == kForwardE4M3) token_scales(32 * group);
                if (!accumulator()) break;
                // the next chunk's accumulators and scales are on their way while this one is stored.  The four chunks are unrolled: what
                // is fetched stays in its registers up to the wait.  (Columns past the tile's are fetched and not used.)
                uint32_t r[2][16];
                auto fetch = [&](int c) {
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl) tmem_fetch_16x32(lanes + (static_cast<uint32_t>(16 * hl) << 16) + (turn & 1) * 256 + c, r[hl]);
                };
                fetch(32 * group);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = 64 * q + 32 * group;
                    const uint32_t buf = staging + (2 * group + (stored & 1)) * kBuffer16;
                    tmem_wait(r[0]);
                    tmem_wait(r[1]);
                    if (c >= columns) break;
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl) {
#pragma unroll
                        for (int o = 0; o < 2; ++o) {
                            float e[8];
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                e[i] = __uint_as_float(r[hl][4 * (i >> 1) + 2 * o + (i & 1)]);
                            }
                            if (kElementwise) {
#pragma unroll
                                for (int i = 0; i < 8; i += 2) {
                                    Pair u = pair(e[i], e[i + 1]);
                                    if (kProduct == kForwardE4M3) u = fma2(u, pair(sx[i], sx[i + 1]) * pair(scale[2 * hl + o]), pair(bias[2 * hl + o]));
                                    else u = u + pair(bias[2 * hl + o]);
                                    e[i] = u.v.x, e[i + 1] = u.v.y;
                                }
                            }
                            if (kElementwise) apply_act(p.finish.act, e);
                            const uint32_t at = 64 * quarter + 32 * hl + 16 * o;         // bytes into the 128 values
                            stmatrix_x4_trans(buf + (at >> 7) * kBox16 + lane * 128 + ((at & 127) ^ ((lane & 7) << 4)), pack2(e[0], e[1]),
                                              pack2(e[2], e[3]), pack2(e[4], e[5]), pack2(e[6], e[7]));
                        }
                    }
                    if (q < 3) {
                        fetch(c + 64);
                        if (kProduct == kForwardE4M3) token_scales(c + 64);
                    }
                    fence_async_shared();
                    if (tid == 0) store_groups_read();       // the other buffer, which is written next
                    named_barrier(2 + group, 128);
                    ++stored;                                // (a tile may have an odd number of chunks)
                    if (tid == 0 && i_cta < p.I) {
                        tma_store_2d(&map_out, buf, i_cta, w.j0 + c);
                        if (i_cta + 64 < p.I) tma_store_2d(&map_out, buf + kBox16, i_cta + 64, w.j0 + c);
                        store_group_end();
                    }
                }
                release();
            }
        }
        if (kForm == kPlain && tid == 0) store_groups_done();
        if (!ok && lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
        __syncwarp();
    }
    tmem_fence_before();
    cluster_sync();                              // no CTA leaves while the other may still reach its barriers
    tmem_fence_after();
    if (warp == 1) tmem_free_pair(tmem, 512);
}

// Adds the parts of a split product in order and finishes: eight neighbouring i of one j a thread, sixteen lanes 128 of i.
template <int kProduct>
__global__ void __launch_bounds__(256)
linear_join_kernel(const __grid_constant__ LinearArgs p)
{
    wait_for_prior_kernel();
    launch_dependents();
    const int per_row = (p.I + 127) / 128 * 16;
    const int64_t index = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, j = index / per_row;
    const int i8 = static_cast<int>(index - j * per_row) * 8;
    const bool mine = j < p.J && i8 < p.I;
    FeatureConstants constants;
    Residual8 residual = {};
    if (kProduct == kForward || kProduct == kForwardE4M3) {
        constants.load(p.finish, i8, mine);
        residual.load(p, j, i8, mine);
    }
    float v[8] = {};
    if (mine) {
        const float* from = p.partial + j * p.I + i8;
        const int64_t stride = static_cast<int64_t>(p.J) * p.I;
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            float a[4], b[4];
            Vec16<float>::unpack(ld_once16(from + s * stride), a);
            Vec16<float>::unpack(ld_once16(from + s * stride + 4), b);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] += a[k], v[4 + k] += b[k];
        }
    }
    finish8<kProduct>(p, j, i8, mine, constants, residual, v);
}

// ---- a few rows ---------------------------------------------------------------------------------------------------

constexpr int kFewThreads = 256;

// CTAs an SM that fit, by the registers of the kernel's launch bounds.
constexpr int few_resident(int rows) { return rows < 4 ? 4 : 3; }

// Sixteen bytes of an operand's row as pairs of 16-bit floats: eight bf16 values, or sixteen e4m3 ones, which are exact in fp16.
template <bool kE4M3>
struct OperandVec {
    static constexpr int kElems = kE4M3 ? 16 : 8;
    uint32_t h[kElems / 2];
    __device__ __forceinline__ OperandVec() {}
    __device__ __forceinline__ explicit OperandVec(const uint4& v)
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kE4M3) h[2 * i] = CodeE4M3::half2_bits(w[i]), h[2 * i + 1] = CodeE4M3::half2_bits(w[i] >> 16);
            else h[i] = w[i];
        }
    }
    // sum[0] and sum[1]: of the even and of the odd columns' products, which are exact in fp32
    __device__ __forceinline__ void dot(const OperandVec& b, float (&sum)[2]) const
    {
#pragma unroll
        for (int i = 0; i < kElems / 2; ++i) {
            if constexpr (kE4M3)
                asm("{\n\t.reg .b16 a, b, c, d;\n\tmov.b32 {a, b}, %2;\n\tmov.b32 {c, d}, %3;\n\t"
                    "fma.rn.f32.f16 %0, a, c, %0;\n\tfma.rn.f32.f16 %1, b, d, %1;\n\t}"
                    : "+f"(sum[0]), "+f"(sum[1]) : "r"(h[i]), "r"(b.h[i]));
            else
                asm("{\n\t.reg .b16 a, b, c, d;\n\tmov.b32 {a, b}, %2;\n\tmov.b32 {c, d}, %3;\n\t"
                    "fma.rn.f32.bf16 %0, a, c, %0;\n\tfma.rn.f32.bf16 %1, b, d, %1;\n\t}"
                    : "+f"(sum[0]), "+f"(sum[1]) : "r"(h[i]), "r"(b.h[i]));
        }
    }
};

// Up to R tokens on the fp32 units: `share` warps (1, 2, 4 or 8 of a CTA's eight) take one feature, its row of W once and the tokens'
// rows from L1, and add their sums in order.  Persistent CTAs; the next feature's first vectors are under way while one is summed up.
// Every vector index is clamped to the row, so that no address lies outside it.  The products of 16-bit floats are added to fp32 sums by one
// instruction (one token, 7168 to 2048 bf16 6.8 us; with the values converted to fp32 first 8.3).  kStaged: the tokens' e4m3 values are
// decoded once a CTA, to fp16 in shared memory (sixteen bytes of either half of a vector together: neighbouring lanes read neighbouring
// ones), since decoding bounds that form (7168 to 16384 23.9 us, 30.6 with every feature's own decoding, four tokens of 512 9.7 and 10.6).
template <bool kE4M3, int R, bool kStaged>
__global__ void __launch_bounds__(kFewThreads, few_resident(R))
linear_few_rows_kernel(const uint8_t* __restrict__ x, const uint8_t* __restrict__ w, int T, int K, int N, int share, void* out, const Finish f)
{
    constexpr int kAhead = 4, kElems = OperandVec<kE4M3>::kElems;        // vectors of W that a lane has in flight
    __shared__ float sums[2][kFewThreads / 32][R];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % share, vecs = K / kElems, each = 8 / share;
    const int tasks = (N + each - 1) / each, stride = 32 * kAhead * share, start = 32 * kAhead * part;
    wait_for_prior_kernel();
    launch_dependents();
    uint4 next[kAhead];
    auto load = [&](int task, int base) {
        const uint8_t* row = w + static_cast<int64_t>(min(task * each + warp / share, N - 1)) * vecs * 16;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = ld_stream16(row + 16 * static_cast<int64_t>(min(base + 32 * i + lane, vecs - 1)));
    };
    load(blockIdx.x, start);
    extern __shared__ uint4 staged[];            // [R][2][vecs]
    if constexpr (kStaged) {
        for (int v = threadIdx.x; v < R * vecs; v += kFewThreads) {
            const int r = v / vecs, at = v - r * vecs;
            const OperandVec<kE4M3> b(__ldg(reinterpret_cast<const uint4*>(x) + static_cast<int64_t>(min(r, T - 1)) * vecs + at));
#pragma unroll
            for (int c = 0; c < 2; ++c) staged[(2 * r + c) * vecs + at] = make_uint4(b.h[4 * c], b.h[4 * c + 1], b.h[4 * c + 2], b.h[4 * c + 3]);
        }
        __syncthreads();
    }
    for (int task = blockIdx.x, turn = 0; task < tasks; task += gridDim.x, turn ^= 1) {
        float sum[R][2] = {};
        int base = start;
        do {
            uint4 now[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) now[i] = next[i];
            // the next vectors, or the first ones of the next task
            const bool last = base + stride >= vecs;
            if (!last || task + gridDim.x < tasks) load(last ? task + gridDim.x : task, last ? start : base + stride);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int v = base + 32 * i + lane;
                if (v >= vecs) continue;
                const OperandVec<kE4M3> a(now[i]);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if constexpr (kStaged) {
                        OperandVec<kE4M3> b;
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const uint4 u = staged[(2 * r + c) * vecs + v];
                            b.h[4 * c] = u.x, b.h[4 * c + 1] = u.y, b.h[4 * c + 2] = u.z, b.h[4 * c + 3] = u.w;
                        }
                        a.dot(b, sum[r]);
                    } else {
                        const int token = R == 1 ? 0 : min(r, T - 1);
                        a.dot(OperandVec<kE4M3>(__ldg(reinterpret_cast<const uint4*>(x + (static_cast<int64_t>(token) * vecs + v) * 16))), sum[r]);
                    }
                }
            }
            base += stride;
        } while (base < vecs);
        float total[R];
#pragma unroll
        for (int r = 0; r < R; ++r) total[r] = warp_sum(sum[r][0] + sum[r][1]);
        if (lane == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r) sums[turn][warp][r] = total[r];
        }
        __syncthreads();
        // one thread a result
        const int i = task * each + threadIdx.x / R, t = threadIdx.x % R;
        if (threadIdx.x >= each * R || i >= N || t >= T) continue;
        float v[1] = {0.0f};
        for (int k = 0; k < share; ++k) v[0] += sums[turn][threadIdx.x / R * share + k][t];
        const int64_t at = static_cast<int64_t>(t) * N + i;
        if (kE4M3) v[0] *= __ldg(f.x_scales + t) * __ldg(f.w_scales + i);
        if (f.bias) v[0] += __bfloat162float(f.bias[i]);
        if (f.pre) static_cast<bf16*>(f.pre)[at] = __float2bfloat16_rn(v[0]);
        apply_act(f.act, v);
        if (f.f32) {
            if (f.residual) v[0] += static_cast<const float*>(f.residual)[at];
            static_cast<float*>(out)[at] = v[0];
        } else {
            if (f.residual) v[0] += __bfloat162float(static_cast<const bf16*>(f.residual)[at]);
            static_cast<bf16*>(out)[at] = __float2bfloat16_rn(v[0]);
        }
    }
}

// d = dout act'(pre) in bf16 (where the products need it) and its column sums: a CTA has 128 features and a slice of the
// tokens, 16 at a time; the sums of its sixteen token rows are added in order and written to partial [gridDim.y][N].
struct GradPreArgs {
    const void* grad_out;
    const void* pre;                     // or null
    const float* pre_scales;             // pre in 8 bits
    int64_t T;
    int N, act, f32;
    bf16* grad_pre;                      // or null
    float* partial;                      // or null
};

__global__ void __launch_bounds__(256, kGradPreCtas)
linear_grad_pre_kernel(const GradPreArgs p)
{
    constexpr int kAhead = kGradPreAhead;
    __shared__ float sums[16][128];
    wait_for_prior_kernel();
    launch_dependents();
    const int i8 = (blockIdx.x * 16 + (threadIdx.x & 15)) * 8, own = threadIdx.x >> 4, groups = (p.N + kPackGroup - 1) / kPackGroup;
    const int64_t step = static_cast<int64_t>(gridDim.y) * 16 * kAhead;
    float total[8] = {};
    if (i8 < p.N) {
        for (int64_t t0 = static_cast<int64_t>(blockIdx.y) * 16 * kAhead + own; t0 < p.T; t0 += step) {
            uint4 d16[kAhead], d32[kAhead], v16[kAhead];
            float scale[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int64_t t = t0 + 16 * a, at = t * p.N + i8;
                d16[a] = d32[a] = v16[a] = make_uint4(0, 0, 0, 0);
                scale[a] = 0.0f;
                if (t >= p.T) continue;
                d16[a] = ld_once16(static_cast<const uint8_t*>(p.grad_out) + at * (p.f32 ? 4 : 2));
                if (p.f32) d32[a] = ld_once16(static_cast<const float*>(p.grad_out) + at + 4);
                if (p.act == COBALT_ACT_NONE) continue;
                if (p.pre_scales) {
                    const uint2 codes = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(p.pre) + at));
                    v16[a].x = codes.x, v16[a].y = codes.y;
                    scale[a] = __ldg(p.pre_scales + t * groups + blockIdx.x);
                } else {
                    v16[a] = ld_once16(static_cast<const bf16*>(p.pre) + at);
                }
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int64_t t = t0 + 16 * a;
                if (t >= p.T) break;
                float d[8];
                if (p.f32) {
                    float x[4], y[4];
                    Vec16<float>::unpack(d16[a], x);
                    Vec16<float>::unpack(d32[a], y);
#pragma unroll
                    for (int k = 0; k < 4; ++k) d[k] = x[k], d[4 + k] = y[k];
                } else {
                    Vec16<bf16>::unpack(d16[a], d);
                }
                if (p.act != COBALT_ACT_NONE) {
                    float v[8];
                    if (p.pre_scales) {
                        float x[4], y[4];
                        CodeI8::decode4_fp16(v16[a].x, x);
                        CodeI8::decode4_fp16(v16[a].y, y);
#pragma unroll
                        for (int k = 0; k < 4; ++k) v[k] = x[k] * scale[a], v[4 + k] = y[k] * scale[a];
                    } else {
                        Vec16<bf16>::unpack(v16[a], v);
                    }
                    apply_slope(p.act, v, d);
                }
                if (p.grad_pre) store8(p.grad_pre, t * p.N + i8, false, d);
#pragma unroll
                for (int k = 0; k < 8; ++k) total[k] += d[k];
            }
        }
    }
    if (!p.partial) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) sums[own][8 * (threadIdx.x & 15) + k] = total[k];
    __syncthreads();
    const int i = blockIdx.x * 128 + threadIdx.x;
    if (threadIdx.x < 128 && i < p.N) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += sums[r][threadIdx.x];
        p.partial[static_cast<int64_t>(blockIdx.y) * p.N + i] = s;
    }
}

// grad_bias: the parts' sums, 32 features a CTA, every warp a slice of the parts.
__global__ void __launch_bounds__(1024)
linear_bias_kernel(const float* partial, int parts, int N, bf16* __restrict__ grad_bias)
{
    __shared__ float slice[32][33];
    wait_for_prior_kernel();
    launch_dependents();
    const int lane = threadIdx.x & 31, own = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (i < N) {
#pragma unroll 8
        for (int k = own; k < parts; k += 32) s += partial[static_cast<int64_t>(k) * N + i];
    }
    slice[own][lane] = s;
    __syncthreads();
    if (own == 0 && i < N) {
        float total = 0.0f;
#pragma unroll
        for (int k = 0; k < 32; ++k) total += slice[k][lane];
        grad_bias[i] = __float2bfloat16_rn(total);
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------

static int check_linear(int64_t T, int32_t K, int32_t N, int deep_unit)
{
    if (T < 0 || K < 1 || N < 1) return COBALT_ERR_INVALID_ARG;
    if (T > (1ll << 31) - (1ll << 21) || K % deep_unit != 0 || N % 8 != 0 || K > COBALT_LINEAR_MAX_WIDTH || N > COBALT_LINEAR_MAX_WIDTH)
        return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

// May start while the kernel before it is at its end; every kernel here waits for that one before it touches memory.
template <typename... Params, typename... Args>
static int launch_after(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchAttribute attr;
    set_programmatic_launch(&attr, true);
    cudaLaunchConfig_t config = {};
    config.gridDim = grid;
    config.blockDim = block;
    config.dynamicSmemBytes = smem;
    config.stream = s;
    config.attrs = &attr;
    config.numAttrs = 1;
    COBALT_CUDA_TRY(cudaLaunchKernelEx(&config, kernel, args...));
    return COBALT_OK;
}

// a: [I, k] or, transposed, [k, I]; b: [J, k] or [k, J].
template <int kProduct, int kForm, bool kStay = false>
static int launch_product(const void* a, const void* b, int64_t I, int64_t J, int64_t k, LinearArgs p, void* workspace, cudaStream_t s)
{
    constexpr bool kAMn = kProduct == kGradRows || kProduct == kGradWeights, kBMn = kProduct == kGradWeights;
    constexpr int kBytes = kProduct == kForwardE4M3 ? 1 : 2, kStepK = kDeepBytes / kBytes;
    const int64_t blocks = deep_blocks(k, kStepK);
    LinearPlan plan = linear_plan(I, J, blocks);
    if (kStay) plan = {kTileN, 1, static_cast<int>(blocks)};
    p.I = static_cast<int>(I);
    p.J = static_cast<int>(J);
    p.n = plan.n;
    p.m_tiles = static_cast<int>((I + kTileM - 1) / kTileM);
    p.j_tiles = static_cast<int>((J + plan.n - 1) / plan.n);
    p.splits = plan.splits;
    p.blocks = static_cast<int>(blocks);
    p.per_split = plan.per_split;
    p.partial = static_cast<float*>(workspace);
    CUtensorMap map_a, map_b, map_out;
    COBALT_TRY(kAMn ? matrix_map(&map_a, a, k, I, 64, kDeep) : matrix_map(&map_a, a, I, k, kStepK, 128, kBytes));
    COBALT_TRY(kBMn ? matrix_map(&map_b, b, k, J, 64, kDeep) : matrix_map(&map_b, b, J, k, kStepK, plan.n / 2, kBytes));
    if (kForm == kPlain) COBALT_TRY(matrix_map(&map_out, p.out, J, I, 64, 32));
    else map_out = map_a;                    // not used
    const void* kernel = reinterpret_cast<const void*>(&linear_kernel<kProduct, kForm, kStay>);
    COBALT_TRY(ensure_kernel_attributes(kernel, kLinearSmem, false));
    int sms = 0;
    COBALT_TRY(sm_count(&sms));
    const int64_t tiles = static_cast<int64_t>(p.m_tiles) * p.j_tiles * p.splits, pairs = tiles < sms / 2 ? tiles : sms / 2;
    if (tiles >= (1ll << 31) - (1 << 16)) return COBALT_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(2 * (pairs < 1 ? 1 : pairs)));
    COBALT_TRY((launch_after(linear_kernel<kProduct, kForm, kStay>, grid, dim3(kLinearThreads), kLinearSmem, s, map_a, map_b, map_out, p)));
    if (p.splits == 1) return COBALT_OK;
    const int64_t threads = J * ((I + 127) / 128 * 16);
    return launch_after(linear_join_kernel<kProduct>, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, s, p);
}

// Calls that the fp32 units take: one token, and two to four while the products are few.  Measured (us, this form / tiles, bf16): two
// tokens, 7168 to 2048 9.0 / 10.8, 4096 to 8192 16.8 / 15.7; four, 2048 to 1408 3.8 / 6.4, 2048 to 4096 9.2 / 8.2.
static bool few_rows(int64_t T, int32_t K, int32_t N) { return T == 1 || (T <= 4 && T * K * N <= (T == 2 ? 1ll << 25 : 1ll << 24)); }

template <bool kE4M3>
static int launch_few_rows(const void* x, const void* w, int T, int K, int N, void* out, const Finish& f, cudaStream_t s)
{
    // warps of a feature: more while there are fewer than 4096 warps and each has at least four vectors a lane
    const int vecs = K / OperandVec<kE4M3>::kElems;
    int share = 1;
    while (share < 8 && N * share < 4096 && vecs >= 256 * share) share *= 2;
    int sms = 0;
    COBALT_TRY(sm_count(&sms));
    const int tasks = (N + 8 / share - 1) / (8 / share), most = few_resident(T > 2 ? 4 : T) * sms;
    const dim3 grid(static_cast<unsigned>(tasks < most ? tasks : most)), block(kFewThreads);
    const uint8_t *a = static_cast<const uint8_t*>(x), *b = static_cast<const uint8_t*>(w);
    auto launch = [&](auto kernel, size_t smem) { return launch_after(kernel, grid, block, smem, s, a, b, T, K, N, share, out, f); };
    if constexpr (kE4M3) {
        // staged where the shared memory of an SM has room for it in all its CTAs
        const int rows = T > 2 ? 4 : T;
        const size_t smem = static_cast<size_t>(rows) * K * 2;
        if (smem <= static_cast<size_t>(220 / few_resident(rows)) * 1024) {
            auto kernel = rows == 1 ? linear_few_rows_kernel<true, 1, true> : rows == 2 ? linear_few_rows_kernel<true, 2, true> : linear_few_rows_kernel<true, 4, true>;
            COBALT_TRY(ensure_kernel_attributes(reinterpret_cast<const void*>(kernel), smem, false));
            return launch(kernel, smem);
        }
    }
    return T == 1 ? launch(linear_few_rows_kernel<kE4M3, 1, false>, 0)
                  : T == 2 ? launch(linear_few_rows_kernel<kE4M3, 2, false>, 0) : launch(linear_few_rows_kernel<kE4M3, 4, false>, 0);
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

size_t cobalt_linear_workspace_bytes(int64_t T, int32_t K, int32_t N)
{
    if (check_linear(T, K, N, 8) != COBALT_OK) return 0;
    return linear_workspace(T, K, N);
}

int cobalt_linear(const void* x, const float* x_scales, const void* w, const float* w_scales, const void* bias, const void* residual, int64_t T,
                  int32_t K, int32_t N, int32_t operand, int32_t act, int32_t out_type, void* pre, float* pre_scales, int32_t pre_type, void* out,
                  void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    if ((operand != COBALT_BF16 && operand != COBALT_E4M3) || (out_type != COBALT_BF16 && out_type != COBALT_F32) || act < COBALT_ACT_NONE ||
        act > COBALT_ACT_GELU || (pre && pre_type != COBALT_BF16 && pre_type != COBALT_I8))
        return COBALT_ERR_INVALID_ARG;
    const bool e4m3 = operand == COBALT_E4M3, pre8 = pre && pre_type == COBALT_I8;
    COBALT_TRY(check_linear(T, K, N, e4m3 ? 16 : 8));
    if (T == 0) return COBALT_OK;
    if (!x || !w || !out || (e4m3 && (!x_scales || !w_scales)) || (pre8 && !pre_scales)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned4(x_scales) || !aligned16(w) || !aligned16(w_scales) || !aligned16(bias) || !aligned16(residual) ||
        !aligned16(pre) || !aligned16(pre_scales) || !aligned16(out) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < linear_workspace(T, K, N)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    LinearArgs p = {};
    COBALT_TRY(device_error_word(&p.err_word));
    p.out = out;
    p.finish = {static_cast<const bf16*>(bias), residual, e4m3 ? x_scales : nullptr, e4m3 ? w_scales : nullptr, act, out_type == COBALT_F32, pre,
                pre8 ? pre_scales : nullptr};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (few_rows(T, K, N) && !pre8)
        return e4m3 ? launch_few_rows<true>(x, w, static_cast<int>(T), K, N, out, p.finish, s)
                    : launch_few_rows<false>(x, w, static_cast<int>(T), K, N, out, p.finish, s);
    const int form = out_type == COBALT_F32 ? kLong : residual || pre ? kFull : kPlain;
#define COBALT_LINEAR(FORM) \
    (e4m3 ? launch_product<kForwardE4M3, FORM>(w, x, N, T, K, p, workspace, s) : launch_product<kForward, FORM>(w, x, N, T, K, p, workspace, s))
    return form == kLong ? COBALT_LINEAR(kLong) : form == kFull ? COBALT_LINEAR(kFull) : COBALT_LINEAR(kPlain);
#undef COBALT_LINEAR
}

int cobalt_linear_backward(const void* grad_out, const void* x, const void* w, const void* pre, const float* pre_scales, int32_t pre_type,
                           int64_t T, int32_t K, int32_t N, int32_t act, int32_t grad_type, void* grad_pre, void* grad_x, void* grad_w,
                           void* grad_bias, void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    if ((grad_type != COBALT_BF16 && grad_type != COBALT_F32) || act < COBALT_ACT_NONE || act > COBALT_ACT_GELU ||
        (act != COBALT_ACT_NONE && pre_type != COBALT_BF16 && pre_type != COBALT_I8))
        return COBALT_ERR_INVALID_ARG;
    COBALT_TRY(check_linear(T, K, N, 8));
    const bool none = act == COBALT_ACT_NONE, pre8 = !none && pre_type == COBALT_I8, converts = !none || grad_type == COBALT_F32;
    const bool products = grad_x || grad_w;
    if (T > 0 && (!products && !grad_bias)) return COBALT_ERR_INVALID_ARG;
    if (T > 0 && (!grad_out || (grad_x && !w) || (grad_w && !x) || (!none && !pre) || (pre8 && !pre_scales) || (products && converts && !grad_pre)))
        return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_out) || !aligned16(x) || !aligned16(w) || !aligned16(pre) || !aligned16(pre_scales) || !aligned16(grad_pre) ||
        !aligned16(grad_x) || !aligned16(grad_w) || !aligned16(grad_bias) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    // (for the bias alone K is not known to a caller without x and w)
    if (!workspace || workspace_bytes < (products ? linear_workspace(T, K, N) : bias_bytes(T, N))) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (T == 0) {                                // no rows: the weights' gradients are 0
        if (grad_w) COBALT_CUDA_TRY(cudaMemsetAsync(grad_w, 0, static_cast<size_t>(N) * K * sizeof(bf16), s));
        if (grad_bias) COBALT_CUDA_TRY(cudaMemsetAsync(grad_bias, 0, static_cast<size_t>(N) * sizeof(bf16), s));
        return COBALT_OK;
    }
    LinearArgs p = {};
    COBALT_TRY(device_error_word(&p.err_word));
    const void* d = grad_out;
    if (grad_bias || (products && converts)) {
        GradPreArgs g = {grad_out, pre, pre8 ? pre_scales : nullptr, T, N, act, grad_type == COBALT_F32,
                         products && converts ? static_cast<bf16*>(grad_pre) : nullptr, grad_bias ? static_cast<float*>(workspace) : nullptr};
        const int parts = bias_parts(T, N);
        COBALT_TRY(launch_after(linear_grad_pre_kernel, dim3((N + 127) / 128, parts), dim3(256), 0, s, g));
        if (grad_bias)
            COBALT_TRY(launch_after(linear_bias_kernel, dim3((N + 31) / 32), dim3(1024), 0, s, static_cast<const float*>(g.partial), parts, N,
                                    static_cast<bf16*>(grad_bias)));
        if (converts) d = grad_pre;
    }
    if (grad_x) {
        p.out = grad_x;
        // the operand that stays is loaded once for all of i: where there are tiles enough for every pair to keep one for a while
        if (N <= kStayBlocks * kDeep && K >= 4 * kTileM && T >= 4 * kPlanPairs * kTileN)
            COBALT_TRY((launch_product<kGradRows, kPlain, true>(w, d, K, T, N, p, workspace, s)));
        else
            COBALT_TRY((launch_product<kGradRows, kPlain>(w, d, K, T, N, p, workspace, s)));
    }
    if (grad_w) {
        p.out = grad_w;
        const bool long_sum = linear_plan(K, N, deep_blocks(T, kDeep)).per_split > kTokenBlocks;
        COBALT_TRY((long_sum ? launch_product<kGradWeights, kLong>(x, d, K, N, T, p, workspace, s)
                             : launch_product<kGradWeights, kPlain>(x, d, K, N, T, p, workspace, s)));
    }
    return COBALT_OK;
}

}  // extern "C"
