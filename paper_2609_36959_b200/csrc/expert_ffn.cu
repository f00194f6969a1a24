// The experts between dispatch and combine: a gated feed-forward block over the rows of every slot, and its backward
// pass.  With x a row of slot d, e = slot_expert[d], Wg and Wu the two halves of w_gate_up[e], Wd = w_down[e]:
//
//   g = Wg x    u = Wu x    a = g s u, s = 1 / (1 + exp(-g))    y = Wd a
//   da = Wd^T dy    du = da g s    dg = da u s (1 + g (1 - s))    dx = Wg^T dg + Wu^T du
//   dWg = sum dg x^T    dWu = sum du x^T    dWd = sum dy a^T     over the rows of all slots that hold e
//
// Every step is a product on the tensor cores (tcgen05, bf16 operands, fp32 accumulators in tensor memory) with the
// elementwise part in its epilogue.  One kernel template serves the five products:
//
//   - A CTA pair computes a tile of 256 features (M: 128 a CTA) by up to 256 rows of one slot (N).  The weights are
//     the M side, so that a slot's ragged row count is the N extent of the instruction, a multiple of 32 chosen for
//     every tile: a slot of 40 rows costs 64, not 128 or 256, and a single token streams the weights once.
//     The weight gradients have features on both sides and the rows as the summed extent.
//   - Warp 0 of each CTA feeds a ring of 64-deep blocks by tensor-map loads, which the leading CTA's barriers count for
//     both; warp 1 of the leading CTA issues the products, warps 2 to 5 run the epilogue (and warp 6 clears the ragged ends
//     of slots for the weight gradients).
//     Two accumulators (2 x 256 of 512 columns) let the epilogue of a tile run under the products of the next one.
//   - CTAs are persistent, a pair for every two SMs, and deal the tiles of all slots round robin; the tile list is
//     built on the device from dest_offsets (no copy to the host).
//
// A call of a few rows (a token of generation) is bound by streaming the weights of their experts once; tiles leave SMs
// without work there, so each warp takes one feature of one row on the fp32 units instead (ffn_few_rows_kernel).
//
// Bound by the tensor pipe's energy in long runs (the 1000 W cap; 1150 to 1209 TFLOP/s at 65 536 rows, H 7168, F 2048, forward and
// backward, where cuBLAS holds 1340 to 1400 on one product of that shape), by the touched weights' bytes for few rows an
// expert (384 rows over 105 experts: 635 to 670 us, 90 to 96 % of copy speed).
//
// Every wait is bounded: when one runs out the kernel sets COBALT_DEVERR_WAIT_TIMEOUT, drains its copies, frees its
// tensor memory and returns.
#include <atomic>

#include "numeric.cuh"
#include "slot_ranges.h"
#include "tcgen05.cuh"

namespace cobalt {

typedef __nv_bfloat16 bf16;

// ---- tile lists ------------------------------------------------------------------------------------------------

constexpr int kTileM = 256;              // features of a pair
constexpr int kTileN = 256;              // most rows (or, for weight gradients, columns) of a tile
constexpr int kBlockK = 64;              // depth of one ring slot: 128 bytes, one swizzle row

// Workspace: header, row tiles, experts' segment lists.
struct PlanView {
    int32_t* row_tiles;                  // [1] number of row tiles
    int4* tile;                          // {first row, rows | expert's row tiles << 9, expert, expert's first tile}
    int32_t* seg_start;                  // [E + 1] into segs
    int32_t* expert_blocks;              // [E] 64-row blocks of the expert's rows
    int2* segs;                          // [D] {first row, rows}, slots in ascending order
};

__host__ __device__ inline int64_t max_row_tiles(int64_t P, int D) { return most_row_tiles(P, D, kTileN); }

static size_t plan_bytes(int64_t P, int D, int E)
{
    return 256 + round_up(16 * static_cast<size_t>(max_row_tiles(P, D)), 256) + round_up(4 * static_cast<size_t>(E + 1), 256) +
           round_up(4 * static_cast<size_t>(E), 256) + round_up(8 * static_cast<size_t>(D), 256);
}

static PlanView plan_view(void* workspace, int64_t P, int D, int E)
{
    PlanView v;
    char* p = static_cast<char*>(workspace);
    v.row_tiles = reinterpret_cast<int32_t*>(p);
    p += 256;
    v.tile = reinterpret_cast<int4*>(p);
    p += round_up(16 * static_cast<size_t>(max_row_tiles(P, D)), 256);
    v.seg_start = reinterpret_cast<int32_t*>(p);
    p += round_up(4 * static_cast<size_t>(E + 1), 256);
    v.expert_blocks = reinterpret_cast<int32_t*>(p);
    p += round_up(4 * static_cast<size_t>(E), 256);
    v.segs = reinterpret_cast<int2*>(p);
    return v;
}

constexpr int kPlanThreads = 1024;

// Exclusive prefix of v over the CTA; *total gets the sum.  `scratch`: 32 ints.
__device__ __forceinline__ int block_prefix(int v, int* scratch, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int o = __shfl_up_sync(0xFFFFFFFFu, s, off);
        if (lane >= off) s += o;
    }
    __syncthreads();                     // scratch of the previous call has been read
    if (lane == 31) scratch[warp] = s;
    __syncthreads();
    if (warp == 0) {
        int w = scratch[lane];
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xFFFFFFFFu, w, off);
            if (lane >= off) w += o;
        }
        scratch[lane] = w;
    }
    __syncthreads();
    *total = scratch[31];
    return s - v + (warp > 0 ? scratch[warp - 1] : 0);
}

// Shared memory of the plan kernel, in ints: five arrays by slot, four by expert, and per group of 32 * k consecutive
// slots (one a warp) the number of slots of every expert.
__host__ __device__ inline int plan_groups(int D) { return D <= kPlanThreads ? (D + 31) / 32 : kPlanThreads / 32; }
static size_t plan_smem(int D, int E) { return 4 * (5 * static_cast<size_t>(D) + 4 * static_cast<size_t>(E)) + 2 * static_cast<size_t>(plan_groups(D)) * E; }

// One CTA.  Offsets that decrease are read as their running maximum (disjoint slots: what bounds the tile list, and keeps
// two tiles from writing the same rows), those past P clamped, rows of a slot without a valid expert skipped; all flagged.
// The slots with rows are sorted by expert (counting sort, stable), and row tiles listed in that order, so that the
// slots of an expert's replicas share its weights in L2.
__global__ void __launch_bounds__(kPlanThreads)
ffn_plan_kernel(const uint32_t* __restrict__ offsets, const int32_t* __restrict__ slot_expert, int64_t P, int D, int E, PlanView out,
                uint32_t* __restrict__ err_word)
{
    launch_dependents();
    __shared__ int scratch[32];
    extern __shared__ int plan_shared[];
    int *s_first = plan_shared, *s_rows = s_first + D, *s_expert = s_rows + D, *s_rank = s_expert + D, *s_order = s_rank + D;
    int *e_tiles = s_order + D, *e_blocks = e_tiles + E, *e_start = e_blocks + E, *e_first = e_start + E;
    uint16_t* group_count = reinterpret_cast<uint16_t*>(e_first + E);      // [groups][E]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, groups = plan_groups(D), per_group = (D + groups - 1) / groups;
    const int span = (per_group + 31) / 32 * 32;                           // slots of a group

    for (int i = threadIdx.x; i < groups * E; i += kPlanThreads) group_count[i] = 0;
    for (int i = threadIdx.x; i < E; i += kPlanThreads) e_tiles[i] = e_blocks[i] = e_first[i] = 0;
    bool decreases = false;
    for (int d = threadIdx.x; d < D; d += kPlanThreads) {
        const int64_t a = offsets[d], b = offsets[d + 1];
        decreases |= b < a;
        const int64_t lo = a < P ? a : P, hi = b < P ? b : P;
        const int e = slot_expert[d];
        bool bad = b < a || b > P;
        int rows = hi > lo ? static_cast<int>(hi - lo) : 0;
        if (rows > 0 && (e < 0 || e >= E)) {
            bad = true;
            rows = 0;
        }
        if (bad) flag_error(err_word, COBALT_DEVERR_BAD_SLOT);
        s_first[d] = static_cast<int>(lo);
        s_rows[d] = rows;
        s_expert[d] = rows > 0 ? e : -1;
    }
    if (__syncthreads_or(decreases)) {                                     // one thread: no call in order comes here
        if (threadIdx.x == 0) {
            const int64_t end = offsets[D];
            make_slots_disjoint(D, static_cast<int32_t>(end < P ? end : P), s_first, s_rows, s_expert);
        }
        __syncthreads();
    }
    if (warp < groups) {
        for (int d0 = warp * span; d0 < min(D, (warp + 1) * span); d0 += 32) {
            const int d = d0 + lane, e = d < D ? s_expert[d] : -1;
            const uint32_t same = __match_any_sync(0xFFFFFFFFu, e);
            if (e >= 0) {
                const int before = group_count[warp * E + e], ahead = __popc(same & ((1u << lane) - 1u));
                s_rank[d] = before + ahead;
                atomicAdd(&e_tiles[e], (s_rows[d] + kTileN - 1) / kTileN);
                atomicAdd(&e_blocks[e], (s_rows[d] + kBlockK - 1) / kBlockK);
            }
            __syncwarp();
            if (e >= 0 && (same >> lane) == 1u) group_count[warp * E + e] += static_cast<uint16_t>(__popc(same));   // the last of its kind
            __syncwarp();
        }
    }
    __syncthreads();
    // E <= 1024: an expert a thread
    int slots = 0;
    if (threadIdx.x < E)
        for (int g = 0; g < groups; ++g) {
            const int n = group_count[g * E + threadIdx.x];
            group_count[g * E + threadIdx.x] = static_cast<uint16_t>(slots);
            slots += n;
        }
    int used;
    const int start = block_prefix(slots, scratch, &used);
    if (threadIdx.x < E) {
        e_start[threadIdx.x] = start;
        out.seg_start[threadIdx.x] = start;
        out.expert_blocks[threadIdx.x] = e_blocks[threadIdx.x];
    }
    if (threadIdx.x == 0) out.seg_start[E] = used;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += kPlanThreads) {
        const int e = s_expert[d];
        if (e >= 0) s_order[e_start[e] + group_count[(d / span) * E + e] + s_rank[d]] = d;
    }
    __syncthreads();
    int* s_tile = s_rank;                                                  // by sorted position from here on
    int tiles_before = 0;
    for (int base = 0; base < used; base += kPlanThreads) {
        const int i = base + threadIdx.x, d = i < used ? s_order[i] : 0;
        int total;
        const int at = tiles_before + block_prefix(i < used ? (s_rows[d] + kTileN - 1) / kTileN : 0, scratch, &total);
        if (i < used) {
            s_tile[i] = at;
            if (e_start[s_expert[d]] == i) e_first[s_expert[d]] = at;
            out.segs[i] = make_int2(s_first[d], s_rows[d]);
        }
        tiles_before += total;
    }
    if (threadIdx.x == 0) *out.row_tiles = tiles_before;
    __syncthreads();
    for (int i = warp; i < used; i += kPlanThreads / 32) {
        // the slot's rows in tiles of as equal a number of 32-row units as can be: tiles that share weights then take
        // the same time and stay together
        const int d = s_order[i], e = s_expert[d], rows = s_rows[d];
        const int n = (rows + kTileN - 1) / kTileN, units = (rows + 31) / 32, least = units / n, more = units - least * n;
        for (int k = lane; k < n; k += 32) {
            const int unit = k * least + min(k, more), own = least + (k < more), left = rows - 32 * unit;
            out.tile[s_tile[i] + k] = make_int4(s_first[d] + 32 * unit, min(left, 32 * own) | (e_tiles[e] << 9), e, e_first[e]);
        }
    }
}

// ---- the product kernel ------------------------------------------------------------------------------------------

enum Stage {
    kUp,             // act, pre   = rows     x w_gate_up^T   (gate and up features interleaved by eight along M)
    kDown,           // out        = act      x w_down^T
    kDownBackward,   // grad_pre   from grad_out x w_down
    kUpBackward,     // grad_rows  = grad_pre x w_gate_up
    kWeights         // a weight gradient: (M side)^T x (N side) over the rows
};

struct ProductArgs {
    PlanView plan;
    int P, E, M, N;          // rows; experts; features of the M side; columns of the N side (kWeights)
    int K;                   // summed extent (row stages)
    int F;                   // kUp, kDownBackward: columns of act
    bf16* out;               // kUp: act; kDown, kUpBackward, kWeights: the result; kDownBackward: grad_pre
    bf16* pre;               // kUp: pre or null
    const bf16* pre_in;      // kDownBackward (may be out)
    uint32_t* err_word;
};

template <int kStage>
constexpr int kProductThreads = kStage == 4 /* kWeights */ ? 224 : 192;
constexpr int kHalfBytes = 128 * kBlockK * 2;      // one operand of one CTA in a ring slot: 128 x 64 bf16
constexpr int kSlotBytes = 2 * kHalfBytes;
constexpr int kBoxBytes = 64 * kBlockK * 2;        // MN-major box: 64 values of M or N x 64 of k

template <int kStage>
struct Shape {
    static constexpr bool kWeightsStage = kStage == kWeights;
    static constexpr bool kAMn = kStage == kDownBackward || kStage == kUpBackward || kStage == kWeights;
    static constexpr int kRing = 6;
    // epilogue staging, pitches an odd number of 16-byte units: the eight rows of a matrix fall into different banks
    static constexpr int kPitch = kStage == kUp ? 144 : kStage == kDownBackward ? 528 : kStage == kWeights ? 144 : 272;
    static constexpr int kPlanes = kStage == kUp ? 3 : 1;                     // act, gate, up
    static constexpr int kBuffers = kStage == kUp || kStage == kDown || kStage == kUpBackward ? 2 : 1;
    static constexpr int kStaging = kStage == kWeights ? 4 * 32 * kPitch : kBuffers * kPlanes * 32 * kPitch;
    static constexpr int kBarriers = 256;
    static constexpr int kSmem = kRing * kSlotBytes + kStaging + kBarriers;
};

// Tiles of an expert run in bands of eight row tiles (kWeights: eight tiles of M), the other extent outside: the 74
// pairs at work then cover about 8 x 9 tiles and share both operands in L2.
constexpr int kBand = 8;

struct Tile {
    int expert, m0, n0, n;       // n: extent of the instruction's N (multiple of 32)
    int row0, rows;              // row stages
    int blocks;                  // 64-deep blocks of k
    int seg, seg_end;            // kWeights: the expert's segments
    int2 head;                   // kWeights: the first one
};

template <int kStage>
__device__ __forceinline__ int count_tiles(const ProductArgs& p)
{
    const int mt = (p.M + kTileM - 1) / kTileM;
    if (kStage == kWeights) return p.E * mt * ((p.N + kTileN - 1) / kTileN);
    return *p.plan.row_tiles * mt;
}

template <int kStage>
__device__ __forceinline__ Tile get_tile(const ProductArgs& p, int t)
{
    Tile r;
    const int mt = (p.M + kTileM - 1) / kTileM;
    if (kStage == kWeights) {
        const int nt = (p.N + kTileN - 1) / kTileN;
        r.expert = t / (mt * nt);
        const int in = t - r.expert * mt * nt, band = in / (kBand * nt), high = min(kBand, mt - band * kBand), at = in - band * kBand * nt;
        r.m0 = (band * kBand + at % high) * kTileM;
        r.n0 = at / high * kTileN;
        r.n = min(kTileN, (p.N - r.n0 + 31) / 32 * 32);
        r.row0 = r.rows = 0;
        r.blocks = p.plan.expert_blocks[r.expert];
        r.seg = p.plan.seg_start[r.expert];
        r.seg_end = p.plan.seg_start[r.expert + 1];
        r.head = r.blocks > 0 ? p.plan.segs[r.seg] : make_int2(0, 0);
    } else {
        // all entries between an expert's first and last tile carry its first tile and count
        const int4 any = p.plan.tile[t / mt];
        const int count = static_cast<int>(static_cast<uint32_t>(any.y) >> 9), in = t - any.w * mt;
        const int band = in / (kBand * mt), high = min(kBand, count - band * kBand), at = in - band * kBand * mt;
        const int4 own = p.plan.tile[any.w + band * kBand + at % high];
        r.expert = own.z;
        r.m0 = at / high * kTileM;
        r.n0 = 0;
        r.row0 = own.x;
        r.rows = own.y & 511;
        r.n = (r.rows + 31) / 32 * 32;
        r.blocks = (p.K + kBlockK - 1) / kBlockK;
        r.seg = r.seg_end = 0;
        r.head = make_int2(0, 0);
    }
    return r;
}

// Position in the ring: slot and the parity of its present use.
struct Ring {
    int slot = 0;
    uint32_t phase = 0;
    template <int kRing>
    __device__ __forceinline__ void next()
    {
        if (++slot == kRing) {
            slot = 0;
            phase ^= 1;
        }
    }
};

__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// The saved pre-activations are 16-bit floats of one sign, six exponent and nine mantissa bits: four times finer than
// bf16 (whose rounding here alone made the gradients of rows and weights 1.3 times as inexact as the two roundings that
// they cannot do without: 3.0e-3 against 2.4e-3 in the 2-norm), over 2^-30 .. 2^32, with gradual underflow to 2^-39.
// Larger finite values become the largest one; infinities and NaN stay (the largest exponent, with mantissa 0 and 1).
// Scaled by 2^-96, such a value is an fp32 number whose exponent fits six bits.
constexpr uint32_t kPreInf = 0x7E00u;

__device__ __forceinline__ uint32_t pack_pre(float lo, float hi)
{
    const float scale = __uint_as_float(0x0F800000u);                       // 2^-96
    const float most = __uint_as_float((62u << 23) | (0x1FFu << 14));
    float v[2] = {lo * scale, hi * scale};
    uint32_t c[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t sign = (__float_as_uint(v[i]) >> 16) & 0x8000u;
        const uint32_t b = __float_as_uint(fminf(fabsf(v[i]), most)) + 0x2000u;        // to nearest, halves up
        c[i] = sign | (fabsf(v[i]) < INFINITY ? b >> 14 : v[i] == v[i] ? kPreInf : kPreInf + 1);
    }
    return c[0] | (c[1] << 16);
}

__device__ __forceinline__ float unpack_pre(uint32_t code)                  // in the upper half of the word
{
    const float scale = __uint_as_float(0x6F800000u);                       // 2^96
    const uint32_t sign = code & 0x80000000u, magnitude = (code >> 2) & 0x1FFFC000u;
    const float v = __uint_as_float(magnitude | sign) * scale;
    // the largest exponent: fp32's largest, with the mantissa that there is
    return magnitude >= kPreInf << 14 ? __uint_as_float(sign | (0x7F800000u + (magnitude - (kPreInf << 14)))) : v;
}

// 1 / (1 + exp(-g)): the fast exponential and division are good to a few units of fp32, far below the bf16 results
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.0f, 1.0f + __expf(-g)); }

// Clears k rows valid .. 63 of this CTA's boxes in a ring slot (the loads brought rows of the next slot there).  The
// release that tells of it comes from one lane, behind the others' fences.
__device__ __forceinline__ void clear_tail(uint32_t slot_addr, int boxes_b, int valid, int lane)
{
    const int vectors = (kBlockK - valid) * 8;               // 16-byte vectors of a box
    for (int b = 0; b < 2 + boxes_b; ++b) {
        const uint32_t at = slot_addr + (b < 2 ? b * kBoxBytes : kHalfBytes + (b - 2) * kBoxBytes) + valid * 128;
        for (int i = lane; i < vectors; i += 32) store_shared16(at + i * 16, make_uint4(0, 0, 0, 0));
    }
    fence_async_shared();
    __syncwarp();
}

template <int kStage>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads<kStage>, 1)
ffn_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                   const __grid_constant__ CUtensorMap map_b_part, const __grid_constant__ ProductArgs p)
{
    typedef Shape<kStage> S;
    extern __shared__ __align__(1024) uint8_t smem[];                    // the swizzle counts from 1024-byte boundaries
    const uint32_t base = smem_u32(smem);
    const uint32_t staging = base + S::kRing * kSlotBytes;
    const uint32_t bars = staging + S::kStaging;
    const uint32_t ready = bars, empty = bars + 8 * S::kRing, landed = bars + 16 * S::kRing;
    const uint32_t acc_full = bars + 24 * S::kRing, acc_empty = acc_full + 16, drain = acc_full + 32, tmem_slot = acc_full + 40;
    const int warp = __shfl_sync(0xFFFFFFFFu, static_cast<int>(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kRing; ++i) {
            // leading CTA: the slot can be read.  Both CTAs' loads count on it themselves, so that what they brought is
            // ordered before the products; where a slot's end was cleared, the warp that cleared it arrives instead.
            barrier_init(ready + 8 * i, 2);
            barrier_init(empty + 8 * i, 1);      // the products that read the slot are done
            barrier_init(landed + 8 * i, 1);     // kWeights: this CTA's loads of a block with a slot's end
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(acc_full + 8 * i, 1);
            barrier_init(acc_empty + 8 * i, 8);  // leading CTA: four epilogue warps of each CTA
        }
        barrier_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        prefetch_map(&map_a);
        prefetch_map(&map_b);
    }
    if (warp == 1) tmem_alloc_pair(tmem_slot, 512);
    tmem_fence_before();
    cluster_sync();
    tmem_fence_after();
    wait_for_prior_kernel();                     // the plan, and what the kernel before wrote
    launch_dependents();
    uint32_t tmem;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(tmem_slot) : "memory");

    const int tiles = count_tiles<kStage>(p);
    const int first = blockIdx.x >> 1, step = gridDim.x >> 1;
    bool ok = true;                              // no wait has run out

    if (warp == 0) {
        // ---- loads of this CTA's halves --------------------------------------------------------------------
        const uint32_t pair_ready = peer_address(ready, 0);
        Ring ring;
        int64_t issued = 0;
        // a band reads its row tiles (kWeights: tiles of M) again for every tile of the other extent, and that one once
        const uint64_t once = policy_normal(), again = policy_evict_last();
        const uint64_t policy_a = S::kWeightsStage ? again : once, policy_b = S::kWeightsStage ? once : again;
        Tile next = {};
        if (first < tiles) next = get_tile<kStage>(p, first);
        for (int t = first; t < tiles && ok; t += step) {
            const Tile w = next;
            const int half = w.n / 2, m0 = w.m0 + static_cast<int>(rank) * 128;
            // Boxes wholly outside their tensor are left out: what is in the ring slot then only reaches features, columns or
            // rows of the tile that are not stored.
            const int n0 = w.n0 + static_cast<int>(rank) * half;                               // kWeights
            const int boxes_a = m0 >= p.M ? 0 : !S::kAMn || m0 + 64 >= p.M ? 1 : 2;
            const int boxes_b = n0 >= p.N ? 0 : min((half + 63) / 64, (p.N - n0 + 63) / 64);    // kWeights
            const int row0 = w.row0 + static_cast<int>(rank) * half;                           // row stages
            const int parts_b = min(half, (p.P - row0 + 15) / 16 * 16);                         // rows to load, by 16
            int seg = w.seg, done = 0;
            int2 rows = w.head;
            if (w.blocks == 0 && t + step < tiles) next = get_tile<kStage>(p, t + step);
            for (int k = 0; k < w.blocks; ++k) {
                // the list's loads are under way before the next tile needs them
                if (k == w.blocks / 2 && t + step < tiles) next = get_tile<kStage>(p, t + step);
                if (!(ok = barrier_wait(empty + 8 * ring.slot, ring.phase ^ 1))) break;
                const bool ends = kStage == kWeights && rows.y - done < kBlockK;     // a slot's rows end in this block
                const uint32_t bar = ends ? landed + 8 * ring.slot : pair_ready + 8 * ring.slot;
                const uint32_t a = base + ring.slot * kSlotBytes, b = a + kHalfBytes;
                if (elect_one()) {
                    if (kStage == kWeights) {
                        const uint32_t bytes = (boxes_a + boxes_b) * kBoxBytes;
                        if (ends) barrier_expect(bar, bytes);
                        else barrier_expect_cluster(bar, bytes);
                        if (boxes_a > 0) tma_load_2d(a, &map_a, bar, policy_a, m0, rows.x + done);
                        if (boxes_a > 1) tma_load_2d(a + kBoxBytes, &map_a, bar, policy_a, m0 + 64, rows.x + done);
                        if (boxes_b > 0) tma_load_2d(b, &map_b, bar, policy_b, n0, rows.x + done);
                        if (boxes_b > 1) tma_load_2d(b + kBoxBytes, &map_b, bar, policy_b, n0 + 64, rows.x + done);
                    } else {
                        barrier_expect_cluster(bar, boxes_a * (S::kAMn ? kBoxBytes : kHalfBytes) + max(parts_b, 0) * kBlockK * 2);
                        if (kStage == kUp && boxes_a > 0) tma_load_5d(a, &map_a, bar, policy_a, k * kBlockK, 0, 0, m0 / 16, w.expert);
                        if (kStage == kDown && boxes_a > 0) tma_load_3d(a, &map_a, bar, policy_a, k * kBlockK, m0, w.expert);
                        if (S::kAMn) {
                            if (boxes_a > 0) tma_load_3d(a, &map_a, bar, policy_a, m0, k * kBlockK, w.expert);
                            if (boxes_a > 1) tma_load_3d(a + kBoxBytes, &map_a, bar, policy_a, m0 + 64, k * kBlockK, w.expert);
                        }
                        if (parts_b == 128)
                            tma_load_2d(b, &map_b, bar, policy_b, k * kBlockK, row0);
                        else
                            for (int i = 0; i < parts_b; i += 16) tma_load_2d(b + i * 128, &map_b_part, bar, policy_b, k * kBlockK, row0 + i);
                    }
                }
                __syncwarp();
                ring.next<S::kRing>();
                ++issued;
                if (kStage == kWeights && (done += kBlockK) >= rows.y && ++seg < w.seg_end) {
                    rows = p.plan.segs[seg];
                    done = 0;
                }
            }
        }
        if (!ok) {
            // the copies in flight have to land before the pair's shared memory is given back: the leading CTA waits for
            // its last blocks, which the other CTA's copies count on too, and once more for a block that will not be
            // complete, for those of the other CTA that are further ahead (and for blocks with a slot's end)
            if (lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
            if (rank == 0)
                for (int64_t i = issued > S::kRing ? issued - S::kRing : 0; i <= issued; ++i)
                    (void)barrier_wait(ready + 8 * static_cast<int>(i % S::kRing), static_cast<uint32_t>(i / S::kRing) & 1);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- products (leading CTA) ------------------------------------------------------------------------------
        Ring ring;
        int turn = 0;                            // accumulators used so far
        const bool part = rank == 0;
        Tile next = {};
        if (part && first < tiles) next = get_tile<kStage>(p, first);
        for (int t = first; t < tiles && ok && part; t += step) {
            const Tile w = next;
            if (w.blocks == 0) {
                if (t + step < tiles) next = get_tile<kStage>(p, t + step);
                continue;
            }
            const uint32_t acc = turn & 1, d = tmem + acc * 256;
            const uint32_t idesc = instruction_descriptor(w.n, S::kAMn, S::kWeightsStage);
            if (!(ok = barrier_wait(acc_empty + 8 * acc, ((turn >> 1) & 1) ^ 1))) break;
            tmem_fence_after();
            for (int k = 0; k < w.blocks; ++k) {
                if (k == w.blocks / 2 && t + step < tiles) next = get_tile<kStage>(p, t + step);
                const uint32_t a = base + ring.slot * kSlotBytes;
                if (!(ok = barrier_wait(ready + 8 * ring.slot, ring.phase))) break;
                tmem_fence_after();
                if (elect_one()) {
                    // K-major: 16 values of k are 32 bytes further in the swizzled row; MN-major: two 8-row groups
                    const uint64_t da = S::kAMn ? matrix_descriptor(a, kBoxBytes, 1024) : matrix_descriptor(a, 16, 1024);
                    const uint64_t db = S::kWeightsStage ? matrix_descriptor(a + kHalfBytes, kBoxBytes, 1024)
                                                         : matrix_descriptor(a + kHalfBytes, 16, 1024);
                    constexpr uint32_t step_a = (S::kAMn ? 2048 : 32) >> 4, step_b = (S::kWeightsStage ? 2048 : 32) >> 4;
#pragma unroll
                    for (uint32_t i = 0; i < kBlockK / 16; ++i) mma_pair(d, da + i * step_a, db + i * step_b, idesc, k > 0 || i > 0);
                    mma_commit_pair(empty + 8 * ring.slot);
                }
                __syncwarp();
                ring.next<S::kRing>();
            }
            if (ok) {
                if (elect_one()) mma_commit_pair(acc_full + 8 * acc);
                __syncwarp();
            }
            ++turn;
        }
        if (!ok) {
            if (lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
            if (elect_one()) mma_commit_pair(drain);     // products in flight end before the tensor memory is freed
            (void)barrier_wait(drain, 0);
        }
        __syncwarp();
    } else if (S::kWeightsStage && warp == 6) {
        // ---- weight gradients: k rows past the end of a slot, which belong to the next one, are cleared here, ahead of
        // the products and off their path; then the leading CTA hears of the block
        Ring ring;
        uint32_t phases = 0;                     // of `landed`, a bit a slot: only blocks with a slot's end use it
        Tile next = {};
        if (first < tiles) next = get_tile<kStage>(p, first);
        const uint32_t pair_ready = peer_address(ready, 0);
        for (int t = first; t < tiles && ok; t += step) {
            const Tile w = next;
            if (w.blocks == 0 && t + step < tiles) next = get_tile<kStage>(p, t + step);
            const int boxes_b = (w.n / 2 + 63) / 64;
            int seg = w.seg, left = w.head.y;
            for (int k = 0; k < w.blocks; ++k) {
                if (k == w.blocks / 2 && t + step < tiles) next = get_tile<kStage>(p, t + step);
                if (left < kBlockK) {
                    if (!(ok = barrier_wait(landed + 8 * ring.slot, (phases >> ring.slot) & 1))) break;
                    phases ^= 1u << ring.slot;
                    clear_tail(base + ring.slot * kSlotBytes, boxes_b, left, lane);
                    if (elect_one()) barrier_arrive_cluster(pair_ready + 8 * ring.slot);
                    __syncwarp();
                }
                left -= kBlockK;
                if (left <= 0 && ++seg < w.seg_end) left = p.plan.segs[seg].y;
                ring.next<S::kRing>();
            }
        }
        if (!ok && lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
        __syncwarp();
    } else {
        // ---- epilogue: quarter of the tensor memory lanes by warp, 32 accumulator columns at a time ---------------
        const int quarter = warp & 3, tid = threadIdx.x - 64;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(32 * quarter) << 16);
        int turn = 0, chunk_turn = 0;
        for (int t = first; t < tiles && ok; t += step) {
            const Tile w = get_tile<kStage>(p, t);
            const uint32_t acc = turn & 1;
            if (w.blocks > 0 && kStage != kDownBackward) {
                // one verdict for the four warps: none is left alone at the barriers below
                ok = named_barrier_and(1, 128, barrier_wait(acc_full + 8 * acc, (turn >> 1) & 1));
                if (!ok) break;
                tmem_fence_after();
            }
            const int64_t F = p.F;
            if (kStage == kUp) {
                // TMEM lane 16 i + 8 j + l: gate (j = 0) or up (j = 1) feature 8 i + l, so both are in one thread
                const int f0 = w.m0 / 2 + static_cast<int>(rank) * 64;
                for (int c = 0; c < w.n; c += 32, ++chunk_turn) {
                    const uint32_t buf = staging + (chunk_turn & 1) * (S::kPlanes * 32 * S::kPitch);
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl) {
                        uint32_t r[16], a[4], g[4], u[4];
                        tmem_load_16x32(lanes + (static_cast<uint32_t>(16 * hl) << 16) + acc * 256 + c, r);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float g0 = __uint_as_float(r[4 * i]), g1 = __uint_as_float(r[4 * i + 1]);
                            const float u0 = __uint_as_float(r[4 * i + 2]), u1 = __uint_as_float(r[4 * i + 3]);
                            a[i] = pack2(g0 * sigmoid(g0) * u0, g1 * sigmoid(g1) * u1);
                            if (p.pre) {
                                g[i] = pack_pre(g0, g1);
                                u[i] = pack_pre(u0, u1);
                            }
                        }
                        const uint32_t at = buf + lane * S::kPitch + (16 * quarter + 8 * hl) * 2;
                        stmatrix_x4_trans(at, a[0], a[1], a[2], a[3]);
                        if (p.pre) {
                            stmatrix_x4_trans(at + 32 * S::kPitch, g[0], g[1], g[2], g[3]);
                            stmatrix_x4_trans(at + 64 * S::kPitch, u[0], u[1], u[2], u[3]);
                        }
                    }
                    named_barrier(1, 128);
                    const int v = tid & 7, f = f0 + 8 * v;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int tok = i * 16 + (tid >> 3);
                        if (c + tok < w.rows && f < F) {
                            const int64_t row = w.row0 + c + tok;
                            const uint32_t at = buf + tok * S::kPitch + v * 16;
                            *reinterpret_cast<uint4*>(p.out + row * F + f) = load_shared16(at);
                            if (p.pre) {
                                *reinterpret_cast<uint4*>(p.pre + row * 2 * F + f) = load_shared16(at + 32 * S::kPitch);
                                *reinterpret_cast<uint4*>(p.pre + row * 2 * F + F + f) = load_shared16(at + 64 * S::kPitch);
                            }
                        }
                    }
                }
            } else if (kStage == kDown || kStage == kUpBackward) {
                const int m0 = w.m0 + static_cast<int>(rank) * 128;
                for (int c = 0; c < w.n; c += 32, ++chunk_turn) {
                    const uint32_t buf = staging + (chunk_turn & 1) * (32 * S::kPitch);
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl) {
                        uint32_t r[16];
                        tmem_load_16x32(lanes + (static_cast<uint32_t>(16 * hl) << 16) + acc * 256 + c, r);
#pragma unroll
                        for (int o = 0; o < 2; ++o) {
                            uint32_t v[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                v[i] = pack2(__uint_as_float(r[4 * i + 2 * o]), __uint_as_float(r[4 * i + 2 * o + 1]));
                            stmatrix_x4_trans(buf + lane * S::kPitch + (32 * quarter + 16 * hl + 8 * o) * 2, v[0], v[1], v[2], v[3]);
                        }
                    }
                    named_barrier(1, 128);
                    const int v = tid & 15, m = m0 + 8 * v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int tok = i * 8 + (tid >> 4);
                        if (c + tok < w.rows && m < p.M)
                            *reinterpret_cast<uint4*>(p.out + static_cast<int64_t>(w.row0 + c + tok) * p.M + m) =
                                load_shared16(buf + tok * S::kPitch + v * 16);
                    }
                }
            } else if (kStage == kDownBackward) {
                const int f0 = w.m0 + static_cast<int>(rank) * 128;
                const int v = tid & 31, f = f0 + 8 * (v & 15);
                const int64_t col = (v < 16 ? 0 : F) + f;
                // gate and up come in by rows, a chunk ahead; each thread reads and later overwrites the same vectors
                uint4 x[8];
                auto fetch = [&](int c) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int tok = i * 4 + (tid >> 5);
                        x[i] = make_uint4(0, 0, 0, 0);
                        if (c + tok < w.rows && f < F) x[i] = ld_once16(p.pre_in + static_cast<int64_t>(w.row0 + c + tok) * 2 * F + col);
                    }
                };
                fetch(0);
                ok = named_barrier_and(1, 128, barrier_wait(acc_full + 8 * acc, (turn >> 1) & 1));
                if (!ok) break;
                tmem_fence_after();
                for (int c = 0; c < w.n; c += 32) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) store_shared16(staging + (i * 4 + (tid >> 5)) * S::kPitch + v * 16, x[i]);
                    if (c + 32 < w.n) fetch(c + 32);
                    named_barrier(1, 128);
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl) {
                        uint32_t r[16];
                        tmem_load_16x32(lanes + (static_cast<uint32_t>(16 * hl) << 16) + acc * 256 + c, r);
#pragma unroll
                        for (int o = 0; o < 2; ++o) {
                            const uint32_t at = staging + lane * S::kPitch + (32 * quarter + 16 * hl + 8 * o) * 2;
                            uint32_t gv[4], uv[4];
                            ldmatrix_x4_trans(at, gv);
                            ldmatrix_x4_trans(at + 256, uv);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float g0 = unpack_pre(gv[i] << 16), g1 = unpack_pre(gv[i]), u0 = unpack_pre(uv[i] << 16), u1 = unpack_pre(uv[i]);
                                const float d0 = __uint_as_float(r[4 * i + 2 * o]), d1 = __uint_as_float(r[4 * i + 2 * o + 1]);
                                const float s0 = sigmoid(g0), s1 = sigmoid(g1);
                                gv[i] = pack2(d0 * u0 * s0 * (1.0f + g0 * (1.0f - s0)), d1 * u1 * s1 * (1.0f + g1 * (1.0f - s1)));
                                uv[i] = pack2(d0 * g0 * s0, d1 * g1 * s1);
                            }
                            stmatrix_x4_trans(at, gv[0], gv[1], gv[2], gv[3]);
                            stmatrix_x4_trans(at + 256, uv[0], uv[1], uv[2], uv[3]);
                        }
                    }
                    named_barrier(1, 128);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int tok = i * 4 + (tid >> 5);
                        if (c + tok < w.rows && f < F)
                            st_stream16(p.out + static_cast<int64_t>(w.row0 + c + tok) * 2 * F + col,
                                        load_shared16(staging + tok * S::kPitch + v * 16));
                    }
                }
            } else {
                // weight gradients: TMEM lanes are rows of the result, columns its columns; a warp is on its own
                const int m0 = w.m0 + static_cast<int>(rank) * 128 + 32 * quarter;
                const uint32_t buf = staging + quarter * 32 * S::kPitch;
                bf16* out = p.out + static_cast<int64_t>(w.expert) * p.M * p.N;
                for (int c = 0; c < w.n; c += 64) {
                    const int parts = min(2, (w.n - c) / 32);
#pragma unroll
                    for (int hl = 0; hl < 2; ++hl)
                        for (int q = 0; q < parts; ++q) {
                            uint32_t r[16] = {};
                            if (w.blocks > 0) {
                                tmem_load_16x32(lanes + (static_cast<uint32_t>(16 * hl) << 16) + acc * 256 + c + 32 * q, r);
                            }
#pragma unroll
                            for (int o = 0; o < 2; ++o) {
                                uint32_t v[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    v[i] = pack2(__uint_as_float(r[4 * i + 2 * o]), __uint_as_float(r[4 * i + 2 * o + 1]));
                                stmatrix_x4(buf + (16 * hl + 8 * o + (lane & 7)) * S::kPitch + (32 * q + 8 * (lane >> 3)) * 2, v[0], v[1], v[2],
                                            v[3]);
                            }
                        }
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int m = i * 4 + (lane >> 3), n = w.n0 + c + 8 * (lane & 7);
                        if (m0 + m < p.M && n < p.N && 8 * (lane & 7) < 32 * parts)
                            st_stream16(out + static_cast<int64_t>(m0 + m) * p.N + n, load_shared16(buf + m * S::kPitch + (lane & 7) * 16));
                    }
                    __syncwarp();
                }
            }
            if (w.blocks > 0) {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive_tmem(peer_address(acc_empty + 8 * acc, 0));
                ++turn;
            }
        }
        if (!ok && lane == 0) flag_error(p.err_word, COBALT_DEVERR_WAIT_TIMEOUT);
        __syncwarp();
    }
    tmem_fence_before();
    cluster_sync();                              // no CTA leaves while the other may still reach its barriers
    tmem_fence_after();
    if (warp == 1) tmem_free_pair(tmem, 512);
}

// ---- a few rows ---------------------------------------------------------------------------------------------------

constexpr int kFewThreads = 256;
constexpr int kFewResident = 4;          // CTAs an SM
// Most rows of a call that takes this form.  Measured with every row at another expert (us, this form / tiles): H 7168, F 2048:
// 1 row 23 / 45, 6 rows 85 / 110, 8 rows 113 / 128; H 2048, F 1408: 6 rows 23.7 / 31.2, 8 rows 28.8 / 41.  Beyond, the tiles read a
// shared expert's weights once, this form once a row: 8 rows at one expert 84 / 45.
constexpr int kFewRows = 8;
constexpr int kFewVecs = 2048;           // longest summed extent, in 16-byte vectors: a row in shared memory

__device__ __forceinline__ float dot8(const uint4& w, const uint4& x, float acc)
{
    float a[8], b[8];
    Vec16<bf16>::unpack(w, a);
    Vec16<bf16>::unpack(x, b);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc = fmaf(a[i], b[i], acc);
    return acc;
}

// Expert of row p, -1 for none.  The row's slot is the first one that ends behind it, if the first slot starts no later:
// the plan's rule, offsets as their running maximum.  Bad ranges are flagged by one CTA, as in the plan.  The three loads of
// a slot are under way together.
__device__ __forceinline__ int expert_of_row(const uint32_t* offsets, const int32_t* slot_expert, int P, int D, int E, int p, bool check,
                                             uint32_t* err_word, int* found)
{
    if (threadIdx.x == 0) *found = 0x7FFFFFFF;
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += kFewThreads) {
        const uint32_t a = __ldg(offsets + d), b = __ldg(offsets + d + 1);
        const int e = __ldg(slot_expert + d);
        const bool valid = e >= 0 && e < E;
        // slot in the upper bits, so that the lowest one wins; expert + 1 below (E <= 1024), 0 for none
        if (d == 0 && a > static_cast<uint32_t>(p)) atomicMin(found, -1);      // ahead of the first slot
        if (static_cast<uint32_t>(p) < b) atomicMin(found, d << 12 | (valid ? e + 1 : 0));
        if (check) {
            const uint32_t n = static_cast<uint32_t>(P), lo = min(a, n), hi = min(b, n);
            if (b < a || b > n || (hi > lo && !valid)) flag_error(err_word, COBALT_DEVERR_BAD_SLOT);
        }
    }
    __syncthreads();
    return *found == 0x7FFFFFFF || *found < 0 ? -1 : (*found & 4095) - 1;
}

// kUp: act (and pre) of one row, a warp a feature: its gate and its up row of the weights.  kDown: out of one row, a warp
// two neighbouring features.  blockIdx.y is the row.  Summed in fp32, a lane 8 values of every 256.
template <int kStage>
__global__ void __launch_bounds__(kFewThreads, kFewResident)
ffn_few_rows_kernel(const bf16* x, const bf16* weights, const uint32_t* __restrict__ offsets,
                    const int32_t* __restrict__ slot_expert, int P, int D, int E, int M, int K, bf16* __restrict__ out,
                    bf16* __restrict__ pre, uint32_t* __restrict__ err_word)
{
    extern __shared__ __align__(16) uint4 x_row[];           // [K / 8]
    __shared__ int found;
    const int lane = threadIdx.x & 31, row = blockIdx.y, vecs = K / 8;
    const int tasks = kStage == kUp ? M : M / 2, step = gridDim.x * (kFewThreads / 32);
    if (kStage == kUp) launch_dependents();
    const int e = expert_of_row(offsets, slot_expert, P, D, E, row, kStage == kUp && blockIdx.x == 0 && row == 0, err_word, &found);
    if (e < 0) {                                              // a row of no slot (uniform over the CTA)
        if (kStage == kDown) wait_for_prior_kernel();         // this kernel ends after the one before it all the same
        return;
    }
    // Vectors of each weight row a lane has in flight.  Two, with four CTAs an SM in one wave, against four with two CTAs:
    // 6 rows, H 2048, F 1408 23.7 us against 26.6; 8 rows, H 7168, F 2048 the same 113 us.
    constexpr int kAhead = 2;
    uint4 a[kAhead], b[kAhead];
    // Two rows of the weights: gate and up of feature m, or features m and m + 1.  Task and vector are clamped, not
    // guarded: every address that is formed lies in the expert's weights (what a lane has too many counts as zero).
    auto load = [&](int task, int base) {
        const int own = min(task, tasks - 1);
        const int64_t m = kStage == kUp ? static_cast<int64_t>(e) * 2 * M + own : static_cast<int64_t>(e) * M + 2 * own;
        const bf16 *w0 = weights + m * K, *w1 = w0 + (kStage == kUp ? static_cast<int64_t>(M) : 1) * K;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int v = min(base + lane + 32 * i, vecs - 1);
            a[i] = ld_once16(w0 + 8 * v);
            b[i] = ld_once16(w1 + 8 * v);
        }
    };
    int task = blockIdx.x * (kFewThreads / 32) + (threadIdx.x >> 5);
    load(task, 0);
    if (kStage == kDown) wait_for_prior_kernel();             // x is what the kernel before writes; the weights are not
    for (int i = threadIdx.x; i < vecs; i += kFewThreads) x_row[i] = ld_once16(x + static_cast<int64_t>(row) * K + i * 8);
    __syncthreads();
    for (; task < tasks; task += step) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int base = 0; base < vecs; base += 32 * kAhead) {
            uint4 ca[kAhead], cb[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                ca[i] = a[i];
                cb[i] = b[i];
            }
            // the next vectors, or the first ones of the next task
            const bool last = base + 32 * kAhead >= vecs;
            if (!last || task + step < tasks) load(last ? task + step : task, last ? 0 : base + 32 * kAhead);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int v = base + lane + 32 * i;
                if (v < vecs) {
                    s0 = dot8(ca[i], x_row[v], s0);
                    s1 = dot8(cb[i], x_row[v], s1);
                }
            }
        }
        s0 = warp_sum(s0);
        s1 = warp_sum(s1);
        if (lane == 0) {
            if (kStage == kUp) {
                out[static_cast<int64_t>(row) * M + task] = __float2bfloat16_rn(s0 * sigmoid(s0) * s1);
                if (pre) {
                    const uint32_t both = pack_pre(s0, s1);
                    uint16_t* at = reinterpret_cast<uint16_t*>(pre) + static_cast<int64_t>(row) * 2 * M + task;
                    at[0] = static_cast<uint16_t>(both);
                    at[M] = static_cast<uint16_t>(both >> 16);
                }
            } else {                                          // (M is a multiple of 8)
                *reinterpret_cast<uint32_t*>(out + static_cast<int64_t>(row) * M + 2 * task) = pack2(s0, s1);
            }
        }
    }
}

// ---- host side ----------------------------------------------------------------------------------------------------

template <int kStage>
static int launch_few_rows(const void* x, const void* weights, const uint32_t* offsets, const int32_t* slot_expert, int P, int D, int E,
                           int M, int K, void* out, void* pre, uint32_t* err_word, cudaStream_t s)
{
    const size_t smem = static_cast<size_t>(K) * sizeof(bf16);
    const int tasks = kStage == kUp ? M : M / 2, warps = kFewThreads / 32;
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    // one wave: a CTA looks its row up once and takes several features
    const int all = (tasks + warps - 1) / warps, most = kFewResident * sms / P > 1 ? kFewResident * sms / P : 1;
    cudaLaunchAttribute attr;
    set_programmatic_launch(&attr, true);
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(all < most ? all : most, P);
    config.blockDim = dim3(kFewThreads);
    config.dynamicSmemBytes = smem;
    config.stream = s;
    config.attrs = &attr;
    config.numAttrs = kStage == kDown ? 1 : 0;
    COBALT_CUDA_TRY(cudaLaunchKernelEx(&config, ffn_few_rows_kernel<kStage>, static_cast<const bf16*>(x), static_cast<const bf16*>(weights),
                                       offsets, slot_expert, P, D, E, M, K, static_cast<bf16*>(out), static_cast<bf16*>(pre), err_word));
    return COBALT_OK;
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static int encode_function(EncodeTiled* out)
{
    static std::atomic<EncodeTiled> cached{nullptr};         // the same for every device
    EncodeTiled known = cached.load(std::memory_order_relaxed);
    if (!known) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        COBALT_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !f) return COBALT_ERR_UNSUPPORTED;
        known = reinterpret_cast<EncodeTiled>(f);
        cached.store(known, std::memory_order_relaxed);
    }
    *out = known;
    return COBALT_OK;
}

// A bf16 tensor of up to five dimensions, the first one contiguous; strides of the others in elements.
static int make_map(CUtensorMap* map, const void* ptr, int rank, const uint64_t (&dim)[5], const uint64_t (&stride)[5], const uint32_t (&box)[5])
{
    EncodeTiled encode;
    const int rc = encode_function(&encode);
    if (rc != COBALT_OK) return rc;
    cuuint64_t dims[5], bytes[4];
    cuuint32_t boxes[5], ones[5] = {1, 1, 1, 1, 1};
    for (int i = 0; i < rank; ++i) {
        dims[i] = dim[i];
        boxes[i] = box[i];
        if (i > 0) bytes[i - 1] = stride[i] * 2;
    }
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(ptr), dims, bytes, boxes, ones,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? COBALT_OK : record_cuda_error(cudaErrorInvalidValue);
}

static int rows_map(CUtensorMap* map, const void* ptr, int64_t rows, int64_t columns, uint32_t box_rows)
{
    const uint64_t dim[5] = {static_cast<uint64_t>(columns), static_cast<uint64_t>(rows)}, stride[5] = {1, static_cast<uint64_t>(columns)};
    const uint32_t box[5] = {kBlockK, box_rows};
    return make_map(map, ptr, 2, dim, stride, box);
}

static int weights_map(CUtensorMap* map, const void* ptr, int64_t E, int64_t rows, int64_t columns, uint32_t box_rows)
{
    const uint64_t dim[5] = {static_cast<uint64_t>(columns), static_cast<uint64_t>(rows), static_cast<uint64_t>(E)};
    const uint64_t stride[5] = {1, static_cast<uint64_t>(columns), static_cast<uint64_t>(rows * columns)};
    const uint32_t box[5] = {kBlockK, box_rows, 1};
    return make_map(map, ptr, 3, dim, stride, box);
}

// w_gate_up [E][2][F][H] read so that a box of 128 rows is eight gate rows, eight up rows, the next eight gate rows ...
static int gate_up_map(CUtensorMap* map, const void* ptr, int64_t E, int64_t F, int64_t H)
{
    const uint64_t h = H, f = F;
    const uint64_t dim[5] = {h, 8, 2, f / 8, static_cast<uint64_t>(E)}, stride[5] = {1, h, f * h, 8 * h, 2 * f * h};
    const uint32_t box[5] = {kBlockK, 8, 2, 8, 1};
    return make_map(map, ptr, 5, dim, stride, box);
}

template <int kStage>
static int launch_product(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& b_part, const ProductArgs& p, int64_t max_tiles,
                          cudaStream_t s)
{
    const void* kernel = reinterpret_cast<const void*>(ffn_product_kernel<kStage>);
    int rc = ensure_kernel_attributes(kernel, Shape<kStage>::kSmem, false);
    if (rc != COBALT_OK) return rc;
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    const int64_t pairs = max_tiles < sms / 2 ? max_tiles : sms / 2;
    // may start while the kernel before it (the plan, or a product of the same call) is at its end; it waits for that
    // one before it touches memory
    cudaLaunchAttribute attr;
    set_programmatic_launch(&attr, true);
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(2 * (pairs < 1 ? 1 : pairs)));
    config.blockDim = dim3(kProductThreads<kStage>);
    config.dynamicSmemBytes = Shape<kStage>::kSmem;
    config.stream = s;
    config.attrs = &attr;
    config.numAttrs = 1;
    COBALT_CUDA_TRY(cudaLaunchKernelEx(&config, ffn_product_kernel<kStage>, a, b, b_part, p));
    return COBALT_OK;
}

static int launch_plan(const uint32_t* offsets, const int32_t* slot_expert, int64_t P, int D, const ProductArgs& p, cudaStream_t s)
{
    const size_t bytes = plan_smem(D, p.E);
    // the attribute is set to the most that any call needs, so that concurrent calls agree on it
    const int rc = ensure_kernel_attributes(reinterpret_cast<const void*>(ffn_plan_kernel),
                                            plan_smem(COBALT_MAX_DESTS, COBALT_MAX_EXPERTS), false);
    if (rc != COBALT_OK) return rc;
    // (fewer threads for few slots: 12.7 us against 5 at 32 slots, one warp then writes all the tiles)
    ffn_plan_kernel<<<1, kPlanThreads, bytes, s>>>(offsets, slot_expert, P, D, p.E, p.plan, p.err_word);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

static int64_t m_tiles(int64_t features) { return (features + kTileM - 1) / kTileM; }

static int check_ffn(int64_t P, int32_t D, int32_t E, int32_t H, int32_t F)
{
    if (P < 0 || D < 1 || E < 1 || H < 1 || F < 1) return COBALT_ERR_INVALID_ARG;
    // (row coordinates of a tile may pass the last row by up to a tile, and an expert's tile count has to fit 23 bits)
    if (P > (1ll << 31) - (1ll << 21) || D > COBALT_MAX_DESTS || E > COBALT_MAX_EXPERTS || H % 8 != 0 || F % 8 != 0 || H > COBALT_FFN_MAX_WIDTH ||
        F > COBALT_FFN_MAX_WIDTH)
        return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

#define COBALT_TRY(expr)                       \
    do {                                       \
        const int cobalt_rc__ = (expr);        \
        if (cobalt_rc__ != COBALT_OK) return cobalt_rc__; \
    } while (0)

}  // namespace cobalt

using namespace cobalt;

extern "C" {

size_t cobalt_expert_ffn_workspace_bytes(int64_t P, int32_t D, int32_t E, int32_t H, int32_t F)
{
    if (check_ffn(P, D, E, H, F) != COBALT_OK) return 0;
    return plan_bytes(P, D, E);
}

int cobalt_expert_ffn(const void* rows, const uint32_t* dest_offsets, const int32_t* slot_expert, int64_t P, int32_t D, int32_t E,
                      int32_t H, int32_t F, const void* w_gate_up, const void* w_down, void* act, void* pre, void* out, void* workspace,
                      size_t workspace_bytes, cobalt_stream_t stream)
{
    COBALT_TRY(check_ffn(P, D, E, H, F));
    if (P == 0) return COBALT_OK;
    if (!rows || !dest_offsets || !slot_expert || !w_gate_up || !w_down || !act || !out) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(rows) || !aligned16(dest_offsets) || !aligned16(slot_expert) || !aligned16(w_gate_up) || !aligned16(w_down) ||
        !aligned16(act) || !aligned16(pre) || !aligned16(out) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < plan_bytes(P, D, E)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    ProductArgs p = {};
    COBALT_TRY(device_error_word(&p.err_word));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (P <= kFewRows && H <= 8 * kFewVecs && F <= 8 * kFewVecs) {
        COBALT_TRY(launch_few_rows<kUp>(rows, w_gate_up, dest_offsets, slot_expert, static_cast<int>(P), D, E, F, H, act, pre, p.err_word, s));
        return launch_few_rows<kDown>(act, w_down, dest_offsets, slot_expert, static_cast<int>(P), D, E, H, F, out, nullptr, p.err_word, s);
    }
    p.plan = plan_view(workspace, P, D, E);
    p.P = static_cast<int>(P);
    p.E = E;
    p.F = F;
    const int64_t row_tiles = max_row_tiles(P, static_cast<int>(P < D ? P : D));

    CUtensorMap a, b, part;
    COBALT_TRY(gate_up_map(&a, w_gate_up, E, F, H));
    COBALT_TRY(rows_map(&b, rows, P, H, 128));
    COBALT_TRY(rows_map(&part, rows, P, H, 16));
    CUtensorMap a2, b2, part2;
    COBALT_TRY(weights_map(&a2, w_down, E, H, F, 128));
    COBALT_TRY(rows_map(&b2, act, P, F, 128));
    COBALT_TRY(rows_map(&part2, act, P, F, 16));

    COBALT_TRY(launch_plan(dest_offsets, slot_expert, P, D, p, s));
    p.M = 2 * F;
    p.K = H;
    p.out = static_cast<bf16*>(act);
    p.pre = static_cast<bf16*>(pre);
    COBALT_TRY(launch_product<kUp>(a, b, part, p, row_tiles * m_tiles(p.M), s));
    p.M = H;
    p.K = F;
    p.out = static_cast<bf16*>(out);
    return launch_product<kDown>(a2, b2, part2, p, row_tiles * m_tiles(p.M), s);
}

int cobalt_expert_ffn_backward(const void* grad_out, const void* rows, const uint32_t* dest_offsets, const int32_t* slot_expert, int64_t P,
                               int32_t D, int32_t E, int32_t H, int32_t F, const void* w_gate_up, const void* w_down, const void* pre,
                               const void* act, void* grad_pre, void* grad_rows, void* grad_w_gate_up, void* grad_w_down, void* workspace,
                               size_t workspace_bytes, cobalt_stream_t stream)
{
    COBALT_TRY(check_ffn(P, D, E, H, F));
    if (!dest_offsets || !slot_expert) return COBALT_ERR_INVALID_ARG;
    if (P > 0 && !grad_rows && !grad_w_gate_up && !grad_w_down) return COBALT_ERR_INVALID_ARG;
    if (P > 0 && (!grad_out || !rows || !w_gate_up || !w_down || !pre || !act || !grad_pre)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_out) || !aligned16(rows) || !aligned16(dest_offsets) || !aligned16(slot_expert) || !aligned16(w_gate_up) ||
        !aligned16(w_down) || !aligned16(pre) || !aligned16(act) || !aligned16(grad_pre) || !aligned16(grad_rows) ||
        !aligned16(grad_w_gate_up) || !aligned16(grad_w_down) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < plan_bytes(P, D, E)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    ProductArgs p = {};
    COBALT_TRY(device_error_word(&p.err_word));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (P == 0) {                                // no rows: the weights' gradients are 0
        const size_t bytes = static_cast<size_t>(E) * H * F * sizeof(bf16);
        if (grad_w_gate_up) COBALT_CUDA_TRY(cudaMemsetAsync(grad_w_gate_up, 0, 2 * bytes, s));
        if (grad_w_down) COBALT_CUDA_TRY(cudaMemsetAsync(grad_w_down, 0, bytes, s));
        return COBALT_OK;
    }
    p.plan = plan_view(workspace, P, D, E);
    p.P = static_cast<int>(P);
    p.E = E;
    p.F = F;
    const int64_t row_tiles = max_row_tiles(P, static_cast<int>(P < D ? P : D));
    CUtensorMap a, b, part;
    COBALT_TRY(launch_plan(dest_offsets, slot_expert, P, D, p, s));
    if (grad_rows || grad_w_gate_up) {
        COBALT_TRY(weights_map(&a, w_down, E, H, F, kBlockK));
        COBALT_TRY(rows_map(&b, grad_out, P, H, 128));
        COBALT_TRY(rows_map(&part, grad_out, P, H, 16));
        p.M = F;
        p.K = H;
        p.pre_in = static_cast<const bf16*>(pre);
        p.out = static_cast<bf16*>(grad_pre);
        COBALT_TRY(launch_product<kDownBackward>(a, b, part, p, row_tiles * m_tiles(p.M), s));
    }
    if (grad_rows) {
        COBALT_TRY(weights_map(&a, w_gate_up, E, 2 * static_cast<int64_t>(F), H, kBlockK));
        COBALT_TRY(rows_map(&b, grad_pre, P, 2 * static_cast<int64_t>(F), 128));
        COBALT_TRY(rows_map(&part, grad_pre, P, 2 * static_cast<int64_t>(F), 16));
        p.M = H;
        p.K = 2 * F;
        p.out = static_cast<bf16*>(grad_rows);
        COBALT_TRY(launch_product<kUpBackward>(a, b, part, p, row_tiles * m_tiles(p.M), s));
    }
    if (grad_w_gate_up) {
        COBALT_TRY(rows_map(&a, grad_pre, P, 2 * static_cast<int64_t>(F), kBlockK));
        COBALT_TRY(rows_map(&b, rows, P, H, kBlockK));
        p.M = 2 * F;
        p.N = H;
        p.out = static_cast<bf16*>(grad_w_gate_up);
        COBALT_TRY(launch_product<kWeights>(a, b, b, p, E * m_tiles(p.M) * m_tiles(p.N), s));
    }
    if (grad_w_down) {
        COBALT_TRY(rows_map(&a, grad_out, P, H, kBlockK));
        COBALT_TRY(rows_map(&b, act, P, F, kBlockK));
        p.M = H;
        p.N = F;
        p.out = static_cast<bf16*>(grad_w_down);
        COBALT_TRY(launch_product<kWeights>(a, b, b, p, E * m_tiles(p.M) * m_tiles(p.N), s));
    }
    return COBALT_OK;
}

}  // extern "C"
