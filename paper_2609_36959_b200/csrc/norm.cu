// Layer norm over the H columns of each row, its backward pass and the reduction of its weights' gradients.
//
//   mu = sum x / H    var = sum (x - mu)^2 / H    rstd = 1 / sqrt(var + eps)    z = (x - mu) rstd
//   y  = z gamma + beta
//   g  = dy gamma     dx = rstd (g - mean(g) - z mean(g z))      dgamma = sum_t dy z     dbeta = sum_t dy
//
// A row is read once and stays on the chip, so the variance is the sum of squares about the mean and not a
// difference of two large sums.  All sums are fp32.  The fp32 sum of fp32 values is rounded, which would leave a row of
// large equal values a z of its own; so their differences from that first mean are summed too, exactly where they are
// small, and correct it:
//   mu = mu1 + mean(d)    var = (sum d^2 - mean(d) sum d) / H    with d = x - mu1
// (for bf16 values of one magnitude the first sum is exact: 8 + 14 bits).  A group of threads owns a row: one warp while a
// lane needs at most four 16-byte vectors, the whole CTA above that.
//
// Rows of more than 128 vectors, many of them: persistent CTAs, a thread owns the same columns of every row (its gamma
// and beta, or the sums of their gradients, stay in registers), and rows come in through a ring of bulk copies, so that
// the loads of the next rows run under the sums and barriers of the present ones.  Up to four rows share a barrier.
// Backward: each CTA writes one partial sum a column, and a second kernel adds the partials in a fixed order (no
// atomics: the result does not vary from run to run).
// Measured at 65536 x 7168 bf16: forward 346 us (5.4 TB/s), backward 532 us (5.3 TB/s; bound by the registers of the
// gradient sums, 44 % of the warps an SM can hold, and a barrier for every two rows), column sums 4 us.
#include "numeric.cuh"
#include "tcgen05.cuh"

namespace cobalt {

constexpr int kNormMaxH = 16384;
constexpr int kWarpRowVecs = 128;        // 16-byte vectors of a row up to which one warp takes it (forward: 256)
constexpr int kWarpRowThreads = 256;

// The mean's correction and 1 / sqrt(var + eps) from the sums of d and of d^2 (of h values).  The correction is a division:
// exact for a constant row.  The other two are good to two units.
__device__ __forceinline__ float mean_shift(float sum, float h) { return sum / h; }
__device__ __forceinline__ float shifted_rstd(float shift, float sum, float squares, float inv_h, float eps)
{
    const float part = shift * sum;
    float var = fabsf(part) < INFINITY ? squares - part : squares;     // where it overflows the squares have, too
    if (var < 0.0f) var = 0.0f;                                        // rounding; a NaN stays
    return rsqrtf(fmaf(var, inv_h, eps));
}

// post(sum) of v[0..N) over the CTA, N = 1, 2, 4 or 8; what is computed of a sum is computed by one lane (every lane l
// calls post with the sum of value l % N).  The first log2 N steps of the warp's tree halve the values a lane holds (six
// shuffles for four values, not twenty).  `scratch`: N x 32 floats, not in use by an earlier call.
template <int N, typename Post>
__device__ __forceinline__ void cta_sums(float (&v)[N], float* scratch, Post post)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    constexpr uint32_t kLanes = 0xFFFFFFFFu;
    float r;
    if constexpr (N == 8) {
        float q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = ((lane & 1) ? v[2 * i + 1] : v[2 * i]) + __shfl_xor_sync(kLanes, (lane & 1) ? v[2 * i] : v[2 * i + 1], 1);
        const float a = ((lane & 2) ? q[1] : q[0]) + __shfl_xor_sync(kLanes, (lane & 2) ? q[0] : q[1], 2);
        const float b = ((lane & 2) ? q[3] : q[2]) + __shfl_xor_sync(kLanes, (lane & 2) ? q[2] : q[3], 2);
        r = ((lane & 4) ? b : a) + __shfl_xor_sync(kLanes, (lane & 4) ? a : b, 4);
    } else if constexpr (N == 4) {
        const float a = ((lane & 1) ? v[1] : v[0]) + __shfl_xor_sync(kLanes, (lane & 1) ? v[0] : v[1], 1);
        const float b = ((lane & 1) ? v[3] : v[2]) + __shfl_xor_sync(kLanes, (lane & 1) ? v[2] : v[3], 1);
        r = ((lane & 2) ? b : a) + __shfl_xor_sync(kLanes, (lane & 2) ? a : b, 2);
    } else if constexpr (N == 2) {
        r = ((lane & 1) ? v[1] : v[0]) + __shfl_xor_sync(kLanes, (lane & 1) ? v[0] : v[1], 1);
    } else {
        r = v[0];
    }
#pragma unroll
    for (int off = N; off < 32; off <<= 1) r += __shfl_xor_sync(kLanes, r, off);
    if (lane < N) scratch[warp * N + lane] = r;             // lane l < N holds the sum of value l
    __syncthreads();
    r = 0.0f;
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (lane + 32 * k < warps * N) r += scratch[lane + 32 * k];
#pragma unroll
    for (int off = N; off < 32; off <<= 1) r += __shfl_xor_sync(kLanes, r, off);
    r = post(r);
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = N == 1 ? r : __shfl_sync(kLanes, r, k);
}

// post of cta_sums for sums of d (even) and of d^2 (odd) in turn: the mean's shift and rstd.
struct ShiftAndRstd {
    float h, inv_h, eps;
    __device__ __forceinline__ float operator()(float sum) const
    {
        const float other = __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
        const bool odd = threadIdx.x & 1;                              // (both by all lanes: a branch would run one after the other)
        const float first = odd ? other : sum, squares = odd ? sum : other, shift = mean_shift(first, h);
        const float rstd = shifted_rstd(shift, first, squares, inv_h, eps);
        return odd ? rstd : shift;
    }
};

template <typename T>
constexpr bool kShiftMean = sizeof(T) == 4;

// R rows a group, VPT vectors of each row a thread.
template <typename T, int VPT, int R, bool kCta>
__global__ void __launch_bounds__(1024)
layer_norm_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t rows, int H, float eps, T* y,
                  float* __restrict__ mean, float* __restrict__ rstd)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ float scratch[2][kShiftMean<T> ? 64 : 32];
    static_assert(!kCta || R == 1, "a CTA takes one row here");
    const int group = kCta ? blockDim.x : 32, lane = kCta ? threadIdx.x : (threadIdx.x & 31);
    const int groups = kCta ? 1 : (blockDim.x >> 5), own = kCta ? 0 : (threadIdx.x >> 5);
    const int n_vec = H / N;
    const float h = static_cast<float>(H), inv_h = 1.0f / h;
    const int64_t r0 = (static_cast<int64_t>(blockIdx.x) * groups + own) * R;
    if (r0 >= rows) return;
    uint4 v[R][VPT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = lane + i * group;
            v[r][i] = make_uint4(0, 0, 0, 0);
            if (at < n_vec && r0 + r < rows) v[r][i] = ld_once16(x + (r0 + r) * H + at * N);
        }
    float mu[R], rs[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        mu[r] = 0.0f;                        // vectors past the row's end hold zeros
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float f[N];
            Vec16<T>::unpack(v[r][i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) mu[r] += f[k];
        }
    }
    // (a division where no correction follows: exact for a constant row of bf16 values)
    auto to_mean = [h, inv_h](float sum) { return kShiftMean<T> ? sum * inv_h : sum / h; };
    auto to_rstd = [h, eps](float sum) { return 1.0f / sqrtf(sum / h + eps); };
    if constexpr (kCta) {
        cta_sums<1>(mu, scratch[0], to_mean);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) mu[r] = to_mean(warp_sum(mu[r]));
    }
    float first[R];                          // kShiftMean: sums of the differences
#pragma unroll
    for (int r = 0; r < R; ++r) {
        rs[r] = first[r] = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (lane + i * group < n_vec) {
                float f[N];
                Vec16<T>::unpack(v[r][i], f);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float d = f[k] - mu[r];
                    if (kShiftMean<T>) first[r] += d;
                    rs[r] = fmaf(d, d, rs[r]);
                }
            }
        }
    }
    if constexpr (kCta && kShiftMean<T>) {
        float both[2] = {first[0], rs[0]};
        cta_sums<2>(both, scratch[1], ShiftAndRstd{h, inv_h, eps});
        mu[0] += both[0];
        rs[0] = both[1];
    } else if constexpr (kCta) {
        cta_sums<1>(rs, scratch[1], to_rstd);
    } else if constexpr (kShiftMean<T>) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float sum = warp_sum(first[r]), shift = mean_shift(sum, h);
            rs[r] = shifted_rstd(shift, sum, warp_sum(rs[r]), inv_h, eps);
            mu[r] += shift;
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) rs[r] = to_rstd(warp_sum(rs[r]));
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (lane == 0 && r0 + r < rows) {
            mean[r0 + r] = mu[r];
            rstd[r0 + r] = rs[r];
        }
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * group;
        if (at < n_vec) {
            float g[N], b[N];
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                *reinterpret_cast<float4*>(g + k) = __ldg(reinterpret_cast<const float4*>(gamma + at * N + k));
                *reinterpret_cast<float4*>(b + k) = __ldg(reinterpret_cast<const float4*>(beta + at * N + k));
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float f[N];
                Vec16<T>::unpack(v[r][i], f);
#pragma unroll
                for (int k = 0; k < N; ++k) f[k] = fmaf((f[k] - mu[r]) * rs[r], g[k], b[k]);
                if (r0 + r < rows) st_stream16(y + (r0 + r) * H + at * N, Vec16<T>::pack(f));
            }
        }
    }
}

// Backward, one warp a row; partial: [CTAs][2][H].
template <typename T, int VPT>
__global__ void __launch_bounds__(kWarpRowThreads)
layer_norm_backward_warp_kernel(const T* grad_y, const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                const float* __restrict__ rstd, int64_t rows, int H, T* grad_x, float* __restrict__ partial)
{
    constexpr int N = Vec16<T>::kElems;
    extern __shared__ float sums[];          // [2][H]
    launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = kWarpRowThreads / 32;
    const int n_vec = H / N;
    const float inv_h = 1.0f / static_cast<float>(H);
    float gm[VPT][N], dg[VPT][N], db[VPT][N];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * 32;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            gm[i][k] = at < n_vec ? __ldg(gamma + at * N + k) : 0.0f;
            dg[i][k] = 0.0f;
            db[i][k] = 0.0f;
        }
    }
    const int64_t step = static_cast<int64_t>(gridDim.x) * warps;
    for (int64_t r = static_cast<int64_t>(blockIdx.x) * warps + warp; r < rows; r += step) {
        uint4 xv[VPT], yv[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = lane + i * 32;
            xv[i] = yv[i] = make_uint4(0, 0, 0, 0);
            if (at < n_vec) {
                xv[i] = ld_once16(x + r * H + at * N);
                yv[i] = ld_once16(grad_y + r * H + at * N);
            }
        }
        const float mu = __ldg(mean + r), rs = __ldg(rstd + r);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            float z[N], d[N];
            Vec16<T>::unpack(xv[i], z);
            Vec16<T>::unpack(yv[i], d);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                // past the row's end gamma and dy are 0, and z must not be (a NaN times 0 would stay)
                const float zz = lane + i * 32 < n_vec ? (z[k] - mu) * rs : 0.0f, g = d[k] * gm[i][k];
                s1 += g;
                s2 = fmaf(g, zz, s2);
                dg[i][k] = fmaf(d[k], zz, dg[i][k]);
                db[i][k] += d[k];
            }
        }
        const float c1 = warp_sum(s1) * inv_h, c2 = warp_sum(s2) * inv_h;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = lane + i * 32;
            if (at < n_vec) {
                float z[N], d[N];
                Vec16<T>::unpack(xv[i], z);
                Vec16<T>::unpack(yv[i], d);
#pragma unroll
                for (int k = 0; k < N; ++k) d[k] = rs * (fmaf(d[k], gm[i][k], -c1) - (z[k] - mu) * rs * c2);
                st_stream16(grad_x + r * H + at * N, Vec16<T>::pack(d));
            }
        }
    }
    // the CTA's sum, warp after warp
    for (int w = 0; w < warps; ++w) {
        if (warp == w) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int at = lane + i * 32;
                if (at < n_vec) {
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        sums[at * N + k] = dg[i][k] + (w > 0 ? sums[at * N + k] : 0.0f);
                        sums[H + at * N + k] = db[i][k] + (w > 0 ? sums[H + at * N + k] : 0.0f);
                    }
                }
            }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * H; c += kWarpRowThreads) partial[static_cast<int64_t>(blockIdx.x) * 2 * H + c] = sums[c];
}

__device__ __forceinline__ void bulk_load_row(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
                 "r"(bar)
                 : "memory");
}

// Most threads of a ring CTA: 896 leave 72 registers each; of the rows of more than 1792 vectors, fp32 ones have up to
// 4096 and bf16 ones up to 2048.
template <typename T, int VPT>
constexpr int kRingThreads = VPT == 4 ? (sizeof(T) == 4 ? 1024 : 512) : 896;

// The ring of a persistent CTA: turn i takes rows start + i step .. + R of `Tensors` tensors; a slot holds R rows of the
// first tensor, then R rows of the second.
template <typename T, int R, int kTensors>
struct RowRing {
    const T* src[kTensors];
    uint32_t base, bars, row_bytes;
    int64_t rows, start, step, turns;
    int H, slots;

    __device__ __forceinline__ uint32_t slot_bytes() const { return kTensors * R * row_bytes; }
    __device__ __forceinline__ void init(uint32_t smem, int64_t rows_, int H_, int slots_)
    {
        rows = rows_;
        H = H_;
        slots = slots_;
        row_bytes = static_cast<uint32_t>(H) * sizeof(T);
        base = smem;
        bars = base + static_cast<uint32_t>(slots) * slot_bytes();
        start = static_cast<int64_t>(blockIdx.x) * R;
        step = static_cast<int64_t>(gridDim.x) * R;
        turns = start < rows ? (rows - start + step - 1) / step : 0;
        if (threadIdx.x == 0) {
            for (int s = 0; s < slots; ++s) barrier_init(bars + 8 * s, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncthreads();
        if (threadIdx.x == 0)
            for (int64_t i = 0; i < turns && i < slots; ++i) load(i, static_cast<int>(i));
    }
    __device__ __forceinline__ void load(int64_t turn, int slot) const     // by one thread
    {
        const int64_t r = start + turn * step;
        const uint32_t bytes = static_cast<uint32_t>(rows - r < R ? rows - r : R) * row_bytes, at = base + slot * slot_bytes();
        barrier_expect(bars + 8 * slot, kTensors * bytes);
#pragma unroll
        for (int k = 0; k < kTensors; ++k) bulk_load_row(at + k * R * row_bytes, src[k] + r * H, bytes, bars + 8 * slot);
    }
};

// Forward: gamma and beta of the thread's columns stay in registers, its part of the R rows too.
template <typename T, int VPT, int R>
__global__ void __launch_bounds__(kRingThreads<T, VPT>)
layer_norm_ring_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t rows, int H, float eps, T* y,
                       float* __restrict__ mean, float* __restrict__ rstd, int slots, uint32_t* __restrict__ err_word)
{
    constexpr int N = Vec16<T>::kElems;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float scratch[2][(kShiftMean<T> ? 2 : 1) * R * 32];
    __shared__ volatile int dead;            // a wait ran out: the rest is not waited for
    const int tid = threadIdx.x, n_vec = H / N;
    const float h = static_cast<float>(H), inv_h = 1.0f / h;
    if (tid == 0) dead = 0;
    RowRing<T, R, 1> ring;
    ring.src[0] = x;
    ring.init(smem_u32(smem), rows, H, slots);
    Pair gm[VPT][N / 2], bt[VPT][N / 2];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = tid + i * blockDim.x;
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            gm[i][k / 2] = at < n_vec ? pair(__ldg(gamma + at * N + k), __ldg(gamma + at * N + k + 1)) : pair(0.0f);
            bt[i][k / 2] = at < n_vec ? pair(__ldg(beta + at * N + k), __ldg(beta + at * N + k + 1)) : pair(0.0f);
        }
    }
    int s = 0;
    uint32_t phase = 0;
    for (int64_t turn = 0; turn < ring.turns; ++turn) {
        const int64_t r0 = ring.start + turn * ring.step;
        if (!dead && !barrier_wait(ring.bars + 8 * s, phase)) {
            dead = 1;
            flag_error(err_word, COBALT_DEVERR_WAIT_TIMEOUT);
        }
        const uint8_t* slot = smem + static_cast<size_t>(s) * ring.slot_bytes();
        uint4 v[R][VPT];
        float mu[R], rs[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Pair acc = pair(0.0f);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int at = tid + i * blockDim.x;
                v[r][i] = make_uint4(0, 0, 0, 0);            // past the row's end, and for the rows past the last
                if (at < n_vec && r0 + r < rows) v[r][i] = *reinterpret_cast<const uint4*>(slot + r * ring.row_bytes + at * 16);
                Pair f[N / 2];
                unpack_pairs<T>(v[r][i], f);
#pragma unroll
                for (int k = 0; k < N / 2; ++k) acc = acc + f[k];
            }
            mu[r] = acc.v.x + acc.v.y;
        }
        cta_sums<R>(mu, scratch[0], [h, inv_h](float sum) { return kShiftMean<T> ? sum * inv_h : sum / h; });
        // behind that barrier every thread has its part of the slot in registers
        if (tid == 0 && turn + slots < ring.turns) ring.load(turn + slots, s);
        float both[2 * R];                   // sums of the differences (kShiftMean) and of their squares
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Pair acc = pair(0.0f), first = pair(0.0f);
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (tid + i * blockDim.x < n_vec) {
                    Pair f[N / 2];
                    unpack_pairs<T>(v[r][i], f);
#pragma unroll
                    for (int k = 0; k < N / 2; ++k) {
                        const Pair d = f[k] + pair(-mu[r]);
                        if (kShiftMean<T>) first = first + d;
                        acc = fma2(d, d, acc);
                    }
                }
            }
            both[2 * r] = first.v.x + first.v.y;
            both[2 * r + 1] = rs[r] = acc.v.x + acc.v.y;
        }
        if constexpr (kShiftMean<T>) {
            cta_sums<2 * R>(both, scratch[1], ShiftAndRstd{h, inv_h, eps});
#pragma unroll
            for (int r = 0; r < R; ++r) {
                mu[r] += both[2 * r];
                rs[r] = both[2 * r + 1];
            }
        } else {
            cta_sums<R>(rs, scratch[1], [h, eps](float sum) { return 1.0f / sqrtf(sum / h + eps); });
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r0 + r >= rows) continue;
            if (tid == 0) {
                mean[r0 + r] = mu[r];
                rstd[r0 + r] = rs[r];
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int at = tid + i * blockDim.x;
                if (at < n_vec) {
                    Pair f[N / 2];
                    unpack_pairs<T>(v[r][i], f);
#pragma unroll
                    for (int k = 0; k < N / 2; ++k) f[k] = fma2((f[k] + pair(-mu[r])) * pair(rs[r]), gm[i][k], bt[i][k]);
                    st_stream16(y + (r0 + r) * H + at * N, pack_pairs<T>(f));
                }
            }
        }
        if (++s == slots) {
            s = 0;
            phase ^= 1;
        }
    }
    if (dead && tid == 0)                    // copies in flight land before the shared memory is given back
        for (int64_t i = ring.turns > slots ? ring.turns - slots : 0; i < ring.turns; ++i)
            (void)barrier_wait(ring.bars + 8 * static_cast<int>(i % slots), static_cast<uint32_t>(i / slots) & 1);
}

// Backward: partial: [CTAs][2][H].
template <typename T, int VPT, int R>
__global__ void __launch_bounds__(kRingThreads<T, VPT>)
layer_norm_backward_ring_kernel(const T* grad_y, const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                const float* __restrict__ rstd, int64_t rows, int H, T* grad_x, float* __restrict__ partial, int slots,
                                uint32_t* __restrict__ err_word)
{
    constexpr int N = Vec16<T>::kElems;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float scratch[2][2 * R * 32];
    __shared__ float2 stats[2][R];
    __shared__ volatile int dead;
    const int tid = threadIdx.x, n_vec = H / N;
    const float inv_h = 1.0f / static_cast<float>(H);
    launch_dependents();
    if (tid == 0) dead = 0;
    RowRing<T, R, 2> ring;
    ring.src[0] = x;
    ring.src[1] = grad_y;
    ring.init(smem_u32(smem), rows, H, slots);
    Pair gm[VPT][N / 2], dg[VPT][N / 2], db[VPT][N / 2];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = tid + i * blockDim.x;
#pragma unroll
        for (int k = 0; k < N; k += 2) {
            gm[i][k / 2] = at < n_vec ? pair(__ldg(gamma + at * N + k), __ldg(gamma + at * N + k + 1)) : pair(0.0f);
            dg[i][k / 2] = pair(0.0f);
            db[i][k / 2] = pair(0.0f);
        }
    }
    // mean and rstd of a turn's rows: read two turns ahead by the first R threads, in shared memory one turn ahead
    auto row_stats = [&](int64_t r) { return tid < R && r < rows ? make_float2(__ldg(mean + r), __ldg(rstd + r)) : make_float2(0.0f, 0.0f); };
    if (tid < R) stats[0][tid] = row_stats(ring.start + tid);
    float2 ahead = row_stats(ring.start + ring.step + tid);
    __syncthreads();
    int s = 0, before = 0;
    uint32_t phase = 0;
    for (int64_t turn = 0; turn < ring.turns; ++turn) {
        const int64_t r = ring.start + turn * ring.step;
        if (!dead && !barrier_wait(ring.bars + 8 * s, phase)) {
            dead = 1;
            flag_error(err_word, COBALT_DEVERR_WAIT_TIMEOUT);
        }
        const uint8_t* slot = smem + static_cast<size_t>(s) * ring.slot_bytes();
        float sum[2 * R], mu[R], rs[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            mu[j] = stats[turn & 1][j].x;
            rs[j] = stats[turn & 1][j].y;
            Pair s1 = pair(0.0f), s2 = pair(0.0f);
            if (r + j < rows) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int at = tid + i * blockDim.x;
                    if (at < n_vec) {
                        Pair z[N / 2], d[N / 2];
                        unpack_pairs<T>(*reinterpret_cast<const uint4*>(slot + j * ring.row_bytes + at * 16), z);
                        unpack_pairs<T>(*reinterpret_cast<const uint4*>(slot + (R + j) * ring.row_bytes + at * 16), d);
#pragma unroll
                        for (int k = 0; k < N / 2; ++k) {
                            const Pair zz = (z[k] + pair(-mu[j])) * pair(rs[j]), g = d[k] * gm[i][k];
                            s1 = s1 + g;
                            s2 = fma2(g, zz, s2);
                            dg[i][k] = fma2(d[k], zz, dg[i][k]);
                            db[i][k] = db[i][k] + d[k];
                        }
                    }
                }
            }
            sum[2 * j] = s1.v.x + s1.v.y;
            sum[2 * j + 1] = s2.v.x + s2.v.y;
        }
        if (tid < R) stats[(turn + 1) & 1][tid] = ahead;     // last read before the barrier of the turn before
        ahead = row_stats(r + 2 * ring.step + tid);
        cta_sums<2 * R>(sum, scratch[turn & 1], [inv_h](float total) { return total * inv_h; });
        // behind that barrier every thread is done with the slot before this one
        if (tid == 0 && slots > 1 && turn > 0 && turn - 1 + slots < ring.turns) ring.load(turn - 1 + slots, before);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            if (r + j >= rows) continue;
            const float c1 = sum[2 * j], c2 = sum[2 * j + 1];
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int at = tid + i * blockDim.x;
                if (at < n_vec) {
                    Pair z[N / 2], d[N / 2];
                    unpack_pairs<T>(*reinterpret_cast<const uint4*>(slot + j * ring.row_bytes + at * 16), z);
                    unpack_pairs<T>(*reinterpret_cast<const uint4*>(slot + (R + j) * ring.row_bytes + at * 16), d);
#pragma unroll
                    for (int k = 0; k < N / 2; ++k) {
                        const Pair zz = (z[k] + pair(-mu[j])) * pair(rs[j]);
                        d[k] = pair(rs[j]) * fma2(zz, pair(-c2), fma2(d[k], gm[i][k], pair(-c1)));
                    }
                    st_stream16(grad_x + (r + j) * H + at * N, pack_pairs<T>(d));
                }
            }
        }
        if (slots == 1) {                    // the slot itself comes next
            __syncthreads();
            if (tid == 0 && turn + 1 < ring.turns) ring.load(turn + 1, 0);
        }
        before = s;
        if (++s == slots) {
            s = 0;
            phase ^= 1;
        }
    }
    if (dead && tid == 0)                    // copies in flight land before the shared memory is given back
        for (int64_t i = ring.turns > slots ? ring.turns - slots : 0; i < ring.turns; ++i)
            (void)barrier_wait(ring.bars + 8 * static_cast<int>(i % slots), static_cast<uint32_t>(i / slots) & 1);
    float* out = partial + static_cast<int64_t>(blockIdx.x) * 2 * H;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = tid + i * blockDim.x;
        if (at < n_vec) {
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                *reinterpret_cast<float4*>(out + at * N + k) =
                    make_float4(dg[i][k / 2].v.x, dg[i][k / 2].v.y, dg[i][k / 2 + 1].v.x, dg[i][k / 2 + 1].v.y);
                *reinterpret_cast<float4*>(out + H + at * N + k) =
                    make_float4(db[i][k / 2].v.x, db[i][k / 2].v.y, db[i][k / 2 + 1].v.x, db[i][k / 2 + 1].v.y);
            }
        }
    }
}

// grad_gamma and grad_beta: column sums of the parts, 32 columns a CTA, every warp a slice of the parts.
__global__ void __launch_bounds__(1024)
layer_norm_reduce_kernel(const float* partial, int parts, int H, float* __restrict__ grad_gamma,
                         float* __restrict__ grad_beta)
{
    wait_for_prior_kernel();                             // the parts
    __shared__ float slice[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;              // over 2H columns: gamma's, then beta's
    float s = 0.0f;
    if (col < 2 * H) {
#pragma unroll 4
        for (int p = warp; p < parts; p += 32) s += partial[static_cast<int64_t>(p) * 2 * H + col];
    }
    slice[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < 2 * H) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += slice[i][lane];
        if (col < H) grad_gamma[col] = total;
        else grad_beta[col - H] = total;
    }
}

// How the rows are dealt to threads: vectors a thread holds, threads of a CTA, whether a CTA owns its rows.
struct NormShape {
    int vpt, threads;
    bool cta;
};

// Without the ring: one warp a row up to eight vectors a lane, one CTA above that, two vectors a thread up to 2048 of them.
static NormShape norm_shape(int n_vec)
{
    NormShape s;
    s.cta = n_vec > 2 * kWarpRowVecs;
    if (!s.cta) {
        s.threads = kWarpRowThreads;
        s.vpt = n_vec <= 32 ? 1 : n_vec <= 64 ? 2 : n_vec <= 128 ? 4 : 8;
    } else {
        s.vpt = n_vec <= 2048 ? 2 : 4;
        s.threads = ((n_vec + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    }
    return s;
}

// The ring kernels: one vector a thread up to 896, so that what belongs to its columns takes few registers; `many_rows`
// rows a slot then (twice that fits for every such row, of one tensor times four as of two times two), one row above, and as
// many slots as fit, at most four.
struct RingShape {
    int vpt, threads, rows, slots;
    size_t smem;
    int resident;                        // CTAs an SM
};

constexpr size_t kRingBytes = 208 * 1024;
static_assert(2 * 4 * 896 * 16 <= kRingBytes && 2 * 4 * 512 * 16 <= kRingBytes / 2, "two slots of four rows, or of two of two tensors");

static RingShape ring_shape(int H, int elem_bytes, int tensors, int many_rows)
{
    RingShape s = {};
    const int n_vec = H * elem_bytes / 16;
    s.vpt = n_vec <= 896 ? 1 : n_vec <= 1792 ? 2 : 4;
    s.threads = ((n_vec + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    s.resident = s.threads <= 512 ? 2 : 1;
    const size_t row = static_cast<size_t>(tensors) * H * elem_bytes, room = kRingBytes / s.resident;
    s.rows = s.vpt == 1 ? many_rows : 1;
    s.slots = static_cast<int>(room / (s.rows * row));
    if (s.slots > 4) s.slots = 4;
    if (s.slots < 1) s.slots = 1;
    s.smem = s.slots * (s.rows * row) + 8 * s.slots;
    return s;
}

// The backward kernel's threads: the ring, or one warp a row.
struct NormBackwardShape : RingShape {
    bool cta;
};

static NormBackwardShape norm_backward_shape(int H, int elem_bytes)
{
    NormBackwardShape s = {};
    const int n_vec = H * elem_bytes / 16;
    if (n_vec > kWarpRowVecs) {
        static_cast<RingShape&>(s) = ring_shape(H, elem_bytes, 2, 2);
        s.cta = true;
        return s;
    }
    s.threads = kWarpRowThreads;
    s.vpt = n_vec <= 32 ? 1 : n_vec <= 64 ? 2 : 4;
    s.smem = 2 * sizeof(float) * H;
    s.resident = s.vpt == 4 ? 2 : 4;
    return s;
}

// CTAs (= partial sums) of the backward kernel.
static int64_t norm_parts(int64_t T, const NormBackwardShape& s, int sms)
{
    const int64_t rows = s.cta ? s.rows : s.threads / 32;
    int64_t ctas = (T + rows - 1) / rows;
    if (ctas > static_cast<int64_t>(s.resident) * sms) ctas = static_cast<int64_t>(s.resident) * sms;
    return ctas < 1 ? 1 : ctas;          // no rows: one part of zeros
}

constexpr int kMaxSms = 256;             // the workspace query knows no device: sized for this many

static int check_norm(int64_t T, int32_t H, int32_t dtype)
{
    if (T < 0 || H < 1 || (dtype != COBALT_BF16 && dtype != COBALT_F32)) return COBALT_ERR_INVALID_ARG;
    if (H % 8 != 0 || H > kNormMaxH || T >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

template <typename T, int VPT, int R>
static int launch_norm_ring(const T* x, const float* gamma, const float* beta, int64_t rows, int H, float eps, T* y, float* mean, float* rstd,
                            const RingShape& shape, int sms, uint32_t* err_word, cudaStream_t s)
{
    const int rc = ensure_kernel_attributes(reinterpret_cast<const void*>(layer_norm_ring_kernel<T, VPT, R>), kRingBytes + 64, false);
    if (rc != COBALT_OK) return rc;
    layer_norm_ring_kernel<T, VPT, R><<<shape.resident * sms, shape.threads, shape.smem, s>>>(x, gamma, beta, rows, H, eps, y, mean, rstd,
                                                                                             shape.slots, err_word);
    return COBALT_OK;
}

template <typename T>
static int launch_norm(const T* x, const float* gamma, const float* beta, int64_t rows, int H, float eps, T* y, float* mean, float* rstd,
                       cudaStream_t s)
{
    int sms = 0;
    int rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    const NormShape shape = norm_shape(H / Vec16<T>::kElems);
    const RingShape ring = ring_shape(H, sizeof(T), 1, 4);
    // the ring pays once every CTA has a few turns; below that its start-up costs more than a CTA a row
    if (shape.cta && rows >= static_cast<int64_t>(4) * ring.rows * ring.resident * sms) {
        uint32_t* err_word = nullptr;
        rc = device_error_word(&err_word);
        if (rc != COBALT_OK) return rc;
        if (ring.vpt == 1) return launch_norm_ring<T, 1, 4>(x, gamma, beta, rows, H, eps, y, mean, rstd, ring, sms, err_word, s);
        if (ring.vpt == 4) return launch_norm_ring<T, 4, 1>(x, gamma, beta, rows, H, eps, y, mean, rstd, ring, sms, err_word, s);
        return launch_norm_ring<T, 2, 1>(x, gamma, beta, rows, H, eps, y, mean, rstd, ring, sms, err_word, s);
    }
    // several rows a warp (they share gamma and beta) only where that still leaves every SM eight warps
    const bool several = !shape.cta && shape.vpt < 4 && rows >= static_cast<int64_t>(sms) * 8 * (4 / shape.vpt);
    const int64_t per_cta = shape.cta ? 1 : shape.threads / 32 * (several ? 4 / shape.vpt : 1);
    const unsigned grid = static_cast<unsigned>((rows + per_cta - 1) / per_cta);
#define COBALT_NORM_FWD(VPT, R, CTA) \
    layer_norm_kernel<T, VPT, R, CTA><<<grid, shape.threads, 0, s>>>(x, gamma, beta, rows, H, eps, y, mean, rstd)
    if (shape.cta) {
        if (shape.vpt == 2) COBALT_NORM_FWD(2, 1, true);
        else if constexpr (sizeof(T) == 4) COBALT_NORM_FWD(4, 1, true);
    } else if (several) {
        if (shape.vpt == 1) COBALT_NORM_FWD(1, 4, false);
        else COBALT_NORM_FWD(2, 2, false);
    } else {
        if (shape.vpt == 1) COBALT_NORM_FWD(1, 1, false);
        else if (shape.vpt == 2) COBALT_NORM_FWD(2, 1, false);
        else if (shape.vpt == 4) COBALT_NORM_FWD(4, 1, false);
        else COBALT_NORM_FWD(8, 1, false);
    }
#undef COBALT_NORM_FWD
    return COBALT_OK;
}

template <typename T, int VPT, int R>
static int launch_ring(const T* grad_y, const T* x, const float* gamma, const float* mean, const float* rstd, int64_t rows, int H, T* grad_x,
                       float* partial, const RingShape& shape, unsigned grid, uint32_t* err_word, cudaStream_t s)
{
    const void* kernel = reinterpret_cast<const void*>(layer_norm_backward_ring_kernel<T, VPT, R>);
    const int rc = ensure_kernel_attributes(kernel, kRingBytes + 64, false);
    if (rc != COBALT_OK) return rc;
    layer_norm_backward_ring_kernel<T, VPT, R><<<grid, shape.threads, shape.smem, s>>>(grad_y, x, gamma, mean, rstd, rows, H, grad_x, partial,
                                                                                       shape.slots, err_word);
    return COBALT_OK;
}

template <typename T>
static int launch_norm_backward(const T* grad_y, const T* x, const float* gamma, const float* mean, const float* rstd, int64_t rows, int H,
                                T* grad_x, float* partial, int sms, int* parts, uint32_t* err_word, cudaStream_t s)
{
    const NormBackwardShape shape = norm_backward_shape(H, sizeof(T));
    *parts = static_cast<int>(norm_parts(rows, shape, sms < kMaxSms ? sms : kMaxSms));
    const unsigned grid = static_cast<unsigned>(*parts);
    if (!shape.cta) {
#define COBALT_NORM_BWD(VPT)                                                                                                       \
    layer_norm_backward_warp_kernel<T, VPT><<<grid, shape.threads, shape.smem, s>>>(grad_y, x, gamma, mean, rstd, rows, H, grad_x, partial)
        if (shape.vpt == 1) COBALT_NORM_BWD(1);
        else if (shape.vpt == 2) COBALT_NORM_BWD(2);
        else COBALT_NORM_BWD(4);
#undef COBALT_NORM_BWD
        return COBALT_OK;
    }
    if (shape.vpt == 1) return launch_ring<T, 1, 2>(grad_y, x, gamma, mean, rstd, rows, H, grad_x, partial, shape, grid, err_word, s);
    if (shape.vpt == 4) return launch_ring<T, 4, 1>(grad_y, x, gamma, mean, rstd, rows, H, grad_x, partial, shape, grid, err_word, s);
    return launch_ring<T, 2, 1>(grad_y, x, gamma, mean, rstd, rows, H, grad_x, partial, shape, grid, err_word, s);
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_layer_norm(const void* x, const float* gamma, const float* beta, int64_t T, int32_t H, int32_t dtype, float eps,
                      void* y, float* mean, float* rstd, cobalt_stream_t stream)
{
    int rc = check_norm(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    if (!(eps >= 0.0f)) return COBALT_ERR_INVALID_ARG;
    if (T == 0) return COBALT_OK;
    if (!x || !gamma || !beta || !y || !mean || !rstd || !aligned16(x) || !aligned16(gamma) || !aligned16(beta) ||
        !aligned16(y) || !aligned16(mean) || !aligned16(rstd))
        return COBALT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16)
        rc = launch_norm(static_cast<const __nv_bfloat16*>(x), gamma, beta, T, H, eps, static_cast<__nv_bfloat16*>(y), mean, rstd, s);
    else
        rc = launch_norm(static_cast<const float*>(x), gamma, beta, T, H, eps, static_cast<float*>(y), mean, rstd, s);
    if (rc != COBALT_OK) return rc;
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

size_t cobalt_layer_norm_workspace_bytes(int64_t T, int32_t H)
{
    if (check_norm(T, H, COBALT_F32) != COBALT_OK) return 0;
    int64_t parts = 0;
    for (int bytes = 2; bytes <= 4; bytes += 2) {        // whichever type needs more
        const int64_t p = norm_parts(T, norm_backward_shape(H, bytes), kMaxSms);
        parts = p > parts ? p : parts;
    }
    return round_up(static_cast<size_t>(parts) * 2 * H * sizeof(float), 256);
}

int cobalt_layer_norm_backward(const void* grad_y, const void* x, const float* gamma, const float* mean, const float* rstd,
                               int64_t T, int32_t H, int32_t dtype, void* grad_x, float* grad_gamma, float* grad_beta,
                               void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    int rc = check_norm(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    if (!gamma || !grad_gamma || !grad_beta || !aligned16(gamma) || !aligned16(grad_gamma) || !aligned16(grad_beta))
        return COBALT_ERR_INVALID_ARG;
    if (T > 0 && (!grad_y || !x || !mean || !rstd || !grad_x)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_y) || !aligned16(x) || !aligned16(mean) || !aligned16(rstd) || !aligned16(grad_x) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cobalt_layer_norm_workspace_bytes(T, H)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    uint32_t* err_word = nullptr;
    rc = device_error_word(&err_word);
    if (rc != COBALT_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    float* partial = static_cast<float*>(workspace);
    int parts = 0;
    if (dtype == COBALT_BF16)
        rc = launch_norm_backward(static_cast<const __nv_bfloat16*>(grad_y), static_cast<const __nv_bfloat16*>(x), gamma, mean, rstd, T, H,
                                  static_cast<__nv_bfloat16*>(grad_x), partial, sms, &parts, err_word, s);
    else
        rc = launch_norm_backward(static_cast<const float*>(grad_y), static_cast<const float*>(x), gamma, mean, rstd, T, H,
                                  static_cast<float*>(grad_x), partial, sms, &parts, err_word, s);
    if (rc != COBALT_OK) return rc;
    COBALT_CUDA_TRY(cudaGetLastError());
    cudaLaunchAttribute attr;
    set_programmatic_launch(&attr, true);
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((2 * H + 31) / 32);
    config.blockDim = dim3(1024);
    config.stream = s;
    config.attrs = &attr;
    config.numAttrs = 1;
    COBALT_CUDA_TRY(cudaLaunchKernelEx(&config, layer_norm_reduce_kernel, static_cast<const float*>(partial), parts, H, grad_gamma, grad_beta));
    return COBALT_OK;
}

}  // extern "C"
