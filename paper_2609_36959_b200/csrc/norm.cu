// Layer norm over the H columns of each row, its backward pass and the reduction of its weights' gradients.
//
//   mu = sum x / H    var = sum (x - mu)^2 / H    rstd = 1 / sqrt(var + eps)    z = (x - mu) rstd
//   y  = z gamma + beta
//   g  = dy gamma     dx = rstd (g - mean(g) - z mean(g z))      dgamma = sum_t dy z     dbeta = sum_t dy
//
// A row is read once and stays in registers, so the variance is the sum of squares about the mean and not a
// difference of two large sums.  All sums are fp32.  A group of threads owns a row: one warp while a lane needs at
// most four 16-byte vectors, the whole CTA above that.
//
// Backward: a thread owns the same columns of every row that its group takes, so the weights' gradients add up in
// registers over the rows; each CTA writes one partial sum a column, and a second kernel adds the partials in a
// fixed order (no atomics: the result does not vary from run to run).
#include "numeric.cuh"

namespace cobalt {

constexpr int kNormMaxH = 16384;
constexpr int kWarpRowVecs = 128;        // 16-byte vectors of a row up to which one warp takes it
constexpr int kWarpRowThreads = 256;

// Sum of `v` and `w` over the threads that share a row.
template <bool kCta>
__device__ __forceinline__ float2 row_sum2(float v, float w, float2* scratch)
{
    v = warp_sum(v);
    w = warp_sum(w);
    if (!kCta) return make_float2(v, w);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if (lane == 0) scratch[warp] = make_float2(v, w);
    __syncthreads();
    const float2 p = lane < warps ? scratch[lane] : make_float2(0.0f, 0.0f);
    return make_float2(warp_sum(p.x), warp_sum(p.y));
}

template <typename T, int VPT, bool kCta>
__global__ void __launch_bounds__(1024)
layer_norm_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t rows,
                  int H, float eps, T* y, float* __restrict__ mean, float* __restrict__ rstd)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ float2 scratch[2][32];
    const int group = kCta ? blockDim.x : 32, lane = kCta ? threadIdx.x : (threadIdx.x & 31);
    const int groups = kCta ? 1 : (blockDim.x >> 5), own = kCta ? 0 : (threadIdx.x >> 5);
    const int n_vec = H / N;
    const float h = static_cast<float>(H);
    const int64_t r = static_cast<int64_t>(blockIdx.x) * groups + own;
    if (r >= rows) return;
    const T* row = x + r * H;
    uint4 v[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * group;
        if (at < n_vec) v[i] = ld_once16(row + at * N);
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if (lane + i * group < n_vec) {
            float f[N];
            Vec16<T>::unpack(v[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += f[k];
        }
    }
    const float mu = row_sum2<kCta>(sum, 0.0f, scratch[0]).x / h;   // a division: a constant row has z = 0 exactly
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        if (lane + i * group < n_vec) {
            float f[N];
            Vec16<T>::unpack(v[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) sq = fmaf(f[k] - mu, f[k] - mu, sq);
        }
    }
    const float rs = 1.0f / sqrtf(row_sum2<kCta>(sq, 0.0f, scratch[1]).x / h + eps);
    if (lane == 0) {
        mean[r] = mu;
        rstd[r] = rs;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * group;
        if (at < n_vec) {
            float f[N];
            Vec16<T>::unpack(v[i], f);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 g = __ldg(reinterpret_cast<const float4*>(gamma + at * N + k));
                const float4 b = __ldg(reinterpret_cast<const float4*>(beta + at * N + k));
                f[k] = fmaf((f[k] - mu) * rs, g.x, b.x);
                f[k + 1] = fmaf((f[k + 1] - mu) * rs, g.y, b.y);
                f[k + 2] = fmaf((f[k + 2] - mu) * rs, g.z, b.z);
                f[k + 3] = fmaf((f[k + 3] - mu) * rs, g.w, b.w);
            }
            st_stream16(y + r * H + at * N, Vec16<T>::pack(f));
        }
    }
}

// partial: [parts][2][H], one part a group of threads.
template <typename T, int VPT, bool kCta>
__global__ void __launch_bounds__(kCta ? 1024 : kWarpRowThreads)
layer_norm_backward_kernel(const T* grad_y, const T* __restrict__ x, const float* __restrict__ gamma,
                           const float* __restrict__ mean, const float* __restrict__ rstd, int64_t rows, int H,
                           T* grad_x, float* __restrict__ partial)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ float2 scratch[2][32];
    const int group = kCta ? blockDim.x : 32, lane = kCta ? threadIdx.x : (threadIdx.x & 31);
    const int groups = kCta ? 1 : (blockDim.x >> 5), own = kCta ? 0 : (threadIdx.x >> 5);
    const int n_vec = H / N;
    const float inv_h = 1.0f / static_cast<float>(H);
    const int64_t part = static_cast<int64_t>(blockIdx.x) * groups + own, parts = static_cast<int64_t>(gridDim.x) * groups;
    float gm[VPT][N], dg[VPT][N], db[VPT][N];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * group;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            gm[i][k] = at < n_vec ? __ldg(gamma + at * N + k) : 0.0f;
            dg[i][k] = 0.0f;
            db[i][k] = 0.0f;
        }
    }
    int turn = 0;
    for (int64_t r = part; r < rows; r += parts) {
        uint4 xv[VPT], yv[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = lane + i * group;
            if (at < n_vec) {
                xv[i] = ld_once16(x + r * H + at * N);
                yv[i] = ld_once16(grad_y + r * H + at * N);
            }
        }
        const float mu = __ldg(mean + r), rs = __ldg(rstd + r);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (lane + i * group < n_vec) {
                float z[N], d[N];
                Vec16<T>::unpack(xv[i], z);
                Vec16<T>::unpack(yv[i], d);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float zz = (z[k] - mu) * rs, g = d[k] * gm[i][k];
                    s1 += g;
                    s2 = fmaf(g, zz, s2);
                    dg[i][k] = fmaf(d[k], zz, dg[i][k]);
                    db[i][k] += d[k];
                }
            }
        }
        const float2 s = row_sum2<kCta>(s1, s2, scratch[turn]);
        turn ^= 1;                       // the next row's sums go to the other half: one barrier a row is enough
        const float c1 = s.x * inv_h, c2 = s.y * inv_h;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = lane + i * group;
            if (at < n_vec) {
                float z[N], d[N];
                Vec16<T>::unpack(xv[i], z);
                Vec16<T>::unpack(yv[i], d);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float zz = (z[k] - mu) * rs;
                    d[k] = rs * (fmaf(d[k], gm[i][k], -c1) - zz * c2);
                }
                st_stream16(grad_x + r * H + at * N, Vec16<T>::pack(d));
            }
        }
    }
    float* out = partial + part * 2 * H;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = lane + i * group;
        if (at < n_vec) {
#pragma unroll
            for (int k = 0; k < N; ++k) {
                out[at * N + k] = dg[i][k];
                out[H + at * N + k] = db[i][k];
            }
        }
    }
}

// grad_gamma and grad_beta: column sums of the parts, 32 columns a CTA, every warp a slice of the parts.
__global__ void __launch_bounds__(256)
layer_norm_reduce_kernel(const float* __restrict__ partial, int parts, int H, float* __restrict__ grad_gamma,
                         float* __restrict__ grad_beta)
{
    __shared__ float slice[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int col = blockIdx.x * 32 + lane;              // over 2H columns: gamma's, then beta's
    float s = 0.0f;
    if (col < 2 * H)
        for (int p = warp; p < parts; p += 8) s += partial[static_cast<int64_t>(p) * 2 * H + col];
    slice[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < 2 * H) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) total += slice[i][lane];
        if (col < H) grad_gamma[col] = total;
        else grad_beta[col - H] = total;
    }
}

// How the rows are dealt to threads: vectors a thread holds, threads of a CTA, whether a CTA owns a row.
struct NormShape {
    int vpt, threads;
    bool cta;
};

static NormShape norm_shape(int n_vec)
{
    NormShape s;
    s.cta = n_vec > kWarpRowVecs;
    if (!s.cta) {
        s.threads = kWarpRowThreads;
        s.vpt = n_vec <= 32 ? 1 : n_vec <= 64 ? 2 : 4;
    } else {
        s.vpt = n_vec <= 1024 ? 1 : n_vec <= 2048 ? 2 : 4;
        s.threads = ((n_vec + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    }
    return s;
}

// Parts (= row groups in flight) of the backward kernel.
static int64_t norm_parts(int64_t rows, const NormShape& s, int sms)
{
    const int64_t groups = s.cta ? 1 : s.threads / 32;
    const int64_t resident = s.cta ? (s.threads <= 512 ? 4 : 2) : 2;
    int64_t ctas = (rows + groups - 1) / groups;
    if (ctas > resident * sms) ctas = resident * sms;
    if (ctas < 1) ctas = 1;
    return ctas * groups;
}

constexpr int kMaxSms = 256;             // the workspace query knows no device: sized for this many

#define COBALT_NORM_CASES(T, CALL)                        \
    do {                                                  \
        if (shape.cta) {                                  \
            if (shape.vpt == 1) CALL(T, 1, true);         \
            else if (shape.vpt == 2) CALL(T, 2, true);    \
            else CALL(T, 4, true);                        \
        } else {                                          \
            if (shape.vpt == 1) CALL(T, 1, false);        \
            else if (shape.vpt == 2) CALL(T, 2, false);   \
            else CALL(T, 4, false);                       \
        }                                                 \
    } while (0)

static int check_norm(int64_t T, int32_t H, int32_t dtype)
{
    if (T < 0 || H < 1 || (dtype != COBALT_BF16 && dtype != COBALT_F32)) return COBALT_ERR_INVALID_ARG;
    if (H % 8 != 0 || H > kNormMaxH || T >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_layer_norm(const void* x, const float* gamma, const float* beta, int64_t T, int32_t H, int32_t dtype, float eps,
                      void* y, float* mean, float* rstd, cobalt_stream_t stream)
{
    const int rc = check_norm(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    if (!(eps >= 0.0f)) return COBALT_ERR_INVALID_ARG;
    if (T == 0) return COBALT_OK;
    if (!x || !gamma || !beta || !y || !mean || !rstd || !aligned16(x) || !aligned16(gamma) || !aligned16(beta) ||
        !aligned16(y) || !aligned16(mean) || !aligned16(rstd))
        return COBALT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormShape shape = norm_shape(H / (dtype == COBALT_BF16 ? 8 : 4));
    const int64_t groups = shape.cta ? 1 : shape.threads / 32;
    const unsigned grid = static_cast<unsigned>((T + groups - 1) / groups);
#define COBALT_NORM_FWD(TT, VPT, CTA)                                                                            \
    layer_norm_kernel<TT, VPT, CTA><<<grid, shape.threads, 0, s>>>(static_cast<const TT*>(x), gamma, beta, T, H, eps, \
                                                                   static_cast<TT*>(y), mean, rstd)
    if (dtype == COBALT_BF16) COBALT_NORM_CASES(__nv_bfloat16, COBALT_NORM_FWD);
    else COBALT_NORM_CASES(float, COBALT_NORM_FWD);
#undef COBALT_NORM_FWD
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

size_t cobalt_layer_norm_workspace_bytes(int64_t T, int32_t H)
{
    if (check_norm(T, H, COBALT_F32) != COBALT_OK) return 0;
    int64_t parts = 0;
    for (int elems = 4; elems <= 8; elems += 4) {        // whichever type needs more
        const int64_t p = norm_parts(T, norm_shape(H / elems), kMaxSms);
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
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const NormShape shape = norm_shape(H / (dtype == COBALT_BF16 ? 8 : 4));
    const int64_t groups = shape.cta ? 1 : shape.threads / 32;
    const int64_t parts = norm_parts(T, shape, sms < kMaxSms ? sms : kMaxSms);   // no rows: one part of zeros
    const unsigned grid = static_cast<unsigned>(parts / groups);
    float* partial = static_cast<float*>(workspace);
#define COBALT_NORM_BWD(TT, VPT, CTA)                                                                                  \
    layer_norm_backward_kernel<TT, VPT, CTA><<<grid, shape.threads, 0, s>>>(static_cast<const TT*>(grad_y),            \
                                                                            static_cast<const TT*>(x), gamma, mean, rstd, \
                                                                            T, H, static_cast<TT*>(grad_x), partial)
    if (dtype == COBALT_BF16) COBALT_NORM_CASES(__nv_bfloat16, COBALT_NORM_BWD);
    else COBALT_NORM_CASES(float, COBALT_NORM_BWD);
#undef COBALT_NORM_BWD
    COBALT_CUDA_TRY(cudaGetLastError());
    layer_norm_reduce_kernel<<<static_cast<unsigned>((2 * H + 31) / 32), 256, 0, s>>>(partial, static_cast<int>(parts), H,
                                                                                      grad_gamma, grad_beta);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // extern "C"
