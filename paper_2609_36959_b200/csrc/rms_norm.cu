// Root-mean-square norm of a sum, and its backward pass.
//
//   s = x + r, held in the type of x      rstd = 1 / sqrt(sum s^2 / H + eps)      z = s rstd      y = z gamma
//   g = dy gamma      dx = dr = rstd (g - z mean(g z)) + ds      dgamma = sum_t dy z
//
// r is the residual stream, ds the gradient that comes down it past the norm.  The norm is that of s as it is held, so that
// the backward pass differentiates what the forward pass computed.  y goes out as it is and / or in 8 bits with scales
// (packed.cuh); the backward pass takes s as it is or in 8 bits.  All sums are fp32.
//
// Both directions are bound by HBM: 2 + 2 bytes in and 2 + 2 out a bf16 value forward (one less with 8-bit rows), 6 in and 2 out
// backward.  A row is read once and stays in registers.
#include "packed.cuh"
#include "tcgen05.cuh"

namespace cobalt {

constexpr int kRmsMaxH = 16384;
constexpr int kRmsWarpVecs = 128;            // 16-byte vectors of a row up to which one warp takes it

// The sum over the CTA (kCta; `scratch` 32 floats that no earlier call still reads) or the warp, for every thread.
template <bool kCta>
__device__ __forceinline__ float row_sum(float v, float* scratch)
{
    v = warp_sum(v);
    if (kCta) {
        const int lane = threadIdx.x & 31;
        if (lane == 0) scratch[threadIdx.x >> 5] = v;
        __syncthreads();
        v = warp_sum(lane < (blockDim.x >> 5) ? scratch[lane] : 0.0f);
    }
    return v;
}

struct RmsForward {
    const void* x;
    const void* residual;                    // or null
    const float* gamma;
    int64_t rows;
    int H;
    float eps;
    void* sum;                               // or null
    void* y;                                 // or null
    uint8_t* q;                              // or null
    float* scales;
    int code, group;                         // of q: COBALT_E4M3 or COBALT_I8; 0 (the row) or 128
    float* rstd;                             // or null
};

template <typename Code, int N>
__device__ __forceinline__ void store_group_codes(uint8_t* q, const float (&y)[N], const GroupScale& g)
{
    uint32_t w[N / 4];
#pragma unroll
    for (int k = 0; k < N / 4; ++k) {
        float t[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = g.factor > 0.0f ? y[4 * k + i] * g.factor : 0.0f;
        w[k] = Code::encode4(t);             // y is itself a rounded value: a code at a border may go either way
    }
    if constexpr (N == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
}

// A row a CTA (kCta) or a warp, up to VPT vectors a thread.
template <typename T, int VPT, bool kCta>
__global__ void __launch_bounds__(1024)
rms_norm_kernel(const RmsForward p)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ float scratch[32];
    __shared__ uint32_t scratch_max[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_vec = p.H / N;
    const int first = kCta ? threadIdx.x : lane, step = kCta ? blockDim.x : 32;
    const int64_t row = kCta ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * (blockDim.x >> 5) + warp;
    if (row >= p.rows) return;
    const int64_t at_row = row * p.H;
    const T *x = static_cast<const T*>(p.x) + at_row, *residual = static_cast<const T*>(p.residual) + at_row;
    uint4 v[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = first + i * step;
        v[i] = make_uint4(0, 0, 0, 0);
        if (at < n_vec) v[i] = ld_once16(x + at * N);
    }
    if (p.residual) {
        uint4 r[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            r[i] = make_uint4(0, 0, 0, 0);
            if (at < n_vec) r[i] = ld_once16(residual + at * N);
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            float a[N], b[N];
            Vec16<T>::unpack(v[i], a);
            Vec16<T>::unpack(r[i], b);
#pragma unroll
            for (int k = 0; k < N; ++k) a[k] += b[k];
            v[i] = Vec16<T>::pack(a);
            if (p.sum && at < n_vec) st_stream16(static_cast<T*>(p.sum) + at_row + at * N, v[i]);
        }
    }
    float squares = 0.0f;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float f[N];
        Vec16<T>::unpack(v[i], f);
#pragma unroll
        for (int k = 0; k < N; ++k) squares = fmaf(f[k], f[k], squares);
    }
    const float rstd = rsqrtf(row_sum<kCta>(squares, scratch) / static_cast<float>(p.H) + p.eps);
    if (p.rstd && first == 0) p.rstd[row] = rstd;

    GroupScale own = {};
    if (p.q && p.group == 0) {               // the row's scale ahead of its codes
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float f[N];
            Vec16<T>::unpack(v[i], f);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 g = __ldg(reinterpret_cast<const float4*>(p.gamma + at * N + k));
                most = abs_max(abs_max(abs_max(abs_max(most, f[k] * rstd * g.x), f[k + 1] * rstd * g.y), f[k + 2] * rstd * g.z), f[k + 3] * rstd * g.w);
            }
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        if (kCta) {
            if (lane == 0) scratch_max[warp] = most;
            __syncthreads();
            most = __reduce_max_sync(0xFFFFFFFFu, lane < (blockDim.x >> 5) ? scratch_max[lane] : 0u);
        }
        own = p.code == COBALT_E4M3 ? GroupScale::of<CodeE4M3>(most) : GroupScale::of<CodeI8>(most);
        if (first == 0) p.scales[row] = own.scale;
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = first + i * step;
        const bool mine = at < n_vec;
        float f[N];
        Vec16<T>::unpack(v[i], f);
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const float4 g = mine ? __ldg(reinterpret_cast<const float4*>(p.gamma + at * N + k)) : make_float4(0, 0, 0, 0);
            f[k] = f[k] * rstd * g.x;
            f[k + 1] = f[k + 1] * rstd * g.y;
            f[k + 2] = f[k + 2] * rstd * g.z;
            f[k + 3] = f[k + 3] * rstd * g.w;
        }
        if (mine && p.y) st_stream16(static_cast<T*>(p.y) + at_row + at * N, Vec16<T>::pack(f));
        if (p.q) {
            GroupScale g = own;
            if (p.group != 0) {              // 128 columns: neighbouring lanes, all of them here
                uint32_t most = 0;
#pragma unroll
                for (int k = 0; k < N; ++k) most = mine ? abs_max(most, f[k]) : 0u;
#pragma unroll
                for (int off = 1; off < kPackGroup / N; off <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, off));
                g = p.code == COBALT_E4M3 ? GroupScale::of<CodeE4M3>(most) : GroupScale::of<CodeI8>(most);
                if (mine && at % (kPackGroup / N) == 0) p.scales[row * ((p.H + kPackGroup - 1) / kPackGroup) + at / (kPackGroup / N)] = g.scale;
            }
            if (mine) {
                uint8_t* q = p.q + at_row + at * N;
                if (p.code == COBALT_E4M3) store_group_codes<CodeE4M3>(q, f, g);
                else store_group_codes<CodeI8>(q, f, g);
            }
        }
    }
}

struct RmsBackward {
    const void* grad_y;
    const void* grad_sum;                    // or null
    const void* rows_in;                     // s, as T or as codes
    const float* scales;                     // of the codes
    int groups;                              // scales of a row
    const float* gamma;
    const float* rstd;
    int64_t rows;
    int H;
    void* grad_x;
    float* partial;                          // [CTAs][H]
};

// A vector's worth of s.
template <typename T, typename Code>
struct SavedRows {
    static constexpr int N = Vec16<T>::kElems;
    uint32_t w[N / 4];
    float scale;
    __device__ __forceinline__ void load(const RmsBackward& p, int64_t row, int at)
    {
        const uint8_t* from = static_cast<const uint8_t*>(p.rows_in) + row * p.H + at * N;
        if constexpr (N == 8) {
            const uint2 v = __ldcs(reinterpret_cast<const uint2*>(from));
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = __ldcs(reinterpret_cast<const uint32_t*>(from));
        }
        scale = __ldg(p.scales + row * p.groups + (p.groups > 1 ? at * N / kPackGroup : 0));
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w[i] = 0;
        scale = 0.0f;
    }
    __device__ __forceinline__ void values(float (&f)[N]) const
    {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            float e[4];
            Code::decode4(w[i], e);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[4 * i + k] = e[k] * scale;
        }
    }
};

template <typename T>
struct SavedRows<T, void> {
    static constexpr int N = Vec16<T>::kElems;
    uint4 v;
    __device__ __forceinline__ void load(const RmsBackward& p, int64_t row, int at) { v = ld_once16(static_cast<const T*>(p.rows_in) + row * p.H + at * N); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void values(float (&f)[N]) const { Vec16<T>::unpack(v, f); }
};

// Persistent CTAs; a thread has the same columns of every row, whose gradients of gamma stay in its registers.
template <typename T, typename Code, int VPT, bool kCta>
__global__ void __launch_bounds__(kCta ? 1024 : 256)
rms_norm_backward_kernel(const RmsBackward p)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ float scratch[2][32];
    extern __shared__ float warp_sums[];     // [H], one warp a row only
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_vec = p.H / N;
    const int first = kCta ? threadIdx.x : lane, step = kCta ? blockDim.x : 32;
    const int64_t rows_step = kCta ? gridDim.x : static_cast<int64_t>(gridDim.x) * (blockDim.x >> 5);
    int64_t row = kCta ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * (blockDim.x >> 5) + warp;
    const float inv_h = 1.0f / static_cast<float>(p.H);
    launch_dependents();
    float acc[VPT][N];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int k = 0; k < N; ++k) acc[i][k] = 0.0f;
    int turn = 0;
    for (; row < p.rows; row += rows_step, turn ^= 1) {
        uint4 dy[VPT], ds[VPT];
        SavedRows<T, Code> s[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            dy[i] = make_uint4(0, 0, 0, 0);
            s[i].clear();
            if (at < n_vec) {
                dy[i] = ld_once16(static_cast<const T*>(p.grad_y) + row * p.H + at * N);
                s[i].load(p, row, at);
            }
        }
        const float rstd = __ldg(p.rstd + row);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            ds[i] = make_uint4(0, 0, 0, 0);
            if (p.grad_sum && at < n_vec) ds[i] = ld_once16(static_cast<const T*>(p.grad_sum) + row * p.H + at * N);
        }
        float dot = 0.0f;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float z[N], d[N];
            s[i].values(z);
            Vec16<T>::unpack(dy[i], d);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 g = __ldg(reinterpret_cast<const float4*>(p.gamma + at * N + k));
                const float gm[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float dz = d[k + j] * (z[k + j] * rstd);
                    acc[i][k + j] += dz;
                    dot = fmaf(dz, gm[j], dot);
                }
            }
        }
        const float mean = row_sum<kCta>(dot, scratch[turn]) * inv_h;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float z[N], d[N], e[N];
            s[i].values(z);
            Vec16<T>::unpack(dy[i], d);
            Vec16<T>::unpack(ds[i], e);
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 g = __ldg(reinterpret_cast<const float4*>(p.gamma + at * N + k));
                const float gm[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) d[k + j] = fmaf(rstd, fmaf(-mean, z[k + j] * rstd, d[k + j] * gm[j]), e[k + j]);
            }
            st_stream16(static_cast<T*>(p.grad_x) + row * p.H + at * N, Vec16<T>::pack(d));
        }
    }
    float* out = p.partial + static_cast<int64_t>(blockIdx.x) * p.H;
    if (kCta) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
#pragma unroll
            for (int k = 0; k < N; k += 4)
                *reinterpret_cast<float4*>(out + at * N + k) = make_float4(acc[i][k], acc[i][k + 1], acc[i][k + 2], acc[i][k + 3]);
        }
    } else {
        for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {          // the warps one after the other: a fixed order
            if (warp == w) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int at = first + i * step;
                    if (at >= n_vec) continue;
#pragma unroll
                    for (int k = 0; k < N; ++k) warp_sums[at * N + k] = (w > 0 ? warp_sums[at * N + k] : 0.0f) + acc[i][k];
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < p.H; c += blockDim.x) out[c] = warp_sums[c];
    }
}

// grad_gamma: column sums of the parts, 32 columns a CTA, every warp a slice of the parts.
__global__ void __launch_bounds__(1024)
rms_norm_reduce_kernel(const float* partial, int parts, int H, float* __restrict__ grad_gamma)
{
    wait_for_prior_kernel();                             // the parts
    __shared__ float slice[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < H) {
#pragma unroll 4
        for (int p = warp; p < parts; p += 32) s += partial[static_cast<int64_t>(p) * H + col];
    }
    slice[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < H) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += slice[i][lane];
        grad_gamma[col] = total;
    }
}

struct RmsShape {
    int vpt, threads, resident;              // resident: CTAs an SM (backward)
    bool cta;
};

static RmsShape rms_shape(int n_vec)
{
    RmsShape s = {};
    s.cta = n_vec > kRmsWarpVecs;
    if (!s.cta) {
        s.threads = 256;
        s.vpt = n_vec <= 32 ? 1 : n_vec <= 64 ? 2 : 4;
        s.resident = 4;
    } else {
        s.vpt = n_vec <= 1024 ? 2 : 4;
        s.threads = ((n_vec + s.vpt - 1) / s.vpt + 31) / 32 * 32;
        s.resident = 1024 / s.threads > 4 ? 4 : 1024 / s.threads < 1 ? 1 : 1024 / s.threads;
    }
    return s;
}

constexpr int kMaxSms = 256;                 // the workspace query knows no device: sized for this many

static int64_t rms_parts(int64_t T, const RmsShape& s, int sms)
{
    const int64_t rows = s.cta ? 1 : s.threads / 32;
    int64_t ctas = (T + rows - 1) / rows;
    if (ctas > static_cast<int64_t>(s.resident) * sms) ctas = static_cast<int64_t>(s.resident) * sms;
    return ctas < 1 ? 1 : ctas;              // no rows: one part of zeros
}

static int check_rms(int64_t T, int32_t H, int32_t dtype)
{
    if (T < 0 || H < 1 || (dtype != COBALT_BF16 && dtype != COBALT_F32)) return COBALT_ERR_INVALID_ARG;
    if (H % 8 != 0 || H > kRmsMaxH || T >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

static bool check_code(int32_t code, int32_t group) { return (code == COBALT_E4M3 || code == COBALT_I8) && (group == 0 || group == kPackGroup); }

template <typename T>
static void launch_forward(const RmsForward& p, cudaStream_t s)
{
    const RmsShape shape = rms_shape(p.H / Vec16<T>::kElems);
    const int64_t per_cta = shape.cta ? 1 : shape.threads / 32;
    const unsigned grid = static_cast<unsigned>((p.rows + per_cta - 1) / per_cta);
    if (shape.cta) {
        if (shape.vpt == 2) rms_norm_kernel<T, 2, true><<<grid, shape.threads, 0, s>>>(p);
        else rms_norm_kernel<T, 4, true><<<grid, shape.threads, 0, s>>>(p);
    } else {
        if (shape.vpt == 1) rms_norm_kernel<T, 1, false><<<grid, shape.threads, 0, s>>>(p);
        else if (shape.vpt == 2) rms_norm_kernel<T, 2, false><<<grid, shape.threads, 0, s>>>(p);
        else rms_norm_kernel<T, 4, false><<<grid, shape.threads, 0, s>>>(p);
    }
}

template <typename T, typename Code>
static int launch_backward(const RmsBackward& p, int sms, cudaStream_t s)
{
    const RmsShape shape = rms_shape(p.H / Vec16<T>::kElems);
    const int parts = static_cast<int>(rms_parts(p.rows, shape, sms < kMaxSms ? sms : kMaxSms));
    const size_t smem = shape.cta ? 0 : sizeof(float) * p.H;
    if (shape.cta) {
        if (shape.vpt == 2) rms_norm_backward_kernel<T, Code, 2, true><<<parts, shape.threads, smem, s>>>(p);
        else rms_norm_backward_kernel<T, Code, 4, true><<<parts, shape.threads, smem, s>>>(p);
    } else {
        if (shape.vpt == 1) rms_norm_backward_kernel<T, Code, 1, false><<<parts, shape.threads, smem, s>>>(p);
        else if (shape.vpt == 2) rms_norm_backward_kernel<T, Code, 2, false><<<parts, shape.threads, smem, s>>>(p);
        else rms_norm_backward_kernel<T, Code, 4, false><<<parts, shape.threads, smem, s>>>(p);
    }
    return parts;
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_rms_norm(const void* x, const void* residual, const float* gamma, int64_t T, int32_t H, int32_t dtype, float eps, void* sum,
                    void* y, void* q, float* q_scales, int32_t q_code, int32_t q_group, float* rstd, cobalt_stream_t stream)
{
    int rc = check_rms(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    if (!(eps >= 0.0f) || (q && !check_code(q_code, q_group)) || (!residual && sum)) return COBALT_ERR_INVALID_ARG;
    if (T == 0) return COBALT_OK;
    if (!x || !gamma || (!y && !q) || (q && !q_scales)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(gamma) || !aligned16(sum) || !aligned16(y) || !aligned16(q) ||
        !aligned16(q_scales) || !aligned16(rstd))
        return COBALT_ERR_INVALID_ARG;
    const RmsForward p = {x, residual, gamma, T, H, eps, sum, y, static_cast<uint8_t*>(q), q_scales, q_code, q_group, rstd};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16) launch_forward<__nv_bfloat16>(p, s);
    else launch_forward<float>(p, s);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

size_t cobalt_rms_norm_workspace_bytes(int64_t T, int32_t H)
{
    if (check_rms(T, H, COBALT_F32) != COBALT_OK) return 0;
    int64_t parts = 0;
    for (int elems = 4; elems <= 8; elems += 4) {        // whichever type needs more
        const int64_t p = rms_parts(T, rms_shape(H / elems), kMaxSms);
        parts = p > parts ? p : parts;
    }
    return round_up(static_cast<size_t>(parts) * H * sizeof(float), 256);
}

int cobalt_rms_norm_backward(const void* grad_y, const void* grad_sum, const void* rows, const float* row_scales, int32_t rows_type,
                             int32_t group, const float* gamma, const float* rstd, int64_t T, int32_t H, int32_t dtype, void* grad_x,
                             float* grad_gamma, void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    int rc = check_rms(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    const bool packed = rows_type != dtype;
    if (packed && !check_code(rows_type, group)) return COBALT_ERR_INVALID_ARG;
    if (!gamma || !grad_gamma || (T > 0 && (!grad_y || !rows || !rstd || !grad_x || (packed && !row_scales)))) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_y) || !aligned16(grad_sum) || !aligned16(rows) || !aligned16(row_scales) || !aligned16(gamma) || !aligned16(rstd) ||
        !aligned16(grad_x) || !aligned16(grad_gamma) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cobalt_rms_norm_workspace_bytes(T, H)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    const RmsBackward p = {grad_y, grad_sum, rows, row_scales, group == 0 ? 1 : (H + kPackGroup - 1) / kPackGroup, gamma, rstd, T, H, grad_x,
                           static_cast<float*>(workspace)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int parts = 0;
    if (dtype == COBALT_BF16)
        parts = !packed ? launch_backward<__nv_bfloat16, void>(p, sms, s)
                        : rows_type == COBALT_I8 ? launch_backward<__nv_bfloat16, CodeI8>(p, sms, s) : launch_backward<__nv_bfloat16, CodeE4M3>(p, sms, s);
    else
        parts = !packed ? launch_backward<float, void>(p, sms, s)
                        : rows_type == COBALT_I8 ? launch_backward<float, CodeI8>(p, sms, s) : launch_backward<float, CodeE4M3>(p, sms, s);
    COBALT_CUDA_TRY(cudaGetLastError());
    cudaLaunchAttribute attr;
    set_programmatic_launch(&attr, true);
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((H + 31) / 32);
    config.blockDim = dim3(1024);
    config.stream = s;
    config.attrs = &attr;
    config.numAttrs = 1;
    COBALT_CUDA_TRY(cudaLaunchKernelEx(&config, rms_norm_reduce_kernel, static_cast<const float*>(p.partial), parts, H, grad_gamma));
    return COBALT_OK;
}

}  // extern "C"
