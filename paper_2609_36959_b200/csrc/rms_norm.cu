// Root-mean-square norm of a sum, and its backward pass.
//
//   s = x + r, held in the type of x      rstd = 1 / sqrt(sum s^2 / H + eps)      z = s rstd      y = z gamma
//   g = dy gamma      dx = dr = rstd (g - z mean(g z)) + ds      dgamma = sum_t dy z
//
// r is the residual stream, ds the gradient that comes down it past the norm.  The norm is that of s as it is held, so that
// the backward pass differentiates what the forward pass computed.  y goes out as it is and / or in 8 bits with scales
// (packed.cuh); the backward pass takes s as it is or in 8 bits.  All sums are fp32.
//
// A row is read once and stays in registers.  Forward: a warp or a CTA a row, four vectors a thread, so that five or six rows are under
// way on an SM; with 8-bit rows the largest |s gamma| is found beside the sum of squares.  Bound by HBM: 32768 x 7168 bf16 with
// residual 276 us (6.8 TB/s), with e4m3 rows 258 us (6.4 TB/s).  Backward: persistent CTAs, because the gradients of gamma of a thread's
// columns stay in its registers (one partial sum a CTA and column, added in order by a second kernel).  Those registers leave 28 warps
// an SM, so the next row's loads are under way while one is computed: with ds, 8 bytes a value, 303 us (6.2 TB/s, without loads ahead: two
// rows' worth spills), from int8 rows, 5 bytes, 221 us (5.3 TB/s; 267 without loads ahead), with ds 261 us (6.3 TB/s).  A ring of bulk
// copies ahead of the rows was slower (355 and 351 us): reading it back costs instructions, which the row's two passes are short of.
#include <type_traits>

#include "packed.cuh"
#include "tcgen05.cuh"

namespace cobalt {

constexpr int kRmsMaxH = 16384;
constexpr int kRmsWarpVecs = 128;            // 16-byte vectors of a row up to which one warp takes it

// The sum over the CTA (kCta; `scratch` is not still read after an earlier call) or the warp, for every thread.
template <bool kCta>
__device__ __forceinline__ float row_sum(float v, float (&scratch)[32])
{
    v = warp_sum(v);
    if (!kCta) return v;
    const int lane = threadIdx.x & 31;
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < (blockDim.x >> 5) ? scratch[lane] : 0.0f);
}

// N neighbouring values of gamma.  `wide` (a 32-byte boundary): one load of 32 bytes a lane for bf16 rows; two of 16 touch every line
// twice, and gamma is half of what goes through L1.
template <int N>
__device__ __forceinline__ void load_gamma(const float* gamma, bool wide, float (&g)[N])
{
    if (N == 8 && wide) {
        asm volatile("ld.global.nc.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(g[0]), "=f"(g[1]), "=f"(g[2]), "=f"(g[3]), "=f"(g[N - 4]), "=f"(g[N - 3]), "=f"(g[N - 2]), "=f"(g[N - 1])
                     : "l"(gamma));
    } else {
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            const float4 v = __ldg(reinterpret_cast<const float4*>(gamma + k));
            g[k] = v.x, g[k + 1] = v.y, g[k + 2] = v.z, g[k + 3] = v.w;
        }
    }
}

static inline bool on_32_bytes(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

struct RmsForward {
    const void* x;
    const void* residual;                    // or null
    const float* gamma;
    bool wide;                               // gamma on a 32-byte boundary
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

// A row's codes and scales.  sg is y / rstd, which the codes do not depend on; most its largest value.  sg itself is rounded: a code may
// go either way within 2^-22 of a border (six of ten million values; with the doubtful ones done again from sg four, and 312 us instead
// of 257 at 32768 x 7168).
template <typename Code, int N, int VPT>
__device__ __forceinline__ void store_packed(const RmsForward& p, int64_t row, int first, int step, float rstd, const float (&sg)[VPT][N],
                                             const uint32_t (&most)[VPT], uint32_t row_most)
{
    auto scale_of = [rstd](uint32_t bits) {
        GroupScale g = GroupScale::of<Code>(bits);
        const float most_y = g.most * rstd;              // 0, an infinity or NaN: as pack has it for a group of such y
        const bool finite = abs_bits(most_y) < 0x7F800000u;
        g.scale = finite ? fminf(most_y * (1.0f / Code::kLargest), Code::kMostScale) : __uint_as_float(0x7FC00000u);
        if (!finite || most_y == 0.0f) g.factor = 0.0f;
        return g;
    };
    GroupScale g = scale_of(row_most);
    if (p.group == 0 && first == 0) p.scales[row] = g.scale;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = first + i * step;
        if (at >= p.H / N) continue;
        if (p.group != 0) {
            g = scale_of(most[i]);
            if (at % (kPackGroup / N) == 0) p.scales[row * ((p.H + kPackGroup - 1) / kPackGroup) + at / (kPackGroup / N)] = g.scale;
        }
        uint32_t w[N / 4];
        encode_fast<Code>(sg[i], g, w);
        uint8_t* q = p.q + row * p.H + at * N;
        if constexpr (N == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(q) = w[0];
    }
}

// Most threads of a CTA.
template <typename T, int VPT, bool kCta>
constexpr int kRmsThreads = !kCta ? 256 : VPT == 2 ? 448 : sizeof(T) == 4 ? 1024 : 512;

// A row a CTA (kCta) or a warp, up to VPT vectors a thread.
template <typename T, int VPT, bool kCta, bool kPacked>
__global__ void __launch_bounds__(kRmsThreads<T, VPT, kCta>, !kCta ? 4 : VPT == 4 && sizeof(T) == 2 ? 2 : 1)
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
    float squares = 0.0f, sg[kPacked ? VPT : 1][N];
    uint32_t most[kPacked ? VPT : 1], row_most = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        float f[N];
        Vec16<T>::unpack(v[i], f);
#pragma unroll
        for (int k = 0; k < N; ++k) squares = fmaf(f[k], f[k], squares);
        if constexpr (kPacked) {             // the largest |s gamma| too: times rstd it is the largest |y|, and one barrier serves both
            const int at = first + i * step;
            float g[N] = {};
            if (at < n_vec) load_gamma<N>(p.gamma + at * N, p.wide, g);
            most[i] = 0;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                sg[i][k] = f[k] * g[k];
                if (at < n_vec) most[i] = abs_max(most[i], sg[i][k]);
            }
            row_most = max(row_most, most[i]);
        }
    }
    if (kPacked && p.group == 0) {
        row_most = __reduce_max_sync(0xFFFFFFFFu, row_most);
        if (kCta && lane == 0) scratch_max[warp] = row_most;
    }
    squares = row_sum<kCta>(squares, scratch);
    const float rstd = rsqrtf(squares / static_cast<float>(p.H) + p.eps);
    if (p.rstd && first == 0) p.rstd[row] = rstd;

    if constexpr (!kPacked) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float f[N], g[N];
            load_gamma<N>(p.gamma + at * N, p.wide, g);
            Vec16<T>::unpack(v[i], f);
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = f[k] * rstd * g[k];
            st_stream16(static_cast<T*>(p.y) + at_row + at * N, Vec16<T>::pack(f));
        }
    } else {
        if (p.group == 0) {
            if (kCta) row_most = __reduce_max_sync(0xFFFFFFFFu, lane < (blockDim.x >> 5) ? scratch_max[lane] : 0u);
        } else {                             // 128 columns: neighbouring lanes, all of them here
#pragma unroll
            for (int i = 0; i < VPT; ++i)
#pragma unroll
                for (int off = 1; off < kPackGroup / N; off <<= 1) most[i] = max(most[i], __shfl_xor_sync(0xFFFFFFFFu, most[i], off));
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (!p.y || at >= n_vec) continue;
            float y[N];
#pragma unroll
            for (int k = 0; k < N; ++k) y[k] = sg[i][k] * rstd;
            st_stream16(static_cast<T*>(p.y) + at_row + at * N, Vec16<T>::pack(y));
        }
        if (p.code == COBALT_E4M3) store_packed<CodeE4M3, N, VPT>(p, row, first, step, rstd, sg, most, row_most);
        else store_packed<CodeI8, N, VPT>(p, row, first, step, rstd, sg, most, row_most);
    }
}

struct RmsBackward {
    const void* grad_y;
    const void* grad_sum;                    // or null
    const void* rows_in;                     // s, as T or as codes
    const float* scales;                     // of the codes
    int groups;                              // scales of a row
    const float* gamma;
    bool wide;                               // gamma on a 32-byte boundary
    const float* rstd;
    int64_t rows;
    int H;
    void* grad_x;
    float* partial;                          // [CTAs][H]
};

// A vector's worth of s; values() times a factor.
template <typename T, typename Code>
struct SavedRows {
    static constexpr int N = Vec16<T>::kElems;
    uint32_t w[N / 4];
    float scale;
    __device__ __forceinline__ void load(const RmsBackward& p, int64_t row, int at)
    {
        // volatile, like ld_once16: with the row's other loads, not where the compiler first needs them
        const uint8_t* from = static_cast<const uint8_t*>(p.rows_in) + row * p.H + at * N;
        if constexpr (N == 8)
            asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[N / 4 - 1]) : "l"(from));
        else
            asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(from));
        asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(scale) : "l"(p.scales + row * p.groups + (p.groups > 1 ? at * N / kPackGroup : 0)));
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) w[i] = 0;
        scale = 0.0f;
    }
    __device__ __forceinline__ void values(float factor, Pair (&f)[N / 2]) const
    {
        const Pair by = pair(scale * factor);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            float e[4];
            Code::decode4(w[i], e);
            f[2 * i] = pair(e[0], e[1]) * by;
            f[2 * i + 1] = pair(e[2], e[3]) * by;
        }
    }
};

template <typename T>
struct SavedRows<T, void> {
    static constexpr int N = Vec16<T>::kElems;
    uint4 v;
    __device__ __forceinline__ void load(const RmsBackward& p, int64_t row, int at) { v = ld_once16(static_cast<const T*>(p.rows_in) + row * p.H + at * N); }
    __device__ __forceinline__ void clear() { v = make_uint4(0, 0, 0, 0); }
    __device__ __forceinline__ void values(float factor, Pair (&f)[N / 2]) const
    {
        unpack_pairs<T>(v, f);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) f[i] = f[i] * pair(factor);
    }
};

// What a thread has of a row.
template <typename T, typename Code, int VPT, bool kSum>
struct BackwardRow {
    static constexpr int N = Vec16<T>::kElems;
    uint4 dy[VPT], ds[kSum ? VPT : 1];
    SavedRows<T, Code> s[VPT];
    float rstd;
    __device__ __forceinline__ void load(const RmsBackward& p, int64_t row, int first, int step, int n_vec)
    {
        const bool here = row < p.rows;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            dy[i] = make_uint4(0, 0, 0, 0);
            s[i].clear();
            if (here && at < n_vec) {
                dy[i] = ld_once16(static_cast<const T*>(p.grad_y) + row * p.H + at * N);
                s[i].load(p, row, at);
            }
        }
        rstd = here ? __ldg(p.rstd + row) : 0.0f;
    }
    __device__ __forceinline__ void load_sum(const RmsBackward& p, int64_t row, int first, int step, int n_vec)
    {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            ds[kSum ? i : 0] = make_uint4(0, 0, 0, 0);
            if (row < p.rows && at < n_vec) ds[kSum ? i : 0] = ld_once16(static_cast<const T*>(p.grad_sum) + row * p.H + at * N);
        }
    }
};

// Persistent CTAs; a thread has the same columns of every row, whose gradients of gamma stay in its registers.  kAhead: the next
// row's loads (the second gradient's own at the row's start: it is needed last) are under way while one is computed.
template <typename T, typename Code, int VPT, bool kCta, bool kSum, bool kAhead, int kThreads>
__global__ void __launch_bounds__(kThreads, !kCta && VPT == 1 ? 4 : kThreads <= 448 ? 2 : 1)
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
    Pair acc[VPT][N / 2];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int k = 0; k < N / 2; ++k) acc[i][k] = pair(0.0f);
    BackwardRow<T, Code, VPT, kSum> in, ahead;
    if (kAhead) ahead.load(p, row, first, step, n_vec);
    for (int turn = 0; row < p.rows; row += rows_step, turn ^= 1) {
        if (kAhead) in = ahead;
        else in.load(p, row, first, step, n_vec);
        if (kSum) in.load_sum(p, row, first, step, n_vec);
        if (kAhead) ahead.load(p, row + rows_step, first, step, n_vec);
        Pair dot = pair(0.0f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float gm[N];
            Pair z[N / 2], d[N / 2];
            load_gamma<N>(p.gamma + at * N, p.wide, gm);
            in.s[i].values(in.rstd, z);
            unpack_pairs<T>(in.dy[i], d);
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                const Pair dz = d[k] * z[k];
                acc[i][k] = acc[i][k] + dz;
                dot = fma2(dz, pair(gm[2 * k], gm[2 * k + 1]), dot);
            }
        }
        const float minus_mean = -row_sum<kCta>(dot.v.x + dot.v.y, scratch[turn]) * inv_h;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int at = first + i * step;
            if (at >= n_vec) continue;
            float gm[N];
            Pair z[N / 2], d[N / 2], e[N / 2];
            load_gamma<N>(p.gamma + at * N, p.wide, gm);
            in.s[i].values(in.rstd, z);
            unpack_pairs<T>(in.dy[i], d);
            if (kSum) unpack_pairs<T>(in.ds[kSum ? i : 0], e);
#pragma unroll
            for (int k = 0; k < N / 2; ++k) {
                const Pair v = fma2(pair(minus_mean), z[k], d[k] * pair(gm[2 * k], gm[2 * k + 1]));
                d[k] = kSum ? fma2(pair(in.rstd), v, e[k]) : pair(in.rstd) * v;
            }
            st_stream16(static_cast<T*>(p.grad_x) + row * p.H + at * N, pack_pairs<T>(d));
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
                *reinterpret_cast<float4*>(out + at * N + k) = 
                    make_float4(acc[i][k / 2].v.x, acc[i][k / 2].v.y, acc[i][k / 2 + 1].v.x, acc[i][k / 2 + 1].v.y);
        }
    } else {
        for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) {          // the warps one after the other: a fixed order
            if (warp == w) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) {
                    const int at = first + i * step;
                    if (at >= n_vec) continue;
#pragma unroll
                    for (int k = 0; k < N; ++k) 
                        warp_sums[at * N + k] = (w > 0 ? warp_sums[at * N + k] : 0.0f) + (k & 1 ? acc[i][k / 2].v.y : acc[i][k / 2].v.x);
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
#pragma unroll 8
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
    int vpt, threads;
    bool cta;
    int resident;                            // CTAs of the backward kernels that fit on an SM
};

// Vectors up to which the forward pass takes two a thread instead of four: more threads for a row where its latency counts, and narrow rows
// keep more of them under way.  Two / four, us: 500 x 2048 bf16 with residual 3.5 / 4.0, to e4m3 rows 3.9 / 4.5; 4999 x 2048 14.6 / 14.8 and
// 16.2 / 17.0; 1000 x 7168 11.4 / 11.9 and 14.2 / 13.8; 32768 x 7168 273 / 275 and 312 / 258; 65536 x 2048 161 / 161 and 152 / 146.
static bool few_vectors(int64_t rows, int n_vec) { return rows * n_vec <= (n_vec <= 256 ? 1 << 21 : 1 << 19); }

// A warp a row up to 128 vectors; above, a CTA a row with `vpt` vectors a thread, four of rows of more than `most`.  elems: values of a
// vector.
static RmsShape rms_shape(int H, int elems, int vpt, int most)
{
    const int n_vec = H / elems;
    RmsShape s = {};
    s.cta = n_vec > kRmsWarpVecs;
    if (!s.cta) {
        s.threads = 256;
        s.vpt = n_vec <= 32 ? 1 : n_vec <= 64 ? 2 : 4;
    } else {
        s.vpt = n_vec <= most ? vpt : 4;
        s.threads = ((n_vec + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    }
    // by the registers that the launch bounds leave a thread: a CTA too many would wait for a whole one (32768 x 4096 bf16 with a second
    // gradient, where three fit: 181 us, with four 234)
    const int registers = s.cta ? (s.threads <= 448 && s.vpt == 2 ? 72 : 64) : s.vpt == 1 ? 64 : 128;
    s.resident = 65536 / (registers * s.threads);
    if (s.resident > 8) s.resident = 8;
    return s;
}

constexpr int kMaxSms = 256;                 // the workspace query knows no device: sized for this many

// CTAs (= partial sums) of the backward kernels: as many as fit, and four rows each where there are that many.
static int64_t rms_parts(int64_t T, const RmsShape& s, int sms)
{
    const int64_t rows = s.cta ? 1 : s.threads / 32;
    int64_t ctas = (T + rows - 1) / rows, most = static_cast<int64_t>(s.resident) * sms, by_rows = (ctas + 3) / 4;
    if (by_rows < sms) by_rows = sms;
    if (most > by_rows) most = by_rows;
    if (ctas > most) ctas = most;
    return ctas < 1 ? 1 : ctas;              // no rows: one part of zeros
}

static int check_rms(int64_t T, int32_t H, int32_t dtype)
{
    if (T < 0 || H < 1 || (dtype != COBALT_BF16 && dtype != COBALT_F32)) return COBALT_ERR_INVALID_ARG;
    if (H % 8 != 0 || H > kRmsMaxH || T >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

static bool check_code(int32_t code, int32_t group) { return (code == COBALT_E4M3 || code == COBALT_I8) && (group == 0 || group == kPackGroup); }

template <typename T, bool kPacked>
static void launch_forward(const RmsForward& p, cudaStream_t s)
{
    const RmsShape shape = rms_shape(p.H, Vec16<T>::kElems, few_vectors(p.rows, p.H / Vec16<T>::kElems) ? 2 : 4, 896);
    const int64_t per_cta = shape.cta ? 1 : shape.threads / 32, ctas = (p.rows + per_cta - 1) / per_cta;
    const unsigned grid = static_cast<unsigned>(ctas);
    if (shape.cta) {
        if (shape.vpt == 2) rms_norm_kernel<T, 2, true, kPacked><<<grid, shape.threads, 0, s>>>(p);
        else rms_norm_kernel<T, 4, true, kPacked><<<grid, shape.threads, 0, s>>>(p);
    } else {
        if (shape.vpt == 1) rms_norm_kernel<T, 1, false, kPacked><<<grid, shape.threads, 0, s>>>(p);
        else if (shape.vpt == 2) rms_norm_kernel<T, 2, false, kPacked><<<grid, shape.threads, 0, s>>>(p);
        else rms_norm_kernel<T, 4, false, kPacked><<<grid, shape.threads, 0, s>>>(p);
    }
}

// *parts: the kernel's partial sums.
template <typename T, typename Code, bool kSum>
static int launch_backward(const RmsBackward& p, int sms, int* parts, cudaStream_t s)
{
    const RmsShape shape = rms_shape(p.H, Vec16<T>::kElems, 2, 2048);
    *parts = static_cast<int>(rms_parts(p.rows, shape, sms < kMaxSms ? sms : kMaxSms));
    // The next row's loads ahead, but where their registers spill (32768 x 7168 bf16, us, with / without: rows as they are 224 / 260 without a
    // second gradient, 312 / 304 with one; rows in 8 bits 221 / 267 and 261 / 304; 32768 x 8192: 281 / 287, 337 / 338, 250 / 324, 375 / 331).
    constexpr bool kPlain = std::is_void<Code>::value;
    const size_t smem = shape.cta ? 0 : sizeof(float) * p.H;
    if (shape.cta) {
        if (sizeof(T) == 4 && shape.vpt == 4) rms_norm_backward_kernel<float, Code, 4, true, kSum, false, 1024><<<*parts, shape.threads, smem, s>>>(p);
        else if (shape.threads <= 448) rms_norm_backward_kernel<T, Code, 2, true, kSum, !(kPlain && kSum), 448><<<*parts, shape.threads, smem, s>>>(p);
        else rms_norm_backward_kernel<T, Code, 2, true, kSum, !kSum, 1024><<<*parts, shape.threads, smem, s>>>(p);
    } else {
        if (shape.vpt == 1) rms_norm_backward_kernel<T, Code, 1, false, kSum, false, 256><<<*parts, shape.threads, smem, s>>>(p);
        else if (shape.vpt == 2) rms_norm_backward_kernel<T, Code, 2, false, kSum, false, 256><<<*parts, shape.threads, smem, s>>>(p);
        else rms_norm_backward_kernel<T, Code, 4, false, kSum, false, 256><<<*parts, shape.threads, smem, s>>>(p);
    }
    return COBALT_OK;
}

// code: of rows in 8 bits, -1 for rows as they are.
template <typename T, bool kSum>
static int launch_backward(const RmsBackward& p, int code, int sms, int* parts, cudaStream_t s)
{
    return code == COBALT_I8 ? launch_backward<T, CodeI8, kSum>(p, sms, parts, s)
                             : code == COBALT_E4M3 ? launch_backward<T, CodeE4M3, kSum>(p, sms, parts, s) : launch_backward<T, void, kSum>(p, sms, parts, s);
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_rms_norm(const void* x, const void* residual, const float* gamma, int64_t T, int32_t H, int32_t dtype, float eps, void* sum,
                    void* y, void* q, float* q_scales, int32_t q_code, int32_t q_group, float* rstd, cobalt_stream_t stream)
{
    int rc = check_rms(T, H, dtype);
    if (rc != COBALT_OK) return rc;
    if (!(eps >= 0.0f) || (q && !check_code(q_code, q_group)) || (!residual && sum) || (sum && sum == y)) return COBALT_ERR_INVALID_ARG;
    if (T == 0) return COBALT_OK;
    if (!x || !gamma || (!y && !q) || (q && !q_scales)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(residual) || !aligned16(gamma) || !aligned16(sum) || !aligned16(y) || !aligned16(q) ||
        !aligned4(q_scales) || !aligned16(rstd))
        return COBALT_ERR_INVALID_ARG;
    const RmsForward p = {x, residual, gamma, on_32_bytes(gamma), T, H, eps, sum, y, static_cast<uint8_t*>(q), q_scales, q_code, q_group, rstd};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (dtype == COBALT_BF16) q ? launch_forward<__nv_bfloat16, true>(p, s) : launch_forward<__nv_bfloat16, false>(p, s);
    else q ? launch_forward<float, true>(p, s) : launch_forward<float, false>(p, s);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

size_t cobalt_rms_norm_workspace_bytes(int64_t T, int32_t H)
{
    if (check_rms(T, H, COBALT_F32) != COBALT_OK) return 0;
    int64_t parts = 0;
    for (int elems = 4; elems <= 8; elems += 4) {        // whichever type needs more
        const int64_t p = rms_parts(T, rms_shape(H, elems, 2, 2048), kMaxSms);
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
    if (!aligned16(grad_y) || !aligned16(grad_sum) || !aligned16(rows) || !aligned4(row_scales) || !aligned16(gamma) || !aligned4(rstd) ||
        !aligned16(grad_x) || !aligned16(grad_gamma) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cobalt_rms_norm_workspace_bytes(T, H)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != COBALT_OK) return rc;
    const RmsBackward p = {grad_y, grad_sum, rows, row_scales, group == 0 ? 1 : (H + kPackGroup - 1) / kPackGroup, gamma, on_32_bytes(gamma), rstd, T, H, grad_x,
                           static_cast<float*>(workspace)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int parts = 0;
    const int code = packed ? rows_type : -1;
    if (dtype == COBALT_BF16) rc = grad_sum ? launch_backward<__nv_bfloat16, true>(p, code, sms, &parts, s) : launch_backward<__nv_bfloat16, false>(p, code, sms, &parts, s);
    else rc = grad_sum ? launch_backward<float, true>(p, code, sms, &parts, s) : launch_backward<float, false>(p, code, sms, &parts, s);
    if (rc != COBALT_OK) return rc;
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
