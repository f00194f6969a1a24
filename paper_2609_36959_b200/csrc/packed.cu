// Rows to 8 bits and back (see packed.cuh for the format).
//
//   pack    one read of the rows, codes and scales written: 3 bytes a bf16 value. A thread has two pieces of 64 bytes (32 bf16
//           columns; 32-byte loads and stores), four lanes a group of 128, whose largest value takes two shuffles.
//           With one scale a row a warp or a CTA holds the row in registers between its largest value and the codes.
//   unpack  the same walk without the reduction.
//
// Bound by HBM: 32768 x 7168 bf16 with a scale for 128 columns 114 us (6.2 TB/s), with one a row 118 us, read back 109 us (6.5 TB/s).
// Rows whose width is no multiple of such a piece, or pointers off a 32-byte boundary, take eight columns a piece.
#include "packed.cuh"

namespace cobalt {

constexpr int kPackThreads = 256;
constexpr int kPackMaxH = 16384;

// C columns of a row: 16-byte loads, or 32-byte ones where they are more than eight.
template <typename T, int C>
__device__ __forceinline__ void load_columns(const T* p, uint4 (&v)[C / Vec16<T>::kElems])
{
    constexpr int N = Vec16<T>::kElems;
    if constexpr (C > 8) {
#pragma unroll
        for (int i = 0; i < C / N; i += 2)
            asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w), "=r"(v[i + 1].x), "=r"(v[i + 1].y), "=r"(v[i + 1].z),
                           "=r"(v[i + 1].w)
                         : "l"(p + i * N));
    } else {
#pragma unroll
        for (int i = 0; i < C / N; ++i) v[i] = ld_once16(p + i * N);
    }
}

template <typename T, int C>
__device__ __forceinline__ void store_columns(T* p, const float (&f)[C])
{
    constexpr int N = Vec16<T>::kElems;
    uint4 v[C / N];
#pragma unroll
    for (int i = 0; i < C / N; ++i) {
        float e[N];
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = f[i * N + k];
        v[i] = Vec16<T>::pack(e);
    }
    if constexpr (C > 8) {
#pragma unroll
        for (int i = 0; i < C / N; i += 2)
            asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p + i * N), "r"(v[i].x), "r"(v[i].y),
                         "r"(v[i].z), "r"(v[i].w), "r"(v[i + 1].x), "r"(v[i + 1].y), "r"(v[i + 1].z), "r"(v[i + 1].w)
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < C / N; ++i) st_stream16(p + i * N, v[i]);
    }
}

template <int C>
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&w)[C / 4])
{
    if constexpr (C == 32)
        asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                     "r"(w[C / 4 - 4]), "r"(w[C / 4 - 3]), "r"(w[C / 4 - 2]), "r"(w[C / 4 - 1])
                     : "memory");
    else if constexpr (C == 16)
        st_stream16(p, make_uint4(w[0], w[1], w[2], w[3]));
    else
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

// Pieces of C columns, per_row of them a row, kPieces a thread: a CTA has kPackThreads * kPieces consecutive ones, a thread every
// kPackThreads-th.  One 64-bit division a thread; the other pieces follow by steps.
constexpr int kPieces = 2;

struct Piece {
    int64_t row;
    int at;                              // in the row
    __device__ __forceinline__ explicit Piece(int per_row)
    {
        const int64_t index = static_cast<int64_t>(blockIdx.x) * (kPackThreads * kPieces) + threadIdx.x;
        if (index < (1ll << 31)) {
            row = static_cast<uint32_t>(index) / static_cast<uint32_t>(per_row);
            at = static_cast<int>(static_cast<uint32_t>(index) - static_cast<uint32_t>(row) * per_row);
        } else {
            row = index / per_row;
            at = static_cast<int>(index - row * per_row);
        }
    }
    __device__ __forceinline__ void next(int per_row)
    {
        at += kPackThreads;
        if (at >= per_row) {
            if (at < 2 * per_row) {
                at -= per_row;
                ++row;
            } else {
                const int more = at / per_row;
                row += more;
                at -= more * per_row;
            }
        }
    }
};

// CTAs an SM: four spill a few registers and are faster all the same (32768 x 7168 bf16 114 us, three 118, without a bound two and 134), but
// for e4m3 codes of fp32 (16384 x 4096 66 us with three, 75 with four, 79 without).
template <typename T, typename Code>
constexpr int kPackCtas = sizeof(T) == 4 && Code::kLargest == CodeE4M3::kLargest ? 3 : 4;

// One scale for each 128 columns.  per_row counts the last group's missing columns too: its lanes take part in the shuffles.
template <typename T, typename Code, int C>
__global__ void __launch_bounds__(kPackThreads, kPackCtas<T, Code>)
pack_groups_kernel(const T* __restrict__ x, int64_t rows, int H, uint8_t* __restrict__ q, float* __restrict__ scales)
{
    constexpr int kLanes = kPackGroup / C, N = Vec16<T>::kElems;
    const int groups = (H + kPackGroup - 1) / kPackGroup, per_row = groups * kLanes;
    Piece p(per_row);
    uint4 v[kPieces][C / N];
    int64_t row[kPieces];
    int at[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j, p.next(per_row)) {
        row[j] = p.row;
        at[j] = p.at;
#pragma unroll
        for (int i = 0; i < C / N; ++i) v[j][i] = make_uint4(0, 0, 0, 0);
        if (p.row < rows && p.at * C < H) load_columns<T, C>(x + p.row * H + p.at * C, v[j]);
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < C / N; ++i) most = abs_max16<T>(most, v[j][i]);
#pragma unroll
        for (int off = 1; off < kLanes; off <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, off));
        if (row[j] >= rows || at[j] * C >= H) continue;
        const GroupScale g = GroupScale::of<Code>(most);
        float f[C];
#pragma unroll
        for (int i = 0; i < C / N; ++i) {
            float e[N];
            Vec16<T>::unpack(v[j][i], e);
#pragma unroll
            for (int k = 0; k < N; ++k) f[i * N + k] = e[k];
        }
        uint32_t w[C / 4];
        const int64_t to = row[j] * H + at[j] * C;
        encode_exactly<T, Code>(f, g, w);
        store_codes<C>(q + to, w);
        if (at[j] % kLanes == 0) scales[row[j] * groups + at[j] / kLanes] = g.scale;
    }
}

// One scale a row: kCta the CTA has one row, else each warp.  Up to VPT 16-byte vectors a thread.
template <typename T, typename Code, int VPT, bool kCta>
__global__ void __launch_bounds__(1024)
pack_rows_kernel(const T* __restrict__ x, int64_t rows, int H, uint8_t* __restrict__ q, float* __restrict__ scales)
{
    constexpr int N = Vec16<T>::kElems;
    __shared__ uint32_t scratch[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_vec = H / N;
    const int first = kCta ? threadIdx.x : lane, group = kCta ? blockDim.x : 32;
    const int64_t row = kCta ? blockIdx.x : static_cast<int64_t>(blockIdx.x) * (blockDim.x >> 5) + warp;
    if (row >= rows) return;                                       // a whole warp, or no thread of a CTA
    uint4 v[VPT];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = first + i * group;
        v[i] = make_uint4(0, 0, 0, 0);
        if (at < n_vec) v[i] = ld_once16(x + row * H + at * N);
    }
#pragma unroll
    for (int i = 0; i < VPT; ++i) most = abs_max16<T>(most, v[i]);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    if (kCta) {
        if (lane == 0) scratch[warp] = most;
        __syncthreads();
        most = __reduce_max_sync(0xFFFFFFFFu, lane < (blockDim.x >> 5) ? scratch[lane] : 0u);
    }
    const GroupScale g = GroupScale::of<Code>(most);
    if (first == 0) scales[row] = g.scale;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = first + i * group;
        if (at >= n_vec) continue;
        float f[N];
        Vec16<T>::unpack(v[i], f);
        uint32_t w[N / 4];
        const int64_t to = row * H + at * N;
        encode_exactly<T, Code>(f, g, w);
        if constexpr (N == 8) *reinterpret_cast<uint2*>(q + to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(q + to) = w[0];
    }
}

// groups: scales of a row; a group is 128 columns, or the row if there is one.
template <typename T, typename Code, int C>
__global__ void __launch_bounds__(kPackThreads)
unpack_rows_kernel(const uint8_t* __restrict__ q, const float* __restrict__ scales, int64_t rows, int H, int groups, T* __restrict__ out)
{
    const int per_row = H / C;
    Piece p(per_row);
    uint32_t w[kPieces][C / 4];
    float scale[kPieces];
    int64_t to[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j, p.next(per_row)) {
        to[j] = -1;
        if (p.row >= rows) continue;
        to[j] = p.row * H + p.at * C;
        if constexpr (C == 16) {
            const uint4 v = ld_stream16(q + to[j]);
            w[j][0] = v.x, w[j][1] = v.y, w[j][2] = v.z, w[j][3] = v.w;
        } else {
            const uint2 v = __ldcs(reinterpret_cast<const uint2*>(q + to[j]));
            w[j][0] = v.x, w[j][1] = v.y;
        }
        scale[j] = __ldg(scales + p.row * groups + (groups > 1 ? p.at * C / kPackGroup : 0));
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
        if (to[j] < 0) continue;
        float f[C];
#pragma unroll
        for (int i = 0; i < C / 4; ++i) {
            float e[4];
            Code::decode4(w[j][i], e);
#pragma unroll
            for (int k = 0; k < 4; ++k) f[4 * i + k] = e[k] * scale[j];
        }
        store_columns<T, C>(out + to[j], f);
    }
}

static bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31u) == 0; }

static int64_t piece_ctas(int64_t rows, int64_t per_row) { return (rows * per_row + kPackThreads * kPieces - 1) / (kPackThreads * kPieces); }

template <typename T, typename Code>
static int launch_pack(const T* x, int64_t rows, int H, bool whole_row, uint8_t* q, float* scales, cudaStream_t s)
{
    if (!whole_row) {
        const int64_t groups = (H + kPackGroup - 1) / kPackGroup;
        constexpr int kWide = 64 / sizeof(T);
        if (H % kWide == 0 && aligned32(x) && aligned32(q)) {
            const int64_t ctas = piece_ctas(rows, groups * (kPackGroup / kWide));
            if (ctas >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
            pack_groups_kernel<T, Code, kWide><<<static_cast<unsigned>(ctas), kPackThreads, 0, s>>>(x, rows, H, q, scales);
        } else {
            const int64_t ctas = piece_ctas(rows, groups * (kPackGroup / 8));
            if (ctas >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
            pack_groups_kernel<T, Code, 8><<<static_cast<unsigned>(ctas), kPackThreads, 0, s>>>(x, rows, H, q, scales);
        }
        return COBALT_OK;
    }
    const int n_vec = H / Vec16<T>::kElems;
    const unsigned by_warp = static_cast<unsigned>((rows + 7) / 8), by_cta = static_cast<unsigned>(rows);
    const unsigned threads = static_cast<unsigned>(((n_vec + 3) / 4 + 31) / 32 * 32);
    if (n_vec <= 32) pack_rows_kernel<T, Code, 1, false><<<by_warp, 256, 0, s>>>(x, rows, H, q, scales);
    else if (n_vec <= 128) pack_rows_kernel<T, Code, 4, false><<<by_warp, 256, 0, s>>>(x, rows, H, q, scales);
    else pack_rows_kernel<T, Code, 4, true><<<by_cta, threads, 0, s>>>(x, rows, H, q, scales);
    return COBALT_OK;
}

template <typename T, typename Code>
static int launch_unpack(const uint8_t* q, const float* scales, int64_t rows, int H, bool whole_row, T* out, cudaStream_t s)
{
    const int groups = whole_row ? 1 : (H + kPackGroup - 1) / kPackGroup;
    const bool wide = H % 16 == 0 && aligned32(out);
    const int64_t ctas = piece_ctas(rows, H / (wide ? 16 : 8));
    if (ctas >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    const unsigned grid = static_cast<unsigned>(ctas);
    if (wide) unpack_rows_kernel<T, Code, 16><<<grid, kPackThreads, 0, s>>>(q, scales, rows, H, groups, out);
    else unpack_rows_kernel<T, Code, 8><<<grid, kPackThreads, 0, s>>>(q, scales, rows, H, groups, out);
    return COBALT_OK;
}

static int check_pack(int64_t T, int32_t H, int32_t dtype, int32_t code, int32_t group)
{
    if (T < 0 || H < 1 || (dtype != COBALT_BF16 && dtype != COBALT_F32) || (code != COBALT_E4M3 && code != COBALT_I8) ||
        (group != 0 && group != kPackGroup))
        return COBALT_ERR_INVALID_ARG;
    if (H % 8 != 0 || H > kPackMaxH || T >= (1ll << 31)) return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

}  // namespace cobalt

using namespace cobalt;

extern "C" {

int cobalt_pack_rows(const void* x, int64_t T, int32_t H, int32_t dtype, int32_t code, int32_t group, void* q, float* scales,
                     cobalt_stream_t stream)
{
    int rc = check_pack(T, H, dtype, code, group);
    if (rc != COBALT_OK) return rc;
    if (T == 0) return COBALT_OK;
    if (!x || !q || !scales || !aligned16(x) || !aligned16(q) || !aligned16(scales)) return COBALT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t* codes = static_cast<uint8_t*>(q);
    const bool row = group == 0;
    if (dtype == COBALT_BF16) {
        const __nv_bfloat16* in = static_cast<const __nv_bfloat16*>(x);
        rc = code == COBALT_I8 ? launch_pack<__nv_bfloat16, CodeI8>(in, T, H, row, codes, scales, s)
                               : launch_pack<__nv_bfloat16, CodeE4M3>(in, T, H, row, codes, scales, s);
    } else {
        const float* in = static_cast<const float*>(x);
        rc = code == COBALT_I8 ? launch_pack<float, CodeI8>(in, T, H, row, codes, scales, s)
                               : launch_pack<float, CodeE4M3>(in, T, H, row, codes, scales, s);
    }
    if (rc != COBALT_OK) return rc;
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

int cobalt_unpack_rows(const void* q, const float* scales, int64_t T, int32_t H, int32_t code, int32_t group, int32_t dtype, void* out,
                       cobalt_stream_t stream)
{
    int rc = check_pack(T, H, dtype, code, group);
    if (rc != COBALT_OK) return rc;
    if (T == 0) return COBALT_OK;
    if (!q || !scales || !out || !aligned16(q) || !aligned16(scales) || !aligned16(out)) return COBALT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const uint8_t* codes = static_cast<const uint8_t*>(q);
    const bool row = group == 0;
    if (dtype == COBALT_BF16) {
        __nv_bfloat16* to = static_cast<__nv_bfloat16*>(out);
        rc = code == COBALT_I8 ? launch_unpack<__nv_bfloat16, CodeI8>(codes, scales, T, H, row, to, s)
                               : launch_unpack<__nv_bfloat16, CodeE4M3>(codes, scales, T, H, row, to, s);
    } else {
        float* to = static_cast<float*>(out);
        rc = code == COBALT_I8 ? launch_unpack<float, CodeI8>(codes, scales, T, H, row, to, s)
                               : launch_unpack<float, CodeE4M3>(codes, scales, T, H, row, to, s);
    }
    if (rc != COBALT_OK) return rc;
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // extern "C"
