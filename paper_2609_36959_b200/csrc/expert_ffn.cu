// The experts between dispatch and combine: a gated feed-forward block over the rows of every slot, and its backward
// pass.  With x a row of slot d, e = slot_expert[d], Wg and Wu the two halves of w_gate_up[e], Wd = w_down[e]:
//
//   g = Wg x    u = Wu x    a = g s u, s = 1 / (1 + exp(-g))    y = Wd a
//   da = Wd^T dy    du = da g s    dg = da u s (1 + g (1 - s))    dx = Wg^T dg + Wu^T du
//   dWg = sum dg x^T    dWu = sum du x^T    dWd = sum dy a^T     over the rows of all slots that hold e
//
// First form: plain shared-memory tiles on the fp32 units, right for every size.
#include "numeric.cuh"

namespace cobalt {

typedef __nv_bfloat16 bf16;

constexpr int kTile = 64, kTileK = 16;

// Rows of slot d, clamped so that no bad offset leads out of the buffers.
__device__ __forceinline__ void slot_rows(const uint32_t* offsets, int d, int64_t P, int64_t* first, int64_t* last)
{
    const int64_t a = offsets[d], b = offsets[d + 1];
    *first = a < P ? a : P;
    *last = b < P ? b : P;
    if (*last < *first) *last = *first;
}

// acc[i][j] += sum_k A[m0 + 4 ty + i][k] * B[n0 + 4 tx + j][k] for k in [k0, k1); element strides given.
__device__ __forceinline__ void tile_product(const bf16* A, int64_t am, int64_t ak, int64_t m0, int64_t m1, const bf16* B,
                                             int64_t bn, int64_t bk, int64_t n0, int64_t n1, int64_t k0, int64_t k1,
                                             float (*sa)[kTile + 1], float (*sb)[kTile + 1], float (&acc)[4][4])
{
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (int64_t k = k0; k < k1; k += kTileK) {
        for (int i = threadIdx.x; i < kTile * kTileK; i += 256) {
            const int kk = ak == 1 ? i % kTileK : i / kTile, m = ak == 1 ? i / kTileK : i % kTile;
            sa[kk][m] = (m0 + m < m1 && k + kk < k1) ? __bfloat162float(A[(m0 + m) * am + (k + kk) * ak]) : 0.0f;
        }
        for (int i = threadIdx.x; i < kTile * kTileK; i += 256) {
            const int kk = bk == 1 ? i % kTileK : i / kTile, n = bk == 1 ? i / kTileK : i % kTile;
            sb[kk][n] = (n0 + n < n1 && k + kk < k1) ? __bfloat162float(B[(n0 + n) * bn + (k + kk) * bk]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kTileK; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(sa[kk][4 * ty + i], sb[kk][4 * tx + j], acc[i][j]);
        __syncthreads();
    }
}

enum { kUp, kDown, kDownBackward, kUpBackward };

struct FfnArgs {
    const bf16 *rows, *w_gate_up, *w_down, *grad_out, *pre_in, *act_in;
    bf16 *act, *pre, *out, *grad_pre, *grad_rows;
    const uint32_t* offsets;
    const int32_t* slot_expert;
    int64_t P;
    int D, E, H, F;
    uint32_t* err_word;
};

template <int kStage>
__global__ void __launch_bounds__(256) ffn_rows_kernel(FfnArgs p)
{
    __shared__ float sa[kTileK][kTile + 1], sb[kTileK][kTile + 1];
    const int d = blockIdx.y, e = p.slot_expert[d];
    int64_t first, last;
    slot_rows(p.offsets, d, p.P, &first, &last);
    if (blockIdx.x == 0 && threadIdx.x == 0 && (p.offsets[d + 1] < p.offsets[d] || p.offsets[d + 1] > p.P))
        flag_error(p.err_word, COBALT_DEVERR_BAD_SLOT);
    if (first == last) return;
    if (e < 0 || e >= p.E) {
        if (threadIdx.x == 0) flag_error(p.err_word, COBALT_DEVERR_BAD_SLOT);
        return;
    }
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t H = p.H, F = p.F, n0 = static_cast<int64_t>(blockIdx.x) * kTile;
    const bf16* wgu = p.w_gate_up + static_cast<int64_t>(e) * 2 * F * H;
    const bf16* wd = p.w_down + static_cast<int64_t>(e) * H * F;
    for (int64_t m0 = first; m0 < last; m0 += kTile) {
        float acc[4][4] = {}, acc2[4][4] = {};
        if (kStage == kUp) {
            tile_product(p.rows, H, 1, m0, last, wgu, H, 1, n0, F, 0, H, sa, sb, acc);
            tile_product(p.rows, H, 1, m0, last, wgu + F * H, H, 1, n0, F, 0, H, sa, sb, acc2);
        } else if (kStage == kDown) {
            tile_product(p.act_in, F, 1, m0, last, wd, F, 1, n0, H, 0, F, sa, sb, acc);
        } else if (kStage == kDownBackward) {
            tile_product(p.grad_out, H, 1, m0, last, wd, 1, F, n0, F, 0, H, sa, sb, acc);
        } else {
            tile_product(p.grad_pre, 2 * F, 1, m0, last, wgu, 1, H, n0, H, 0, 2 * F, sa, sb, acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t r = m0 + 4 * ty + i, c = n0 + 4 * tx + j;
                if (r >= last) continue;
                if (kStage == kUp && c < F) {
                    const float g = acc[i][j], u = acc2[i][j];
                    p.act[r * F + c] = __float2bfloat16_rn(g / (1.0f + expf(-g)) * u);
                    if (p.pre) {
                        p.pre[r * 2 * F + c] = __float2bfloat16_rn(g);
                        p.pre[r * 2 * F + F + c] = __float2bfloat16_rn(u);
                    }
                } else if (kStage == kDown && c < H) {
                    p.out[r * H + c] = __float2bfloat16_rn(acc[i][j]);
                } else if (kStage == kDownBackward && c < F) {
                    const float g = __bfloat162float(p.pre_in[r * 2 * F + c]), u = __bfloat162float(p.pre_in[r * 2 * F + F + c]);
                    const float s = 1.0f / (1.0f + expf(-g)), da = acc[i][j];
                    p.grad_pre[r * 2 * F + c] = __float2bfloat16_rn(da * u * s * (1.0f + g * (1.0f - s)));
                    p.grad_pre[r * 2 * F + F + c] = __float2bfloat16_rn(da * g * s);
                } else if (kStage == kUpBackward && c < H) {
                    p.grad_rows[r * H + c] = __float2bfloat16_rn(acc[i][j]);
                }
            }
    }
}

// grad_w[e][m][n] = sum over the rows of e's slots of a[row][m] * b[row][n]
__global__ void __launch_bounds__(256)
ffn_weights_kernel(const bf16* a, int64_t M, const bf16* b, int64_t N, const uint32_t* offsets, const int32_t* slot_expert,
                   int64_t P, int D, bf16* grad_w)
{
    __shared__ float sa[kTileK][kTile + 1], sb[kTileK][kTile + 1];
    const int e = blockIdx.z;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * kTile, n0 = static_cast<int64_t>(blockIdx.x) * kTile;
    float acc[4][4] = {};
    for (int d = 0; d < D; ++d) {
        if (slot_expert[d] != e) continue;
        int64_t first, last;
        slot_rows(offsets, d, P, &first, &last);
        tile_product(a, 1, M, m0, M, b, 1, N, n0, N, first, last, sa, sb, acc);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (m0 + 4 * ty + i < M && n0 + 4 * tx + j < N)
                grad_w[(static_cast<int64_t>(e) * M + m0 + 4 * ty + i) * N + n0 + 4 * tx + j] = __float2bfloat16_rn(acc[i][j]);
}

static int check_ffn(int64_t P, int32_t D, int32_t E, int32_t H, int32_t F)
{
    if (P < 0 || D < 1 || E < 1 || H < 1 || F < 1) return COBALT_ERR_INVALID_ARG;
    if (P >= (1ll << 31) || D > COBALT_MAX_DESTS || E > COBALT_MAX_EXPERTS || H % 8 != 0 || F % 8 != 0 || H > COBALT_FFN_MAX_WIDTH ||
        F > COBALT_FFN_MAX_WIDTH)
        return COBALT_ERR_UNSUPPORTED;
    return COBALT_OK;
}

static unsigned tiles(int64_t n) { return static_cast<unsigned>((n + kTile - 1) / kTile); }

}  // namespace cobalt

using namespace cobalt;

extern "C" {

size_t cobalt_expert_ffn_workspace_bytes(int64_t P, int32_t D, int32_t E, int32_t H, int32_t F)
{
    if (check_ffn(P, D, E, H, F) != COBALT_OK) return 0;
    return 256;
}

int cobalt_expert_ffn(const void* rows, const uint32_t* dest_offsets, const int32_t* slot_expert, int64_t P, int32_t D,
                      int32_t E, int32_t H, int32_t F, const void* w_gate_up, const void* w_down, void* act, void* pre,
                      void* out, void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    int rc = check_ffn(P, D, E, H, F);
    if (rc != COBALT_OK) return rc;
    if (P == 0) return COBALT_OK;
    if (!rows || !dest_offsets || !slot_expert || !w_gate_up || !w_down || !act || !out) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(rows) || !aligned16(dest_offsets) || !aligned16(slot_expert) || !aligned16(w_gate_up) || !aligned16(w_down) ||
        !aligned16(act) || !aligned16(pre) || !aligned16(out) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cobalt_expert_ffn_workspace_bytes(P, D, E, H, F)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    FfnArgs p = {};
    rc = device_error_word(&p.err_word);
    if (rc != COBALT_OK) return rc;
    p.rows = static_cast<const bf16*>(rows); p.w_gate_up = static_cast<const bf16*>(w_gate_up);
    p.w_down = static_cast<const bf16*>(w_down); p.act = static_cast<bf16*>(act); p.act_in = p.act;
    p.pre = static_cast<bf16*>(pre); p.out = static_cast<bf16*>(out);
    p.offsets = dest_offsets; p.slot_expert = slot_expert; p.P = P; p.D = D; p.E = E; p.H = H; p.F = F;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    ffn_rows_kernel<kUp><<<dim3(tiles(F), D), 256, 0, s>>>(p);
    ffn_rows_kernel<kDown><<<dim3(tiles(H), D), 256, 0, s>>>(p);
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

int cobalt_expert_ffn_backward(const void* grad_out, const void* rows, const uint32_t* dest_offsets, const int32_t* slot_expert,
                               int64_t P, int32_t D, int32_t E, int32_t H, int32_t F, const void* w_gate_up, const void* w_down,
                               const void* pre, const void* act, void* grad_pre, void* grad_rows, void* grad_w_gate_up,
                               void* grad_w_down, void* workspace, size_t workspace_bytes, cobalt_stream_t stream)
{
    int rc = check_ffn(P, D, E, H, F);
    if (rc != COBALT_OK) return rc;
    if (!dest_offsets || !slot_expert) return COBALT_ERR_INVALID_ARG;
    if (!grad_rows && !grad_w_gate_up && !grad_w_down) return COBALT_ERR_INVALID_ARG;
    if (P > 0 && (!grad_out || !rows || !w_gate_up || !w_down || !pre || !act || !grad_pre)) return COBALT_ERR_INVALID_ARG;
    if (!aligned16(grad_out) || !aligned16(rows) || !aligned16(dest_offsets) || !aligned16(slot_expert) || !aligned16(w_gate_up) ||
        !aligned16(w_down) || !aligned16(pre) || !aligned16(act) || !aligned16(grad_pre) || !aligned16(grad_rows) ||
        !aligned16(grad_w_gate_up) || !aligned16(grad_w_down) || !aligned16(workspace))
        return COBALT_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < cobalt_expert_ffn_workspace_bytes(P, D, E, H, F)) return COBALT_ERR_WORKSPACE_TOO_SMALL;
    FfnArgs p = {};
    rc = device_error_word(&p.err_word);
    if (rc != COBALT_OK) return rc;
    p.rows = static_cast<const bf16*>(rows); p.w_gate_up = static_cast<const bf16*>(w_gate_up);
    p.w_down = static_cast<const bf16*>(w_down); p.grad_out = static_cast<const bf16*>(grad_out);
    p.pre_in = static_cast<const bf16*>(pre); p.act_in = static_cast<const bf16*>(act);
    p.grad_pre = static_cast<bf16*>(grad_pre); p.grad_rows = static_cast<bf16*>(grad_rows);
    p.offsets = dest_offsets; p.slot_expert = slot_expert; p.P = P; p.D = D; p.E = E; p.H = H; p.F = F;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (P > 0 && (grad_rows || grad_w_gate_up)) {
        ffn_rows_kernel<kDownBackward><<<dim3(tiles(F), D), 256, 0, s>>>(p);
        if (grad_rows) ffn_rows_kernel<kUpBackward><<<dim3(tiles(H), D), 256, 0, s>>>(p);
    }
    if (grad_w_gate_up)
        ffn_weights_kernel<<<dim3(tiles(H), tiles(2 * static_cast<int64_t>(F)), E), 256, 0, s>>>(
            p.grad_pre, 2 * static_cast<int64_t>(F), p.rows, H, dest_offsets, slot_expert, P, D, static_cast<bf16*>(grad_w_gate_up));
    if (grad_w_down)
        ffn_weights_kernel<<<dim3(tiles(F), tiles(H), E), 256, 0, s>>>(p.grad_out, H, p.act_in, F, dest_offsets, slot_expert, P, D,
                                                                       static_cast<bf16*>(grad_w_down));
    COBALT_CUDA_TRY(cudaGetLastError());
    return COBALT_OK;
}

}  // extern "C"
