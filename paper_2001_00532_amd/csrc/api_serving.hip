// C-ABI layer of the products with 4-bit weights and of the mixture of experts: argument checks.  No kernels here.
#include "../../include/psk.h"
#include "psk_internal.h"
#include "psk_mfma.h"

using namespace psk;

static_assert(PSK_F32 == F32 && PSK_F16 == F16 && PSK_BF16 == BF16, "types");

namespace {

// Rows and columns: a launch has fewer than 2^32 threads, 256 of them for 16 rows padded to 256; and places in the copy of a tile of vectors are
// counted in 32 bits.
constexpr int64_t kMaxEdge = (int64_t(1) << 28) - 256;

inline int hip_status(hipError_t e) { return e == hipSuccess ? PSK_OK : PSK_ERR_HIP; }
inline bool type_ok(int t) { return t == PSK_F32 || t == PSK_F16 || t == PSK_BF16; }
inline bool misaligned(const void *p, int to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0; }
inline int bytes_of(int t) { return t == PSK_F32 ? 4 : 2; }
inline bool workspace_ok(const void *p, size_t have, size_t need) { return p && !misaligned(p, 256) && have >= need; }

int check_q4(const psk_q4 *A, int type)
{
    if (!A) return PSK_ERR_NULL;
    if (A->count < 0 || A->rows < 0 || A->cols < 0 || A->rows > kMaxEdge || A->cols > kMaxEdge) return PSK_ERR_SIZE;
    if (A->group < 32 || (A->group & (A->group - 1))) return PSK_ERR_SIZE;
    if (A->scale_type != PSK_F32 && A->scale_type != type) return PSK_ERR_UNSUPPORTED;
    if (A->count == 0 || A->rows == 0 || A->cols == 0) return PSK_OK;
    if (!A->codes || !A->scales) return PSK_ERR_NULL;
    if (A->ld_codes < (A->cols + 31) / 32 * 16 || A->ld_scales < (A->cols + A->group - 1) / A->group) return PSK_ERR_SIZE;
    if (A->count > 1 && (A->stride_codes < 0 || A->stride_scales < 0)) return PSK_ERR_SIZE;
    if (misaligned(A->codes, 16) || A->ld_codes % 16 || (A->count > 1 && A->stride_codes % 16) || misaligned(A->scales, bytes_of(A->scale_type)))
        return PSK_ERR_ALIGNMENT;
    return PSK_OK;
}

WeightsQ4 weights(const psk_q4 &A)
{
    return WeightsQ4{A.codes, A.zeros, A.scales, A.ld_codes, A.ld_scales, A.stride_codes, A.stride_scales, (int)A.rows, (int)A.cols, __builtin_ctz((unsigned)A.group)};
}

// What both forms of the layer have in common.
int check_layer(int64_t n, int64_t dim, int64_t inter, int64_t experts, int32_t top_k, int act, int type, int64_t ldx, int64_t ldy)
{
    if (n < 0 || n > PSK_MAX_VECTORS || dim < 1 || inter < 1 || dim > kMaxEdge || inter > kMaxEdge) return PSK_ERR_SIZE;
    if (experts < 1 || experts > PSK_MOE_MAX_EXPERTS || top_k < 1 || top_k > PSK_MOE_MAX_TOP_K) return PSK_ERR_SIZE;
    if (ldx < dim || ldy < dim) return PSK_ERR_SIZE;
    if (act != PSK_ACT_SILU && act != PSK_ACT_GELU) return PSK_ERR_UNSUPPORTED;
    if (type != PSK_F16 && type != PSK_BF16) return PSK_ERR_UNSUPPORTED;
    return PSK_OK;
}

}  // namespace

extern "C" {

size_t psk_gemm_q4_workspace_bytes(int64_t rows, int64_t cols, int64_t n, int type)
{
    if (rows < 0 || cols < 0 || rows > kMaxEdge || cols > kMaxEdge || n < 0 || n > PSK_MAX_VECTORS || !type_ok(type)) return 0;
    // more than four vectors: their copy in the order of the operands, vectors of 32 bits in three parts
    return n <= 4 ? 256 : (size_t)((n + 15) / 16) * copied_blocks((int)cols) * (type == PSK_F32 ? 3 : 1) * 1024 + 256;
}

int psk_gemm_q4(const psk_q4 *A, int64_t n, int type, const void *X, int64_t ldx, void *Y, int64_t ldy, void *workspace,
                size_t workspace_bytes, void *stream)
{
    if (!type_ok(type)) return PSK_ERR_UNSUPPORTED;
    const int st = check_q4(A, type);
    if (st != PSK_OK) return st;
    if (A->count != 1 || n < 0 || n > PSK_MAX_VECTORS || ldx < A->cols || ldy < A->rows) return PSK_ERR_SIZE;
    if (!workspace_ok(workspace, workspace_bytes, psk_gemm_q4_workspace_bytes(A->rows, A->cols, n, type))) return PSK_ERR_WORKSPACE;
    if (n == 0 || A->rows == 0) return PSK_OK;
    if (!Y || (A->cols > 0 && !X)) return PSK_ERR_NULL;
    if (misaligned(X, bytes_of(type)) || misaligned(Y, bytes_of(type))) return PSK_ERR_ALIGNMENT;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (A->cols == 0)                                      // the kernels load the scale of the last column; here there is none, nor need there be any codes
        return hip_status(type == PSK_F32 ? launch_fill_zero_2d(static_cast<float *>(Y), n, (int32_t)A->rows, ldy, s)
                                          : launch_fill_zero_2d(static_cast<uint16_t *>(Y), n, (int32_t)A->rows, ldy, s));
    const auto launch = type == PSK_F32 ? launch_gemm_q4_of<F32> : (type == PSK_F16 ? launch_gemm_q4_of<F16> : launch_gemm_q4_of<BF16>);
    return hip_status(launch(weights(*A), A->scale_type, (int)n, X, ldx, Y, ldy, workspace, s));
}

size_t psk_moe_route_workspace_bytes(int64_t n, int64_t experts)
{
    if (n < 0 || n > PSK_MAX_VECTORS || experts < 1 || experts > PSK_MOE_MAX_EXPERTS) return 0;
    return align256((size_t)n * (size_t)experts * sizeof(double) + 1);
}

int psk_moe_route(int64_t n, int64_t dim, int64_t experts, int32_t top_k, int score, int normalise, float factor, int type,
                  const void *X, int64_t ldx, int wtype, const void *W, int64_t ldw, const float *bias, int32_t *crd, float *vals,
                  void *workspace, size_t workspace_bytes, void *stream)
{
    if (n < 0 || n > PSK_MAX_VECTORS || dim < 1 || dim > kMaxEdge || experts < 1 || experts > PSK_MOE_MAX_EXPERTS) return PSK_ERR_SIZE;
    if (top_k < 1 || top_k > PSK_MOE_MAX_TOP_K || ldx < dim || ldw < dim) return PSK_ERR_SIZE;
    if (!type_ok(type) || (wtype != PSK_F32 && wtype != type)) return PSK_ERR_UNSUPPORTED;
    if (score != PSK_SCORE_SOFTMAX && score != PSK_SCORE_SIGMOID) return PSK_ERR_UNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, psk_moe_route_workspace_bytes(n, experts))) return PSK_ERR_WORKSPACE;
    if (n == 0) return PSK_OK;
    if (!X || !W || !crd || !vals) return PSK_ERR_NULL;
    if (misaligned(X, bytes_of(type)) || misaligned(W, bytes_of(wtype)) || misaligned(bias, 4) || misaligned(crd, 4) || misaligned(vals, 4))
        return PSK_ERR_ALIGNMENT;
    return hip_status(launch_moe_route((int)n, (int)dim, (int)experts, top_k, score, normalise, factor, type, X, ldx, wtype, W, ldw, bias, crd, vals,
                                       static_cast<double *>(workspace), static_cast<hipStream_t>(stream)));
}

size_t psk_moe_workspace_bytes(int64_t n, int64_t dim, int64_t inter, int64_t experts, int32_t top_k)
{
    if (check_layer(n, dim, inter, experts, top_k, PSK_ACT_SILU, PSK_F16, dim, dim) != PSK_OK) return 0;
    return moe_workspace_bytes(n, dim, inter, experts, top_k);
}

int psk_moe_experts(int64_t n, int64_t dim, int64_t inter, int64_t experts, int32_t top_k, int act, int type, const void *X,
                    int64_t ldx, const int32_t *crd, const float *vals, const void *W1, const void *W3, int64_t ld1,
                    int64_t stride1, const void *W2, int64_t ld2, int64_t stride2, void *Y, int64_t ldy, void *workspace,
                    size_t workspace_bytes, void *stream)
{
    const int st = check_layer(n, dim, inter, experts, top_k, act, type, ldx, ldy);
    if (st != PSK_OK) return st;
    if (ld1 < dim || ld2 < inter || stride1 < 0 || stride2 < 0) return PSK_ERR_SIZE;
    if (!workspace_ok(workspace, workspace_bytes, moe_workspace_bytes(n, dim, inter, experts, top_k))) return PSK_ERR_WORKSPACE;
    if (n == 0) return PSK_OK;
    if (!X || !crd || !vals || !W1 || !W3 || !W2 || !Y) return PSK_ERR_NULL;
    if (misaligned(X, 2) || misaligned(Y, 2) || misaligned(crd, 4) || misaligned(vals, 4) || misaligned(W1, 2) || misaligned(W3, 2) || misaligned(W2, 2))
        return PSK_ERR_ALIGNMENT;
    const MoeCall c = {n, (int)dim, (int)inter, (int)experts, top_k, act, X, ldx, crd, vals, Y, ldy, workspace};
    return hip_status(launch_moe_16(c, type, W1, W3, ld1, stride1, W2, ld2, stride2, static_cast<hipStream_t>(stream)));
}

int psk_moe_experts_q4(int64_t n, int32_t top_k, int act, int type, const void *X, int64_t ldx, const int32_t *crd,
                       const float *vals, const psk_q4 *W1, const psk_q4 *W3, const psk_q4 *W2, void *Y, int64_t ldy,
                       void *workspace, size_t workspace_bytes, void *stream)
{
    const psk_q4 *all[3] = {W1, W3, W2};
    for (const psk_q4 *w : all) {
        const int st = check_q4(w, type);
        if (st != PSK_OK) return st;
    }
    const int64_t dim = W1->cols, inter = W1->rows, experts = W1->count;
    const int st = check_layer(n, dim, inter, experts, top_k, act, type, ldx, ldy);
    if (st != PSK_OK) return st;
    if (W3->rows != inter || W3->cols != dim || W2->rows != dim || W2->cols != inter || W3->count != experts || W2->count != experts || W3->group != W1->group)
        return PSK_ERR_SIZE;
    if (W3->scale_type != W1->scale_type || W2->scale_type != W1->scale_type) return PSK_ERR_UNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, moe_workspace_bytes(n, dim, inter, experts, top_k))) return PSK_ERR_WORKSPACE;
    if (n == 0) return PSK_OK;
    if (!X || !crd || !vals || !Y) return PSK_ERR_NULL;
    if (misaligned(X, 2) || misaligned(Y, 2) || misaligned(crd, 4) || misaligned(vals, 4)) return PSK_ERR_ALIGNMENT;
    const MoeCall c = {n, (int)dim, (int)inter, (int)experts, top_k, act, X, ldx, crd, vals, Y, ldy, workspace};
    const auto launch = type == PSK_F16 ? launch_moe_q4_of<F16> : launch_moe_q4_of<BF16>;
    return hip_status(launch(c, W1->scale_type, weights(*W1), weights(*W3), weights(*W2), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
