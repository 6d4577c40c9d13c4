// C-ABI layer of the products of 8-bit integers and of the embedding: argument checks.  No kernels here.
#include "../../include/psk.h"
#include "psk_internal.h"

using namespace psk;

namespace {

constexpr int64_t kMaxEdge = (int64_t(1) << 28) - 256;     // as for the products with 4-bit weights
constexpr int kTableI8 = 3;

inline int hip_status(hipError_t e) { return e == hipSuccess ? PSK_OK : PSK_ERR_HIP; }
inline bool type_ok(int t) { return t == PSK_F32 || t == PSK_F16 || t == PSK_BF16; }
inline bool misaligned(const void *p, int to) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(to - 1)) != 0; }
inline int bytes_of(int t) { return t == PSK_F32 ? 4 : 2; }
inline bool workspace_ok(const void *p, size_t have, size_t need) { return p && !misaligned(p, 256) && have >= need; }
inline int64_t pieces(int64_t cols) { return (cols + 15) / 16 * 16; }
// rows in memory: elements from the first to the last fit 2^62
inline bool ld_ok(int64_t ld, int64_t width) { return ld >= width && ld < (int64_t(1) << 31); }

int check_codes(const void *codes, int64_t ld, int64_t cols)
{
    if (!codes) return PSK_ERR_NULL;
    if (ld < pieces(cols) || ld > PSK_I8_MAX_LD) return PSK_ERR_SIZE;
    return misaligned(codes, 16) || ld % 16 ? PSK_ERR_ALIGNMENT : PSK_OK;
}

// `most`: columns
int check_i8(const psk_i8 *A, int64_t most)
{
    if (!A) return PSK_ERR_NULL;
    if (A->rows < 0 || A->cols < 0 || A->rows > kMaxEdge || A->cols > most) return PSK_ERR_SIZE;
    if (A->rows == 0) return PSK_OK;
    if (!A->scales) return PSK_ERR_NULL;
    if (misaligned(A->scales, 4)) return PSK_ERR_ALIGNMENT;
    return A->cols == 0 ? PSK_OK : check_codes(A->codes, A->ld, A->cols);
}

// Codes of tokens in a workspace: whole lines, zeros behind the columns; their scales; what psk_gemm_i8 has there.
int64_t line(int64_t cols) { return (cols + 127) / 128 * 128; }
size_t codes_bytes(int64_t cols, int64_t n) { return align256((size_t)n * (size_t)line(cols) + 1); }
size_t scales_bytes(int64_t n) { return align256((size_t)n * 4 + 1); }

}  // namespace

extern "C" {

int psk_quant_i8(int64_t n, int64_t cols, int type, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales, void *stream)
{
    if (!type_ok(type)) return PSK_ERR_UNSUPPORTED;
    if (n < 0 || n > kMaxEdge || cols < 0 || cols > PSK_I8_MAX_COLS || !ld_ok(ldx, cols)) return PSK_ERR_SIZE;
    if (n == 0) return PSK_OK;
    if (!scales || (cols > 0 && !X)) return PSK_ERR_NULL;
    if (misaligned(scales, 4) || misaligned(X, bytes_of(type))) return PSK_ERR_ALIGNMENT;
    if (cols > 0) {
        const int st = check_codes(codes, ldc, cols);
        if (st != PSK_OK) return st;
    }
    return hip_status(launch_quant_i8((int)n, (int)cols, (int)pieces(cols), type, X, ldx, codes, ldc, scales, static_cast<hipStream_t>(stream)));
}

size_t psk_gemm_i8_workspace_bytes(int64_t rows, int64_t cols, int64_t n)
{
    if (rows < 0 || rows > kMaxEdge || cols < 0 || cols > PSK_I8_MAX_COLS || n < 0 || n > PSK_MAX_VECTORS) return 0;
    return align256(gemm_i8_workspace_bytes((int)rows, (int)cols, (int)n) + 1);
}

int psk_gemm_i8(const psk_i8 *A, int64_t n, const int8_t *X, int64_t ldx, const float *scales, const float *bias, int type, void *Y, int64_t ldy,
                void *workspace, size_t workspace_bytes, void *stream)
{
    if (!type_ok(type)) return PSK_ERR_UNSUPPORTED;
    int st = check_i8(A, PSK_I8_MAX_COLS);
    if (st != PSK_OK) return st;
    if (n < 0 || n > PSK_MAX_VECTORS || !ld_ok(ldy, A->rows)) return PSK_ERR_SIZE;
    if (!workspace_ok(workspace, workspace_bytes, psk_gemm_i8_workspace_bytes(A->rows, A->cols, n))) return PSK_ERR_WORKSPACE;
    if (n == 0 || A->rows == 0) return PSK_OK;
    if (!Y || !scales) return PSK_ERR_NULL;
    if (A->cols > 0) {
        st = check_codes(X, ldx, A->cols);
        if (st != PSK_OK) return st;
    }
    if (misaligned(Y, bytes_of(type)) || misaligned(scales, 4) || misaligned(bias, 4)) return PSK_ERR_ALIGNMENT;
    if (gemv_i8_takes((int)A->cols, (int)n))
        return hip_status(launch_gemv_i8((int)A->rows, (int)A->cols, (int)n, A->codes, A->ld, A->scales, X, ldx, scales, bias, type, Y, ldy,
                                         static_cast<hipStream_t>(stream)));
    return hip_status(launch_gemm_i8((int)A->rows, (int)A->cols, (int)n, A->codes, A->ld, A->scales, X, ldx, scales, bias, type, Y, ldy, workspace,
                                     static_cast<hipStream_t>(stream)));
}

size_t psk_linear_i8_workspace_bytes(int64_t rows, int64_t cols, int64_t n, int type)
{
    const size_t sums = psk_gemm_i8_workspace_bytes(rows, cols, n);
    return !type_ok(type) || sums == 0 ? 0 : codes_bytes(cols, n) + scales_bytes(n) + sums;
}

int psk_linear_i8(const psk_i8 *A, int64_t n, int type, const void *X, int64_t ldx, const float *bias, void *Y, int64_t ldy, void *workspace,
                  size_t workspace_bytes, void *stream)
{
    if (!type_ok(type)) return PSK_ERR_UNSUPPORTED;
    const int st = check_i8(A, PSK_I8_MAX_COLS);
    if (st != PSK_OK) return st;
    if (n < 0 || n > PSK_MAX_VECTORS || !ld_ok(ldx, A->cols) || !ld_ok(ldy, A->rows)) return PSK_ERR_SIZE;
    if (!workspace_ok(workspace, workspace_bytes, psk_linear_i8_workspace_bytes(A->rows, A->cols, n, type))) return PSK_ERR_WORKSPACE;
    if (n == 0 || A->rows == 0) return PSK_OK;
    if (!Y || (A->cols > 0 && !X)) return PSK_ERR_NULL;
    if (misaligned(X, bytes_of(type)) || misaligned(Y, bytes_of(type)) || misaligned(bias, 4)) return PSK_ERR_ALIGNMENT;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (gemv_i8_takes((int)A->cols, (int)n))
        return hip_status(launch_gemv_i8((int)A->rows, (int)A->cols, (int)n, A->codes, A->ld, A->scales, X, ldx, nullptr, bias, type, Y, ldy, s));
    const int64_t ld = line(A->cols);
    int8_t *const codes = static_cast<int8_t *>(workspace);
    float *const scales = reinterpret_cast<float *>(codes + codes_bytes(A->cols, n));
    void *const sums = reinterpret_cast<char *>(scales) + scales_bytes(n);
    const hipError_t e = launch_quant_i8((int)n, (int)A->cols, (int)ld, type, X, ldx, codes, ld, scales, s);
    if (e != hipSuccess) return PSK_ERR_HIP;
    return hip_status(launch_gemm_i8((int)A->rows, (int)A->cols, (int)n, A->codes, A->ld, A->scales, codes, ld, scales, bias, type, Y, ldy, sums, s));
}

int psk_embed(int64_t n, int64_t rows, int64_t dim, const int32_t *ids, float factor, int type, const void *E, int64_t lde, int ytype, void *Y,
              int64_t ldy, void *stream)
{
    if (!type_ok(type) || !type_ok(ytype)) return PSK_ERR_UNSUPPORTED;
    if (n < 0 || n > PSK_MAX_TOKENS || rows < 0 || rows > kMaxEdge || dim < 0 || dim > kMaxEdge || !ld_ok(lde, dim) || !ld_ok(ldy, dim)) return PSK_ERR_SIZE;
    if (n == 0 || dim == 0) return PSK_OK;
    if (!ids || !Y || (rows > 0 && !E)) return PSK_ERR_NULL;
    if (misaligned(ids, 4) || misaligned(E, bytes_of(type)) || misaligned(Y, bytes_of(ytype))) return PSK_ERR_ALIGNMENT;
    return hip_status(launch_embed((int)n, (int)rows, (int)dim, ids, factor, type, E, lde, nullptr, ytype, Y, ldy, static_cast<hipStream_t>(stream)));
}

int psk_embed_i8(const psk_i8 *E, int64_t n, const int32_t *ids, float factor, int ytype, void *Y, int64_t ldy, void *stream)
{
    if (!type_ok(ytype)) return PSK_ERR_UNSUPPORTED;
    const int st = check_i8(E, PSK_I8_MAX_LD);
    if (st != PSK_OK) return st;
    if (n < 0 || n > PSK_MAX_TOKENS || !ld_ok(ldy, E->cols)) return PSK_ERR_SIZE;
    if (n == 0 || E->cols == 0) return PSK_OK;
    if (!ids || !Y) return PSK_ERR_NULL;
    if (misaligned(ids, 4) || misaligned(Y, bytes_of(ytype))) return PSK_ERR_ALIGNMENT;
    return hip_status(launch_embed((int)n, (int)E->rows, (int)E->cols, ids, factor, kTableI8, E->codes, E->ld, E->scales, ytype, Y, ldy,
                                   static_cast<hipStream_t>(stream)));
}

size_t psk_embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t dim)
{
    if (n < 0 || n > PSK_MAX_TOKENS || rows < 0 || rows > kMaxEdge || dim < 0 || dim > kMaxEdge) return 0;
    return embed_grad_workspace_bytes(n, dim);
}

int psk_embed_grad(int64_t n, int64_t rows, int64_t dim, const int32_t *ids, int32_t padding, float factor, int type, const void *dY, int64_t ldy,
                   int gtype, void *dE, int64_t lde, int accumulate, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!type_ok(type) || (gtype != PSK_F32 && gtype != type)) return PSK_ERR_UNSUPPORTED;
    if (n < 0 || n > PSK_MAX_TOKENS || rows < 0 || rows > kMaxEdge || dim < 0 || dim > kMaxEdge || !ld_ok(ldy, dim) || !ld_ok(lde, dim)) return PSK_ERR_SIZE;
    if (!workspace_ok(workspace, workspace_bytes, embed_grad_workspace_bytes(n, dim))) return PSK_ERR_WORKSPACE;
    if (rows == 0 || dim == 0 || (n == 0 && accumulate)) return PSK_OK;
    if (!dE || (n > 0 && (!ids || !dY))) return PSK_ERR_NULL;
    if (misaligned(ids, 4) || misaligned(dY, bytes_of(type)) || misaligned(dE, bytes_of(gtype))) return PSK_ERR_ALIGNMENT;
    return hip_status(launch_embed_grad((int)n, (int)rows, (int)dim, ids, padding, factor, type, dY, ldy, gtype, dE, lde, accumulate != 0, workspace,
                                        static_cast<hipStream_t>(stream)));
}

}  // extern "C"
