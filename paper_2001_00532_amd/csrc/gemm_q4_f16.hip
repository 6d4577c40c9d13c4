// Products with 4-bit weights, vectors of type f16 (gemm_q4.h).
#include "gemm_q4.h"

namespace psk {
template hipError_t launch_gemm_q4_of<F16>(const WeightsQ4 &A, int scale_type, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, void *space, hipStream_t s);
}
