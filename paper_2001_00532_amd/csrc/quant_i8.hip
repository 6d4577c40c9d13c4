// Tokens in 8 bits (formulas: gemm_i8.h).  A workgroup per row; the first 8192 columns stay in registers between the two passes, later ones are read
// again.  Bound by reading the rows.
#include "gemm_i8.h"

namespace psk {
namespace {

// Columns from `cols` up to `fill` (a multiple of 16) become zeros.
template <int T>
__global__ __launch_bounds__(256) void k_quant(int n, int cols, int fill, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales)
{
    constexpr int KEPT = 4, ES = T == F32 ? 4 : 2;
    __shared__ unsigned part[4];
    for (int64_t t = blockIdx.x; t < n; t += gridDim.x) {
        const char *row = static_cast<const char *>(X) + t * ldx * ES;
        float v[KEPT][8];
        unsigned most = 0;
#pragma unroll
        for (int u = 0; u < KEPT; ++u) {
            const int k = 8 * (u * 256 + (int)threadIdx.x);
            if (k < cols) {
                load_cols<T>(row, k, cols, v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u][i] = 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < KEPT; ++u)
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, size_bits(v[u][i]));
        for (int k = 8 * (KEPT * 256 + (int)threadIdx.x); k < cols; k += 2048) {
            float w[8];
            load_cols<T>(row, k, cols, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, size_bits(w[i]));
        }
        most = wave_max(most);
        __syncthreads();                                   // the last row's maximum has been read
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
        const Quantiser q(max(max(part[0], part[1]), max(part[2], part[3])));
        if (threadIdx.x == 0) scales[t] = q.scale();
        int8_t *to = codes + t * ldc;
#pragma unroll
        for (int u = 0; u < KEPT; ++u) {
            const int k = 8 * (u * 256 + (int)threadIdx.x);
            if (k >= fill) break;
            int c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = q.code(v[u][i]);
            *reinterpret_cast<uint2 *>(to + k) = make_uint2(pack4(c), pack4(c + 4));
        }
        for (int k = 8 * (KEPT * 256 + (int)threadIdx.x); k < fill; k += 2048) {
            float w[8];
            load_cols<T>(row, k, cols, w);
            int c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = q.code(w[i]);
            *reinterpret_cast<uint2 *>(to + k) = make_uint2(pack4(c), pack4(c + 4));
        }
    }
}

}  // namespace

hipError_t launch_quant_i8(int n, int cols, int fill, int type, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales, hipStream_t s)
{
    const dim3 grid((unsigned)(n < 65536 ? n : 65536)), block(256);
    if (type == F32) PSK_LAUNCH((k_quant<F32>), grid, block, 0, s, n, cols, fill, X, ldx, codes, ldc, scales);
    else if (type == F16) PSK_LAUNCH((k_quant<F16>), grid, block, 0, s, n, cols, fill, X, ldx, codes, ldc, scales);
    else PSK_LAUNCH((k_quant<BF16>), grid, block, 0, s, n, cols, fill, X, ldx, codes, ldc, scales);
    return take_launch_status();
}

}  // namespace psk
