// Tokens in 8 bits (formulas: gemm_i8.h).  A workgroup per row; the first 8192 columns stay in registers between the two passes, later ones are read
// again.  Bound by reading the rows: 2048 x 4096 bf16 in 7.7 us, 3.3 TB/s read and written; 32 rows 3.7, a launch and one trip to memory;
// 131072 x 4096 286 us, 5.6 TB/s.
#include "gemm_i8.h"

namespace psk {
namespace {

// Columns from `cols` up to `fill` (a multiple of 16) become zeros.
// KEPT: pieces of 2048 columns that stay (2048 x 4096: 9.6 us with four of them for the two there are).
template <int T, int KEPT>
__global__ __launch_bounds__(256) void k_quant(int n, int cols, int fill, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales)
{
    constexpr int ES = T == F32 ? 4 : 2;
    __shared__ unsigned part[4];
    for (int64_t t = blockIdx.x; t < n; t += gridDim.x) {
        const char *row = static_cast<const char *>(X) + t * ldx * ES;
        Raw8<T> raw[KEPT];
        unsigned most = 0;
#pragma unroll
        for (int u = 0; u < KEPT; ++u) row_load<T>(raw[u], row, 8 * (u * 256 + (int)threadIdx.x), cols);
#pragma unroll
        for (int u = 0; u < KEPT; ++u) {
            float v[8];
            row_get<T>(raw[u], 8 * (u * 256 + (int)threadIdx.x), cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, size_bits(v[i]));
        }
        for (int k = 8 * (KEPT * 256 + (int)threadIdx.x); k < cols; k += 2048) {
            Raw8<T> r;
            float v[8];
            row_load<T>(r, row, k, cols);
            row_get<T>(r, k, cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = max(most, size_bits(v[i]));
        }
        most = wave_max(most);
        __syncthreads();                                   // the last row's maximum has been read
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
        __syncthreads();
        const Quantiser q(max(max(part[0], part[1]), max(part[2], part[3])));
        if (threadIdx.x == 0) scales[t] = q.scale();
        int8_t *to = codes + t * ldc;
        auto put = [&](const Raw8<T> &r, int k) {
            float v[8];
            int c[8];
            row_get<T>(r, k, cols, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = q.code(v[i]);
            *reinterpret_cast<uint2 *>(to + k) = make_uint2(pack4(c), pack4(c + 4));
        };
#pragma unroll
        for (int u = 0; u < KEPT; ++u) {
            const int k = 8 * (u * 256 + (int)threadIdx.x);
            if (k < fill) put(raw[u], k);
        }
        for (int k = 8 * (KEPT * 256 + (int)threadIdx.x); k < fill; k += 2048) {
            Raw8<T> r;
            row_load<T>(r, row, k, cols);
            put(r, k);
        }
    }
}

// Less than eight columns: a thread per row.
template <int T>
__global__ __launch_bounds__(256) void k_quant_short(int n, int cols, int fill, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales)
{
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < n; t += (int64_t)gridDim.x * 256) {
        unsigned most = 0;
        for (int k = 0; k < cols; ++k) most = max(most, size_bits(element<T>(X, t * ldx + k)));
        const Quantiser q(most);
        scales[t] = q.scale();
        for (int k = 0; k < fill; ++k) codes[t * ldc + k] = (int8_t)(k < cols ? q.code(element<T>(X, t * ldx + k)) : 0);
    }
}

template <int T>
void launch(int n, int cols, int fill, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales, hipStream_t s)
{
    const int64_t blocks = cols < 8 ? ((int64_t)n + 255) / 256 : n;
    const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536)), block(256);
    if (cols < 8) PSK_LAUNCH((k_quant_short<T>), grid, block, 0, s, n, cols, fill, X, ldx, codes, ldc, scales);
    else PSK_LAUNCH((cols <= 2048 ? k_quant<T, 1> : (cols <= 4096 ? k_quant<T, 2> : k_quant<T, 4>)), grid, block, 0, s, n, cols, fill, X, ldx, codes, ldc, scales);
}

}  // namespace

hipError_t launch_quant_i8(int n, int cols, int fill, int type, const void *X, int64_t ldx, int8_t *codes, int64_t ldc, float *scales, hipStream_t s)
{
    const auto go = type == F32 ? launch<F32> : (type == F16 ? launch<F16> : launch<BF16>);
    go(n, cols, fill, X, ldx, codes, ldc, scales, s);
    return take_launch_status();
}

}  // namespace psk
