// Y = X A^T, A in 4 bits with a scale per group of columns, a few vectors X.
//
//   Y[t][i] = sum_g s_ig sum_{j in g} (q_ij - z_ig) X[t][j]
//
// Bound by reading the codes once (half a byte per weight).  A workgroup owns 16 rows; its waves take turns at chunks of 128
// columns, so that together they read consecutive pieces of the rows, and their sums meet in LDS.
#include "psk_internal.h"
#include "psk_mfma.h"

namespace psk {
namespace {

constexpr int KW = 8;

template <int XT, int S, int GB, int NT>
__global__ __launch_bounds__(64 * KW) void k_gemm_q4(WeightsQ4 A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16, PER = XT == F32 ? 5 : 16;
    __shared__ float lds[KW * NT * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    const int row0 = blockIdx.x * 16, t0 = blockIdx.y * (PER * NT);
    SpanQ4<T, 1, GB, S> span;
    span.set(0, A, 0, min(row0 + m, A.rows - 1), quarter);
    v4f acc[1][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[0][t] = v4f{0, 0, 0, 0};
    if constexpr (XT == F32) {
        Rows32<NT> x;
        x.cols = A.cols;
        x.part = m % 3;
#pragma unroll
        for (int t = 0; t < NT; ++t) x.p[t] = static_cast<const float *>(X) + (int64_t)min(t0 + PER * t + m / 3, n - 1) * ldx;
        span_product<SpanQ4<T, 1, GB, S>, NT>(span, x, A.cols, wave, KW, quarter, acc);
    } else {
        Rows16<NT> x;
        x.cols = A.cols;
#pragma unroll
        for (int t = 0; t < NT; ++t) x.p[t] = static_cast<const unsigned short *>(X) + (int64_t)min(t0 + PER * t + m, n - 1) * ldx;
        span_product<SpanQ4<T, 1, GB, S>, NT>(span, x, A.cols, wave, KW, quarter, acc);
    }
    put_sums<NT>(lds, wave, lane, acc[0]);
    __syncthreads();
    for (int o = threadIdx.x; o < NT * PER * 16; o += 64 * KW) {
        const int tile = o / (PER * 16), v = o / 16 % PER, i = o % 16;
        if (t0 + tile * PER + v >= n || row0 + i >= A.rows) continue;
        float y;
        if constexpr (XT == F32)
            y = get_sum<KW, NT>(lds, tile, 3 * v, i) + (get_sum<KW, NT>(lds, tile, 3 * v + 1, i) + get_sum<KW, NT>(lds, tile, 3 * v + 2, i));
        else
            y = get_sum<KW, NT>(lds, tile, v, i);
        store_as<XT>(Y, (int64_t)(t0 + tile * PER + v) * ldy + row0 + i, y);
    }
}

template <int XT, int S, int GB>
void by_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    constexpr int PER = XT == F32 ? 5 : 16;
    const int tiles = (n + PER - 1) / PER, rows = (A.rows + 15) / 16;
    if (tiles <= 1) PSK_LAUNCH((k_gemm_q4<XT, S, GB, 1>), dim3(rows, 1), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
    else if (tiles == 2) PSK_LAUNCH((k_gemm_q4<XT, S, GB, 2>), dim3(rows, 1), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
    else PSK_LAUNCH((k_gemm_q4<XT, S, GB, 4>), dim3(rows, (tiles + 3) / 4), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
}
template <int XT, int S>
void by_group(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    if (A.shift == 5) by_vectors<XT, S, 1>(A, n, X, ldx, Y, ldy, s);
    else if (A.shift == 6) by_vectors<XT, S, 2>(A, n, X, ldx, Y, ldy, s);
    else by_vectors<XT, S, 4>(A, n, X, ldx, Y, ldy, s);
}

}  // namespace

hipError_t launch_gemm_q4(const WeightsQ4 &A, int scale_type, int n, int type, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    if (type == F32) by_group<F32, F32>(A, n, X, ldx, Y, ldy, s);
    else if (type == F16 && scale_type == F16) by_group<F16, F16>(A, n, X, ldx, Y, ldy, s);
    else if (type == F16) by_group<F16, F32>(A, n, X, ldx, Y, ldy, s);
    else if (scale_type == BF16) by_group<BF16, BF16>(A, n, X, ldx, Y, ldy, s);
    else by_group<BF16, F32>(A, n, X, ldx, Y, ldy, s);
    return take_launch_status();
}

}  // namespace psk
