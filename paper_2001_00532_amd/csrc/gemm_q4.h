// Y = X A^T, A in 4 bits with a scale per group of columns, a few vectors X.
//
//   Y[t][i] = sum_g s_ig sum_{j in g} (q_ij - z_ig) X[t][j]
//
// Bound by reading the codes once (half a byte per weight).  A workgroup owns 16 rows; its waves take turns at chunks of 128
// columns, so that together they read consecutive pieces of the rows, and their sums meet in LDS.
#pragma once
#include "psk_internal.h"
#include "psk_mfma.h"

namespace psk {
namespace {

constexpr int KW = 8;

template <int XT> struct Vectors { typedef Plain16<XT> type; };
template <> struct Vectors<F32> { typedef Parts32 type; };

// Up to four vectors, 16 R rows.
template <int XT, int S, int GB, bool Z, int R>
__global__ __launch_bounds__(64 * KW) void k_gemv_q4(WeightsQ4 A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16;
    __shared__ float lds[KW * R * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    const int row0 = blockIdx.x * (16 * R);
    SpanQ4<T, R, 2, GB, S, Z> span;
#pragma unroll
    for (int r = 0; r < R; ++r) span.set(r, A, 0, min(row0 + 16 * r + m, A.rows - 1), quarter, A.cols);
    typename Vectors<XT>::type x;
    x.set(X, min(m >> 2, n - 1) * ldx + 32 * (m & 3) + 8 * quarter);
    float y[R];
    few_product(span, x, A.cols, wave, KW, lane, y);
    put_few<R>(lds, wave, lane, y);
    __syncthreads();
    for (int o = threadIdx.x; o < 64 * R; o += 64 * KW) {
        const int r = o >> 6, v = o >> 4 & 3, i = o & 15;
        if (v < n && row0 + 16 * r + i < A.rows) store_as<XT>(Y, v * ldy + row0 + 16 * r + i, get_sum<KW, R, 4>(lds, r, v, i));
    }
}

// NT tiles of 16 vectors, 16 R rows.
template <int XT, int S, int GB, int R, int NT>
__global__ __launch_bounds__(64 * KW) void k_gemm_q4(WeightsQ4 A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16;
    __shared__ float lds[KW * R * NT * 256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    const int row0 = blockIdx.x * (16 * R), t0 = blockIdx.y * (16 * NT);
    SpanQ4<T, R, 1, GB, S, true> span;
#pragma unroll
    for (int r = 0; r < R; ++r) span.set(r, A, 0, min(row0 + 16 * r + m, A.rows - 1), quarter, A.cols);
    typename Vectors<XT>::type x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t].set(X, min(t0 + 16 * t + m, n - 1) * ldx + 8 * quarter);
    v4f acc[R][NT], flat[R * NT];
    tile_product<SpanQ4<T, R, 1, GB, S, true>, NT>(span, x, A.cols, wave, KW, lane, acc);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) flat[r * NT + t] = acc[r][t];
    put_sums<R * NT>(lds, wave, lane, flat);
    __syncthreads();
    for (int o = threadIdx.x; o < R * NT * 256; o += 64 * KW) {
        const int k = o >> 8, v = t0 + 16 * (k % NT) + (o >> 4 & 15), i = row0 + 16 * (k / NT) + (o & 15);
        if (v < n && i < A.rows) store_as<XT>(Y, v * ldy + i, get_sum<KW, R * NT, 16>(lds, k, o >> 4 & 15, o & 15));
    }
}

template <int XT, int S, int GB, bool Z>
void few_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    const int rows = (A.rows + 15) / 16;
    if (rows >= 2048) PSK_LAUNCH((k_gemv_q4<XT, S, GB, Z, 2>), dim3((rows + 1) / 2), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
    else PSK_LAUNCH((k_gemv_q4<XT, S, GB, Z, 1>), dim3(rows), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
}
template <int XT, int S, int GB>
void more_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    const int rows = (A.rows + 15) / 16;
    if (n <= 16) PSK_LAUNCH((k_gemm_q4<XT, S, GB, 1, 1>), dim3(rows, 1), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
    else PSK_LAUNCH((k_gemm_q4<XT, S, GB, 2, 2>), dim3((rows + 1) / 2, (n + 31) / 32), dim3(64 * KW), 0, s, A, n, X, ldx, Y, ldy);
}
template <int XT, int S>
void by_group(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    if (n > 4) {
        if (A.shift == 5) more_vectors<XT, S, 1>(A, n, X, ldx, Y, ldy, s);
        else if (A.shift == 6) more_vectors<XT, S, 2>(A, n, X, ldx, Y, ldy, s);
        else more_vectors<XT, S, 4>(A, n, X, ldx, Y, ldy, s);
        return;
    }
#define PSK_FEW(GB) (A.zeros ? few_vectors<XT, S, GB, true>(A, n, X, ldx, Y, ldy, s) : few_vectors<XT, S, GB, false>(A, n, X, ldx, Y, ldy, s))
    if (A.shift == 5) PSK_FEW(1);
    else if (A.shift == 6) PSK_FEW(2);
    else if (A.shift == 7) PSK_FEW(4);
    else PSK_FEW(8);
#undef PSK_FEW
}

}  // namespace

template <int XT>
hipError_t launch_gemm_q4_of(const WeightsQ4 &A, int scale_type, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    if (XT != F32 && scale_type == XT) by_group<XT, XT>(A, n, X, ldx, Y, ldy, s);
    else by_group<XT, F32>(A, n, X, ldx, Y, ldy, s);
    return take_launch_status();
}

}  // namespace psk
