// Y = X A^T, A in 4 bits with a scale per group of columns, a few vectors X.
//
//   Y[t][i] = sum_g s_ig sum_{j in g} (q_ij - z_ig) X[t][j]
//
// The codes less their zero points are exact in the operands, and the scale multiplies a group's sum in 32 bits, so only sums and the result
// are rounded.  Bound by reading the codes once (half a byte per weight) and, from five vectors on, by the instructions that
// dequantise them.  A workgroup owns 16 R rows; its waves share the columns, and their sums meet in LDS.
//
// Three ways, by the rules in by_group, more_vectors and few_vectors_by_columns:
//   up to four vectors            k_gemv_q4        32768 x 8192, one vector of bf16, groups of 64: 29.7 us = 4.8 TB/s of codes and scales
//   more, up to 4096 (f32: 2048) columns  k_gemm_q4_kept   10240 x 4096, 16 vectors of bf16: 11.0 us; 8192 x 4096, 64 vectors of f16: 16.5 us
//   more, longer rows             k_gemm_q4        4096 x 8192, 16 vectors of bf16: 9.6 us; 64 vectors of f16: 17.4 us
#pragma once
#include "psk_internal.h"
#include "psk_mfma.h"

namespace psk {
namespace {

template <int XT> struct Vectors { typedef Plain16<XT> type; };
template <> struct Vectors<F32> { typedef Parts32 type; };

// Up to four vectors, 16 R rows.  A matrix instruction has room for 16 vectors: its rows 4 v + j hold columns of block j of vector v, so four
// blocks of columns are one load of vectors, and of each block's product the lane keeps the element that is its vector's.
// R = 1: two sets of rows per workgroup are slower (32768 x 8192 29 to 33 us, with one 28; 4096 x 4096 6.9 and 4.8), there are fewer waves to
// ask for memory.
template <int XT, int S, int GB, bool Z, int R, int P, int KW>
__global__ __launch_bounds__(64 * KW) void k_gemv_q4(WeightsQ4 A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16;
    typedef SpanQ4<T, R, P, GB, S, Z> SPAN;
    __shared__ float lds[KW * R * 64];
    __shared__ v4u places[KW * EXCHANGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = blockIdx.x * (16 * R);
    SPAN span;
#pragma unroll
    for (int r = 0; r < R; ++r) span.set(r, A, 0, row0 + 16 * r, A.rows, lane, A.cols);
    typename Vectors<XT>::type x;
    x.set(X, min(lane >> 2 & 3, n - 1) * ldx + few_column<SPAN>(lane));
    float y[R];
    few_product(span, x, A.cols, wave, KW, lane, Exchange(places + EXCHANGE * wave, lane), y);
    put_few<R>(lds, wave, lane, y);
    __syncthreads();
    for (int o = threadIdx.x; o < 64 * R; o += 64 * KW) {
        const int r = o >> 6, v = o >> 4 & 3, i = o & 15;
        if (v < n && row0 + 16 * r + i < A.rows) store_as<XT>(Y, v * ldy + row0 + 16 * r + i, get_sum<KW, R, 4>(lds, r, v, i) * SPAN::unit);
    }
}

// The copy of the vectors for k_gemm_q4 (and of those of 32 bits for k_gemm_q4_kept), in the order of the operands: a lane's load is then 16 bytes of a
// kilobyte in one piece, where the rows themselves would cost a compute unit twice the time.  A wave per tile and four blocks.
template <int XT, int GB>
__global__ __launch_bounds__(256) void k_gemm_q4_copy(int n, int cols, const void *X, int64_t ldx, v4u *copy)
{
    typedef typename Vectors<XT>::type V;
    typedef SpanQ4<XT == F16 ? F16 : BF16, 1, 2, GB, F32, false> SPAN;
    const int lane = threadIdx.x & 63, block = blockIdx.x * 4 + (threadIdx.x >> 6), tile = blockIdx.y, blocks = copied_blocks(cols);
    V x;
    x.set(X, min(16 * tile + (lane & 15), n - 1) * ldx);
    copy_block<SPAN>(x, cols, block, lane, copy + (int64_t)tile * blocks * V::P * 64);
}

// NT tiles of 16 vectors, 16 R rows: for rows that are too long to keep the vectors.
template <int XT, int S, int GB, bool Z, int R, int NT, int KW>
__global__ __launch_bounds__(64 * KW) void k_gemm_q4(WeightsQ4 A, int n, const v4u *copy, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16;
    typedef SpanQ4<T, R, 2, GB, S, Z> SPAN;
    __shared__ float lds[KW * R * NT * 256];
    __shared__ v4u places[KW * EXCHANGE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = blockIdx.x * (16 * R), t0 = blockIdx.y * NT, last = (n - 1) >> 4, blocks = copied_blocks(A.cols);
    SPAN span;
#pragma unroll
    for (int r = 0; r < R; ++r) span.set(r, A, 0, row0 + 16 * r, A.rows, lane, A.cols);
    Copied<typename Vectors<XT>::type> x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) x[t].set(copy, min(t0 + t, last), blocks, lane);
    v4f acc[R][NT], flat[R * NT];
    tile_product<SPAN, NT>(span, x, A.cols, wave, KW, Exchange(places + EXCHANGE * wave, lane), acc);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) flat[r * NT + t] = acc[r][t];
    put_sums<R * NT>(lds, wave, lane, flat);
    __syncthreads();
    for (int o = threadIdx.x; o < R * NT * 256; o += 64 * KW) {
        const int k = o >> 8, v = 16 * (t0 + k % NT) + (o >> 4 & 15), i = row0 + 16 * (k / NT) + (o & 15);
        if (v < n && i < A.rows) store_as<XT>(Y, v * ldy + i, get_sum<KW, R * NT, 16>(lds, k, o >> 4 & 15, o & 15) * SPAN::unit);
    }
}

// Up to 256 KW columns: the vectors kept (KeptQ4), workgroups that stay.  16-bit vectors are brought into the operands' order here; those of 32
// bits come from the copy.  Takes 9 vector instructions per eight codes of f16 and 19 of bf16, and these bound it: weights of two or three sets
// of rows requested ahead instead of one take as long (10.3, 11.1 and 11.5 us for 10240 x 4096 times 16).
// 10240 x 4096 times 16 vectors 10.2 us, by k_gemm_q4 with its copy 13.3; 8192 x 4096 times 64 16.5, by k_gemm_q4 23.
// Beyond 4096 columns it would take more than the 16 waves of a workgroup.
// Vectors of 32 bits hold three parts, of which 16 waves do not fit into the registers, so they are kept up to 2048 columns only: 10240 x 4096 times 16
// 19.9 us by k_gemm_q4, 23.2 kept; 8192 x 4096 times 64 42.7 and 59.6; 8192 x 2048 times 64 24.9 and 19.6, times 16 (10240 rows) 10.2 and 11.6.
template <int XT, int S, int GB, int KW>
__global__ __launch_bounds__(64 * KW) void k_gemm_q4_kept(WeightsQ4 A, int n, const void *X, int64_t ldx, const v4u *copy, void *Y, int64_t ldy)
{
    constexpr int T = XT == F16 ? F16 : BF16;
    typedef typename Vectors<XT>::type V;
    typedef KeptQ4<T, 1, GB, S, KW, V> K;
    __shared__ typename K::Space space;
    const int tile = blockIdx.y;
    const WeightsQ4 w[1] = {A};
    K k(space, w, 0, A.rows, A.cols);
    if constexpr (XT == F32) {
        Copied<V> x;
        x.set(copy, tile, copied_blocks(A.cols), k.lane);
        keep_copied(k, x);
    } else {
        keep_rows<T>(k, static_cast<const unsigned short *>(X), ldx, n, tile);
    }
    k.run(blockIdx.x, gridDim.x, (A.rows + 15) / 16, [&](int set, const float *sums) {
        for (int o = threadIdx.x; o < 256; o += 64 * KW) {
            const int v = 16 * tile + (o >> 4), i = set * 16 + (o & 15);
            if (v < n && i < A.rows) store_as<XT>(Y, v * ldy + i, get_sum<KW, 1, 16>(sums, 0, o >> 4, o & 15) * K::unit);
        }
    });
}

template <int XT, int S, int GB, bool Z, int P>
void few_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    PSK_LAUNCH((k_gemv_q4<XT, S, GB, Z, 1, P, 4>), dim3((A.rows + 15) / 16), dim3(256), 0, s, A, n, X, ldx, Y, ldy);
}
// Four pieces of 128 columns in a chunk for long rows, two for short ones, of which no wave would else get one: 4096 x 4096 4.4 us (two: 5.3),
// 1024 x 1024 2.9 (two: 2.7).  Vectors of 32 bits: two, four would not fit into the registers.
template <int XT, int S, int GB, bool Z>
void few_vectors_by_columns(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, hipStream_t s)
{
    constexpr int LONG = XT == F32 ? 2 : 4;
    // (GB = 8 stands for groups of 256 columns and more, of which a long chunk may hold two)
    if (A.cols >= 2048 && GB == 8 && A.shift > 8) few_vectors<XT, S, GB == 8 ? 4 * LONG : GB, Z, LONG>(A, n, X, ldx, Y, ldy, s);
    else if (A.cols >= 2048) few_vectors<XT, S, GB, Z, LONG>(A, n, X, ldx, Y, ldy, s);
    else few_vectors<XT, S, GB, Z, 2>(A, n, X, ldx, Y, ldy, s);
}
// Workgroups for KeptQ4: as many as are on the chip at once (1024 threads to a compute unit) for all tiles together, no more than sets of rows.
// 8192 x 4096 times 64, 16 waves: 64 workgroups for each of four tiles 16.7 us, 128 19.5, 256 26; 10240 x 2048 times 16, 8 waves: 512 6.5 us, 320 7.1, 256 6.7.
inline int kept_groups(int sets, int tiles, int kw)
{
    const int n = 256 * (16 / kw) / tiles;
    return n < 1 ? 1 : (n < sets ? n : sets);
}
template <int XT, int S, int GB, int KW>
void kept_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, const v4u *copy, hipStream_t s)
{
    const int rows = (A.rows + 15) / 16, tiles = (n + 15) / 16;
    PSK_LAUNCH((k_gemm_q4_kept<XT, S, GB, KW>), dim3(kept_groups(rows, tiles, KW), tiles), dim3(64 * KW), 0, s, A, n, X, ldx, copy, Y, ldy);
}
template <int XT, int S, int GB>
void more_vectors(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, void *space, hipStream_t s)
{
    const int rows = (A.rows + 15) / 16, tiles = (n + 15) / 16;
    v4u *copy = static_cast<v4u *>(space);
    const bool kept = kept_fits(A) && (XT != F32 || A.cols <= 2048);
    // Longer rows: one tile and set of rows per workgroup where there is one tile (10240 x 4096 times 16 13.3 us, two sets of rows 13.7 to 15.7) or there
    // would be few workgroups (2048 x 8192 times 32 9.0 us, two and two 15.9; 2048 x 8192 times 64, 512 workgroups, in f32 27, two sets of rows 20).
    // (kept vectors are in natural order, as for groups of 32 columns)
    if (!kept) PSK_LAUNCH((k_gemm_q4_copy<XT, GB>), dim3(copied_blocks(A.cols) / 4, tiles), dim3(256), 0, s, n, A.cols, X, ldx, copy);
    else if (XT == F32) PSK_LAUNCH((k_gemm_q4_copy<XT, 1>), dim3(copied_blocks(A.cols) / 4, tiles), dim3(256), 0, s, n, A.cols, X, ldx, copy);
    if (kept) {
        if (A.cols <= 1024) kept_vectors<XT, S, GB, 4>(A, n, X, ldx, Y, ldy, copy, s);
        else if (XT == F32 || A.cols <= 2048) kept_vectors<XT, S, GB, 8>(A, n, X, ldx, Y, ldy, copy, s);
        else if constexpr (XT != F32) kept_vectors<XT, S, GB, 16>(A, n, X, ldx, Y, ldy, copy, s);
    } else if (tiles == 1 || (int64_t)rows * tiles <= 256) PSK_LAUNCH((k_gemm_q4<XT, S, GB, true, 1, 1, 4>), dim3(rows, tiles), dim3(256), 0, s, A, n, copy, Y, ldy);
    else if constexpr (XT == F32) PSK_LAUNCH((k_gemm_q4<XT, S, GB, true, 2, 1, 4>), dim3((rows + 1) / 2, tiles), dim3(256), 0, s, A, n, copy, Y, ldy);
    else PSK_LAUNCH((k_gemm_q4<XT, S, GB, true, 2, 2, 4>), dim3((rows + 1) / 2, (tiles + 1) / 2), dim3(256), 0, s, A, n, copy, Y, ldy);
}
template <int XT, int S>
void by_group(const WeightsQ4 &A, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, void *space, hipStream_t s)
{
    // four vectors: 10240 x 4096 8.6 us here, 10.1 with the vectors kept; 2048 x 1024 2.9 and 4.0
    if (n > 4) {
        if (A.shift == 5) more_vectors<XT, S, 1>(A, n, X, ldx, Y, ldy, space, s);
        else if (A.shift == 6) more_vectors<XT, S, 2>(A, n, X, ldx, Y, ldy, space, s);
        else if (A.shift == 7) more_vectors<XT, S, 4>(A, n, X, ldx, Y, ldy, space, s);
        else more_vectors<XT, S, 8>(A, n, X, ldx, Y, ldy, space, s);
        return;
    }
#define PSK_FEW(GB) (A.zeros ? few_vectors_by_columns<XT, S, GB, true>(A, n, X, ldx, Y, ldy, s) : few_vectors_by_columns<XT, S, GB, false>(A, n, X, ldx, Y, ldy, s))
    if (A.shift == 5) PSK_FEW(1);
    else if (A.shift == 6) PSK_FEW(2);
    else if (A.shift == 7) PSK_FEW(4);
    else PSK_FEW(8);
#undef PSK_FEW
}

}  // namespace

template <int XT>
hipError_t launch_gemm_q4_of(const WeightsQ4 &A, int scale_type, int n, const void *X, int64_t ldx, void *Y, int64_t ldy, void *space, hipStream_t s)
{
    if (XT != F32 && scale_type == XT) by_group<XT, XT>(A, n, X, ldx, Y, ldy, space, s);
    else by_group<XT, F32>(A, n, X, ldx, Y, ldy, space, s);
    return take_launch_status();
}

}  // namespace psk
