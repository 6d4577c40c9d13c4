// Y = X A^T in 8-bit integers (formulas: gemm_i8.h).
//
// Tiles of tokens x channels, 128 columns a step.  Both operands go from memory to LDS without passing registers, a step or more ahead of its use; a wave's
// load is 8 rows of 128 bytes, and which 16 bytes of its row a lane asks for is turned by the row, so that reading the operands' order (16 rows x 16
// bytes, row by row) meets each bank once.  One barrier a step: behind it the step's operands are there and the stage before is free.
#include "gemm_i8.h"

namespace psk {
namespace {

constexpr int STEP = 128;                                  // columns, and bytes of a row of a stage

// 16 bytes per lane from base + offset to LDS at `to` + 16 lane.
__device__ __forceinline__ void to_lds(const void *base, unsigned offset, const void *to)
{
    const unsigned at = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(offset), "s"(base) : "memory");
}
// All but the last N loads of this wave are there, its LDS reads are done, and so are those of the other waves.
template <int N>
__device__ __forceinline__ void step_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

template <int YT>
__device__ __forceinline__ void put4(void *Y, int64_t at, const float (&v)[4], int count)
{
    if (count >= 4) {
        if constexpr (YT == F32) {
            *reinterpret_cast<v4f_e *>(static_cast<float *>(Y) + at) = v4f{v[0], v[1], v[2], v[3]};
        } else {
            *reinterpret_cast<v4s_u *>(static_cast<unsigned short *>(Y) + at) = v4s{narrow<YT>(v[0]), narrow<YT>(v[1]), narrow<YT>(v[2]), narrow<YT>(v[3])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < count) store_as<YT>(Y, at + i, v[i]);
    }
}

// BT tokens x BR channels by WT x WR waves, S stages.
template <int YT, int BT, int BR, int WT, int WR, int S>
__global__ __launch_bounds__(64 * WT * WR) void k_gemm_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, Finish f, void *Y,
                                                          int64_t ldy, unsigned tiles_r, unsigned tiles)
{
    constexpr int NW = WT * WR, LOADS = (BT + BR) / 8 / NW, TT = BT / WT / 16, TR = BR / WR / 16, STAGE = (BT + BR) * STEP;
    static_assert((BT + BR) % (8 * NW) == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) int8_t lds[S * STAGE];
    const unsigned tile = blockIdx.y * gridDim.x + blockIdx.x;
    if (tile >= tiles) return;
    const int t0 = (int)(tile / tiles_r) * BT, r0 = (int)(tile % tiles_r) * BR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wave / WR, wr = wave % WR;
    const int blocks = (cols + STEP - 1) / STEP, most = ((cols + 15) & ~15) - 16 - (blocks - 1) * STEP;      // the last piece of the last step

    // where a lane's 16 bytes come from: row 8 q + lane / 8 of the stage, piece lane % 8 turned by the row
    const int8_t *const x0 = X + (int64_t)t0 * ldx, *const a0 = A + (int64_t)r0 * lda;
    const int8_t *base[LOADS];
    unsigned from[LOADS], end[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int q = i * NW + wave, row = 8 * q + (lane >> 3), piece = 16 * ((lane & 7) ^ (lane >> 3));
        const bool x = 8 * q < BT;
        base[i] = x ? x0 : a0;
        from[i] = x ? (unsigned)min(row, n - 1 - t0) * (unsigned)ldx : (unsigned)min(row - BT, rows - 1 - r0) * (unsigned)lda;
        end[i] = from[i] + (unsigned)min(piece, most);
        from[i] += (unsigned)piece;
    }
    auto fetch = [&](int step) {
        int8_t *const to = lds + step % S * STAGE + wave * 1024;
        const int64_t k = (int64_t)step * STEP;
        if (step < blocks - 1) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) to_lds(base[i] + k, from[i], to + i * NW * 1024);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) to_lds(base[i] + k, end[i], to + i * NW * 1024);
        }
    };
    for (int k = 0; k < S - 1 && k < blocks; ++k) fetch(k);

    v4i acc[TR][TT];
#pragma unroll
    for (int r = 0; r < TR; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = v4i{0, 0, 0, 0};
    const int in16 = lane & 15, quarter = lane >> 4;
    for (int k = 0; k < blocks; ++k) {
        if (k + S - 2 < blocks - 1) step_barrier<(S - 2) * LOADS>();
        else step_barrier<0>();
        if (k + S - 1 < blocks) fetch(k + S - 1);
        const int8_t *const st = lds + k % S * STAGE;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int place = in16 * STEP + 16 * ((4 * h + quarter) ^ (lane & 7));
            v4i x[TT], a[TR];
#pragma unroll
            for (int t = 0; t < TT; ++t) x[t] = *reinterpret_cast<const v4i *>(st + ((wt * TT + t) * 16) * STEP + place);
#pragma unroll
            for (int r = 0; r < TR; ++r) a[r] = *reinterpret_cast<const v4i *>(st + (BT + (wr * TR + r) * 16) * STEP + place);
            if (k == blocks - 1) {
#pragma unroll
                for (int t = 0; t < TT; ++t) x[t] = first_bytes(x[t], cols - k * STEP - 64 * h - 16 * quarter);
            }
#pragma unroll
            for (int r = 0; r < TR; ++r)
#pragma unroll
                for (int t = 0; t < TT; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[r], x[t], acc[r][t], 0, 0, 0);
        }
    }
    // channel 4 (lane / 16) + i of token lane % 16
#pragma unroll
    for (int r = 0; r < TR; ++r) {
        const int row = r0 + (wr * TR + r) * 16 + 4 * quarter;
        float a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = f.a[min(row + i, rows - 1)];
            b[i] = f.bias ? f.bias[min(row + i, rows - 1)] : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < TT; ++t) {
            const int token = t0 + (wt * TT + t) * 16 + in16;
            if (token >= n || row >= rows) continue;
            const float s = f.s[token];
            const float v[4] = {finish(acc[r][t][0], a[0], s, b[0]), finish(acc[r][t][1], a[1], s, b[1]), finish(acc[r][t][2], a[2], s, b[2]),
                                finish(acc[r][t][3], a[3], s, b[3])};
            put4<YT>(Y, token * ldy + row, v, rows - row);
        }
    }
}

template <int YT, int BT, int BR, int WT, int WR, int S>
void tiles(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, hipStream_t s)
{
    const unsigned r = (unsigned)((rows + BR - 1) / BR), all = r * (unsigned)((n + BT - 1) / BT), x = all < 65536 ? all : 65536;
    PSK_LAUNCH((k_gemm_i8<YT, BT, BR, WT, WR, S>), dim3(x, (all + x - 1) / x), dim3(64 * WT * WR), 0, s, rows, cols, n, A, lda, X, ldx, f, Y, ldy, r, all);
}

template <int YT>
hipError_t launch(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, hipStream_t s)
{
    if (n <= 64) tiles<YT, 32, 64, 1, 4, 4>(rows, cols, n, A, lda, X, ldx, f, Y, ldy, s);
    else if (n <= 512) tiles<YT, 128, 128, 2, 2, 3>(rows, cols, n, A, lda, X, ldx, f, Y, ldy, s);
    else tiles<YT, 256, 256, 2, 4, 2>(rows, cols, n, A, lda, X, ldx, f, Y, ldy, s);
    return take_launch_status();
}

}  // namespace

hipError_t launch_gemm_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const float *a, const int8_t *X, int64_t ldx, const float *xs, const float *bias,
                          int type, void *Y, int64_t ldy, hipStream_t s)
{
    const Finish f = {a, xs, bias};
    const auto go = type == F32 ? launch<F32> : (type == F16 ? launch<F16> : launch<BF16>);
    return go(rows, cols, n, A, lda, X, ldx, f, Y, ldy, s);
}

}  // namespace psk
