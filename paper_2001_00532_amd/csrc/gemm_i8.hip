// Y = X A^T in 8-bit integers (formulas: gemm_i8.h).
//
// Tiles of tokens x channels, 128 columns a step.  Both operands go from memory to LDS without passing registers, a step or more ahead of its use; a wave's
// load is 8 rows of 128 bytes (in whole lines: steps of 64 columns, with twice the stages, took 477 us where these took 424, both with zeros for data), and which 16 bytes of its row a
// lane asks for is turned by the row, so that reading the operands' order meets each bank once.  One barrier a step: behind it the step's operands are there and
// the stage before is free.
//
// 8192 tokens x 16384 channels x 4096 columns: 427 to 436 us a call, 2.5 to 2.6 POP/s; 449 to 452 in a trace.  Power bounds it: an earlier form took 486 us,
// and with zeros for data 388.  2048 x 8192 x 4096: 55 us, a tile to a compute unit.
#include "gemm_i8.h"
#include "gemm_i8_plan.h"

namespace psk {
namespace {

constexpr int M = 16;                                      // channels and tokens of a matrix instruction, over 64 columns (32 x 32 x 32: 531 us for 486)

// 16 bytes per lane from base + offset to LDS at `to` + 16 lane.
__device__ __forceinline__ void to_lds(const void *base, unsigned offset, const void *to)
{
    const unsigned at = (unsigned)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)to);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(offset), "s"(base) : "m0", "memory");
}
// All but the last N loads of this wave are there, its LDS reads are done, and so are those of the other waves.
template <int N>
__device__ __forceinline__ void step_barrier()
{
    __builtin_amdgcn_s_waitcnt(0xc07f);                    // lgkmcnt(0), so that the compiler knows
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(N) : "memory");
}

// By how much the eight pieces of a row are turned.  A read of 16 bytes a lane goes through the banks by sixteen lanes, 0-3, 12-15, 20-23 and 24-27 first, which
// then have a place of their own among the 256 bytes of all banks.
__device__ __forceinline__ int turn(int row) { return row & 7; }

// BT tokens x BR channels by WT x WR waves, S stages.  YT = SUMS: workgroup z has the columns from z * part on, and its sums go to Y as they are, n rows of `ldy`
// (a multiple of 4).
constexpr int SUMS = -1;
template <int YT, int BT, int BR, int WT, int WR, int S>
__global__ __launch_bounds__(64 * WT * WR) void k_gemm_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, Finish f, void *Y,
                                                          int64_t ldy, unsigned tiles_r, unsigned tiles, int part_cols)
{
    constexpr int NW = WT * WR, LOADS = (BT + BR) / 8 / NW, TT = BT / WT / M, TR = BR / WR / M, STAGE = (BT + BR) * STEP, READS = TT + TR;
    static_assert((BT + BR) % (8 * NW) == 0, "whole loads");
    __shared__ __attribute__((aligned(1024))) int8_t lds[S * STAGE];
    const unsigned tile = blockIdx.y * gridDim.x + blockIdx.x;
    if (tile >= tiles) return;
    if constexpr (YT == SUMS) {
        const int first = blockIdx.z * part_cols;
        X += first;
        A += first;
        cols = min(cols - first, part_cols);
    }
    const int t0 = (int)(tile / tiles_r) * BT, r0 = (int)(tile % tiles_r) * BR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wave / WR, wr = wave % WR;
    const int blocks = (cols + STEP - 1) / STEP, left = cols - (blocks - 1) * STEP, most = ((left + 15) & ~15) - 16;      // the last piece of the last step

    // where a lane's 16 bytes come from: row 8 q + lane / 8 of the stage, piece lane % 8 turned by the row
    const int8_t *const x0 = X + (int64_t)t0 * ldx, *const a0 = A + (int64_t)r0 * lda;
    const int8_t *base[LOADS];
    unsigned from[LOADS], end[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int q = i * NW + wave, row = 8 * q + (lane >> 3), piece = 16 * ((lane & 7) ^ turn(row));
        const bool x = 8 * q < BT;
        base[i] = x ? x0 : a0;
        from[i] = x ? (unsigned)min(row, n - 1 - t0) * (unsigned)ldx : (unsigned)min(row - BT, rows - 1 - r0) * (unsigned)lda;
        end[i] = from[i] + (unsigned)min(piece, most);
        from[i] += (unsigned)piece;
    }
    // loads first .. last - 1 of a step
    auto fetch = [&](int step, int first, int last) {
        int8_t *const to = lds + step % S * STAGE + wave * 1024;
        const int64_t k = (int64_t)step * STEP;
        if (step < blocks - 1) {
#pragma unroll
            for (int i = first; i < last; ++i) to_lds(base[i] + k, from[i], to + i * NW * 1024);
        } else if (step == blocks - 1) {
#pragma unroll
            for (int i = first; i < last; ++i) to_lds(base[i] + k, end[i], to + i * NW * 1024);
        }
    };
    // Step k is there for all waves, and step k - 1 has been read by all.  Behind the last column the tokens' codes become zeros (once).
    auto arrive = [&](int k) {
        if (k + S - 2 < blocks - 1) step_barrier<(S - 2) * LOADS>();
        else step_barrier<0>();
        if (k == blocks - 1 && left < STEP) {
            int8_t *const st = lds + k % S * STAGE;
            for (int i = threadIdx.x; i < BT * 8; i += 64 * NW) {
                const int piece = 16 * ((i & 7) ^ turn(i >> 3));
                v4i *const at = reinterpret_cast<v4i *>(st + 16 * i);
                if (piece + 16 > left) *at = first_bytes(*at, left - piece);
            }
            step_barrier<0>();
        }
    };
    const int in = lane & (M - 1), part = lane / M;
    const int xrow = (wt * TT * M + in) * STEP, arow = (BT + wr * TR * M + in) * STEP;
    struct Operands { v4i x[TT], a[TR]; };                 // of half a step, 64 columns
    // reads first .. last - 1 of a half
    auto read = [&](Operands &o, int k, int half, int first, int last) {
        const int8_t *const st = lds + k % S * STAGE + 16 * ((4 * half + part) ^ turn(in));
#pragma unroll
        for (int i = first; i < last; ++i) {
            if (i < TT) o.x[i] = *reinterpret_cast<const v4i *>(st + xrow + i * M * STEP);
            else o.a[i - TT] = *reinterpret_cast<const v4i *>(st + arow + (i - TT) * M * STEP);
        }
    };
    v4i acc[TR][TT];
#pragma unroll
    for (int r = 0; r < TR; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = v4i{0, 0, 0, 0};
    // `beside` before the products of each row of instructions
    auto multiply = [&](const Operands &now, auto beside) {
#pragma unroll
        for (int r = 0; r < TR; ++r) {
            beside(r);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[r][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now.a[r], now.x[t], acc[r][t], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // The operands of a half are read while the half before is multiplied, across the barrier too, a share of them and of the loads before the products of each
    // row of instructions.  (All reads first: the instructions' unit waits for the LDS of eight waves, and a step of 256 x 256 takes 2750 cycles without its
    // loads, of 2048 for the products.)  The last step is written apart: where it is a branch of the loop, the compiler waits for the reads of the step
    // behind the barrier.
    for (int k = 0; k < S - 1; ++k) fetch(k, 0, LOADS);
    Operands o[2];
    if (blocks > 0) {
        arrive(0);
        fetch(S - 1, 0, LOADS);
        read(o[0], 0, 0, 0, READS);
    }
    for (int k = 0; k + 1 < blocks; ++k) {
        multiply(o[0], [&](int r) { read(o[1], k, 1, r * READS / TR, (r + 1) * READS / TR); });
        arrive(k + 1);
        multiply(o[1], [&](int r) {
            read(o[0], k + 1, 0, r * READS / TR, (r + 1) * READS / TR);
            fetch(k + S, r * LOADS / TR, (r + 1) * LOADS / TR);
        });
    }
    if (blocks > 0) {
        multiply(o[0], [&](int r) { read(o[1], blocks - 1, 1, r * READS / TR, (r + 1) * READS / TR); });
        multiply(o[1], [](int) {});
    }

    if constexpr (YT == SUMS) {
        v4i *const to = static_cast<v4i *>(Y) + blockIdx.z * (n * ldy >> 2);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int r = 0; r < TR; ++r) {
                const int token = t0 + (wt * TT + t) * M + in, row = r0 + (wr * TR + r) * M + 4 * part;
                if (token < n && row < rows) to[(token * ldy + row) >> 2] = acc[r][t];
            }
    } else {
        // A lane has four channels of a token, 4 (lane / 16) + 0 .. 3 of every 16.  They change places in LDS, 16 tokens of the wave at a time, and leave in
        // pieces of 16 bytes, a token's one after the other.  (Stored as they are, and with the tokens' scales loaded one by one, they took 22 us for a tile.)
        constexpr int ES = YT == F32 ? 4 : 2, EACH = 16 / ES, PIECES = TR * M / EACH, PITCH = PIECES * 16 + 16;
        static_assert(NW * M * PITCH <= S * STAGE, "room in LDS");
        const int row0 = r0 + wr * TR * M;
        float a[TR][4], b[TR][4], s[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t) s[t] = f.s[min(t0 + (wt * TT + t) * M + in, n - 1)];
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[r][i] = f.a[min(row0 + r * M + 4 * part + i, rows - 1)];
        if (f.bias) {
#pragma unroll
            for (int r = 0; r < TR; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) b[r][i] = f.bias[min(row0 + r * M + 4 * part + i, rows - 1)];
        } else {
#pragma unroll
            for (int r = 0; r < TR; ++r)
#pragma unroll
                for (int i = 0; i < 4; ++i) b[r][i] = 0.0f;
        }
        step_barrier<0>();                                     // the last step has been read
        int8_t *const room = lds + wave * M * PITCH;
#pragma unroll
        for (int t = 0; t < TT; ++t) {
#pragma unroll
            for (int r = 0; r < TR; ++r) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = finish(acc[r][t][i], a[r][i], s[t], b[r][i]);
                int8_t *const at = room + in * PITCH + (r * M + 4 * part) * ES;
                if constexpr (YT == F32) *reinterpret_cast<v4f *>(at) = v4f{v[0], v[1], v[2], v[3]};
                else *reinterpret_cast<v4s *>(at) = v4s{narrow<YT>(v[0]), narrow<YT>(v[1]), narrow<YT>(v[2]), narrow<YT>(v[3])};
            }
            wave_fence();
#pragma unroll
            for (int i = 0; i < M * PIECES; i += 64) {
                const int at = i + lane, token = t0 + (wt * TT + t) * M + at / PIECES, row = row0 + at % PIECES * EACH;
                if (M * PIECES % 64 && at >= M * PIECES) continue;
                const int8_t *const from = room + at / PIECES * PITCH + at % PIECES * 16;
                const v4u v = *reinterpret_cast<const v4u *>(from);
                if (token >= n || row >= rows) continue;
                char *const to = static_cast<char *>(Y) + (token * ldy + row) * ES;
                if (row + EACH <= rows) {
                    if constexpr (YT == F32) put_result(reinterpret_cast<v4f_e *>(to), __builtin_bit_cast(v4f, v), f.aside);
                    else put_result(reinterpret_cast<v4u_u *>(to), v, f.aside);
                } else {
                    for (int e = 0; row + e < rows; ++e) {
                        if constexpr (YT == F32) reinterpret_cast<float *>(to)[e] = reinterpret_cast<const float *>(from)[e];
                        else reinterpret_cast<unsigned short *>(to)[e] = reinterpret_cast<const unsigned short *>(from)[e];
                    }
                }
            }
            wave_fence();
        }
    }
}

// The sums of all parts of the columns, and what becomes of them; a thread takes four channels of a token.
template <int YT>
__global__ __launch_bounds__(256) void k_gemm_i8_join(int rows, int n, int parts, const v4i *__restrict__ sums, int64_t pitch, Finish f, void *Y, int64_t ldy)
{
    const int64_t quads = pitch >> 2, all = n * quads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int token = (int)(i / quads), row = (int)(i % quads) * 4;
        v4i sum = sums[i];
        for (int p = 1; p < parts; ++p) sum += sums[p * all + i];
        const float s = f.s[token];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (row + e < rows) store_as<YT>(Y, token * ldy + row + e, finish(sum[e], f.a[row + e], s, f.bias ? f.bias[row + e] : 0.0f));
    }
}

template <int YT, int BT, int BR, int WT, int WR, int S>
void tiles(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, int parts, int part_cols,
           hipStream_t s)
{
    const unsigned r = (unsigned)((rows + BR - 1) / BR), all = r * (unsigned)((n + BT - 1) / BT), x = all < 65536 ? all : 65536;
    PSK_LAUNCH((k_gemm_i8<YT, BT, BR, WT, WR, S>), dim3(x, (all + x - 1) / x, parts), dim3(64 * WT * WR), 0, s, rows, cols, n, A, lda, X, ldx, f, Y, ldy, r, all,
               part_cols);
}

template <int YT>
void launch_shape(int shape, int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, int parts,
                  int part_cols, hipStream_t s)
{
    if constexpr (YT != SUMS) {
        if (shape == SHAPE_COUNT - 1) return tiles<YT, 256, 256, 2, 4, 2>(rows, cols, n, A, lda, X, ldx, f, Y, ldy, parts, part_cols, s);
    }
    decltype(&tiles<YT, 16, 16, 1, 1, 8>) const go[SHAPE_COUNT - 1] = {
        tiles<YT, 16, 16, 1, 1, 8>, tiles<YT, 16, 32, 1, 2, 8>, tiles<YT, 32, 32, 2, 2, 6>, tiles<YT, 32, 64, 1, 4, 4>, tiles<YT, 64, 32, 4, 1, 4>,
        tiles<YT, 64, 64, 2, 2, 4>, tiles<YT, 128, 64, 4, 2, 4>, tiles<YT, 128, 128, 2, 4, 4>, tiles<YT, 256, 128, 4, 2, 3>};
    go[shape](rows, cols, n, A, lda, X, ldx, f, Y, ldy, parts, part_cols, s);
}

template <int YT>
hipError_t launch(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, void *sums, hipStream_t s)
{
    const Choice c = choose(rows, cols, n);
    if (c.parts == 1) {
        launch_shape<YT>(c.shape, rows, cols, n, A, lda, X, ldx, f, Y, ldy, 1, cols, s);
    } else {
        const int64_t pitch = pitch_of(rows), blocks = (n * pitch / 4 + 255) / 256;
        launch_shape<SUMS>(c.shape, rows, cols, n, A, lda, X, ldx, f, sums, pitch, c.parts, c.part_cols, s);
        PSK_LAUNCH((k_gemm_i8_join<YT>), dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, s, rows, n, c.parts, static_cast<const v4i *>(sums), pitch, f, Y,
                   ldy);
    }
    return take_launch_status();
}

}  // namespace

// Room for the sums of parts of the columns: that for n tokens is enough for fewer.
size_t gemm_i8_workspace_bytes(int rows, int cols, int n)
{
    const int64_t most = MOST_PARTS * (int64_t)n * pitch_of(rows) * 4;
    return cols <= STEP ? 0 : (size_t)(most < SUM_ROOM ? most : SUM_ROOM);
}

hipError_t launch_gemm_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const float *a, const int8_t *X, int64_t ldx, const float *xs, const float *bias,
                          int type, void *Y, int64_t ldy, void *sums, hipStream_t s)
{
    // (8192 tokens x 16384 channels in bf16: 426 to 431 us for 448 to 450)
    const Finish f = {a, xs, bias, (int64_t)n * rows * (type == F32 ? 4 : 2) >= ASIDE};
    const auto go = type == F32 ? launch<F32> : (type == F16 ? launch<F16> : launch<BF16>);
    return go(rows, cols, n, A, lda, X, ldx, f, Y, ldy, sums, s);
}

}  // namespace psk
