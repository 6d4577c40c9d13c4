// Y = X A^T in 8-bit integers (formulas: gemm_i8.h).
//
// Tiles of tokens x channels, 128 columns a step.  Both operands go from memory to LDS without passing registers, a step or more ahead of its use; a wave's
// load is 8 rows of 128 bytes, and which 16 bytes of its row a lane asks for is turned by the row, so that reading the operands' order (16 rows x 16
// bytes, row by row) meets each bank once.  One barrier a step: behind it the step's operands are there and the stage before is free.
#include "gemm_i8.h"

namespace psk {
namespace {

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

typedef int v16i __attribute__((ext_vector_type(16)));

// One matrix instruction: M channels x M tokens over 1024 / M columns, 16 bytes of a row to a lane.
template <int M> struct Product;
template <> struct Product<16> {
    typedef v4i Sum;
    static __device__ __forceinline__ Sum go(v4i a, v4i x, Sum c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, x, c, 0, 0, 0); }
};
template <> struct Product<32> {
    typedef v16i Sum;
    static __device__ __forceinline__ Sum go(v4i a, v4i x, Sum c) { return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, x, c, 0, 0, 0); }
};

// By how much the pieces of a row of STEP bytes are turned.  A read of 16 bytes a lane goes through the banks by sixteen lanes, 0-3, 12-15, 20-23 and 24-27
// first, which then have a place of their own among the 256 bytes of all banks.
template <int M, int STEP>
__device__ __forceinline__ int turn(int row)
{
    if constexpr (STEP == 64) return -(row >> 2) & 3;
    else return M == 32 ? (row & 7) ^ (row >> 4 & 1) : row & 7;
}

// BT tokens x BR channels by WT x WR waves, S stages of STEP columns, instructions of M x M.
template <int YT, int BT, int BR, int WT, int WR, int S, int M, int STEP>
__global__ __launch_bounds__(64 * WT * WR) void k_gemm_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, Finish f, void *Y,
                                                          int64_t ldy, unsigned tiles_r, unsigned tiles)
{
    constexpr int NW = WT * WR, LINES = 1024 / STEP, PER = STEP / 16, LOADS = (BT + BR) / LINES / NW, TT = BT / WT / M, TR = BR / WR / M, STAGE = (BT + BR) * STEP, PARTS = STEP * M / 1024;
    static_assert((BT + BR) % (LINES * NW) == 0 && BT % LINES == 0, "whole loads");
    typedef typename Product<M>::Sum Sum;
    __shared__ __attribute__((aligned(1024))) int8_t lds[S * STAGE];
    const unsigned tile = blockIdx.y * gridDim.x + blockIdx.x;
    if (tile >= tiles) return;
    const int t0 = (int)(tile / tiles_r) * BT, r0 = (int)(tile % tiles_r) * BR;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wt = wave / WR, wr = wave % WR;
    const int blocks = (cols + STEP - 1) / STEP, left = cols - (blocks - 1) * STEP, most = ((left + 15) & ~15) - 16;      // the last piece of the last step

    // where a lane's 16 bytes come from: row LINES q + lane / PER of the stage, piece lane % PER turned by the row
    const int8_t *const x0 = X + (int64_t)t0 * ldx, *const a0 = A + (int64_t)r0 * lda;
    const int8_t *base[LOADS];
    unsigned from[LOADS], end[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int q = i * NW + wave, row = LINES * q + lane / PER, piece = 16 * ((lane % PER) ^ turn<M, STEP>(row));
        const bool x = LINES * q < BT;
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
    // Step k is there for all waves, and step k - 1 has been read by all.  Behind the last column the tokens' codes become zeros (once).
    auto arrive = [&](int k) {
        if (k + S - 2 < blocks - 1) step_barrier<(S - 2) * LOADS>();
        else step_barrier<0>();
        if (k + S - 1 < blocks) fetch(k + S - 1);
        if (left < STEP && k == blocks - 1) {
            int8_t *const st = lds + k % S * STAGE;
            for (int i = threadIdx.x; i < BT * PER; i += 64 * NW) {
                const int piece = 16 * ((i % PER) ^ turn<M, STEP>(i / PER));
                v4i *const at = reinterpret_cast<v4i *>(st + 16 * i);
                if (piece + 16 > left) *at = first_bytes(*at, left - piece);
            }
            step_barrier<0>();
        }
    };
    const int in = lane & (M - 1), part = lane / M;
    const int xrow = (wt * TT * M + in) * STEP, arow = (BT + wr * TR * M + in) * STEP;
    struct Operands { v4i x[TT], a[TR]; };
    auto read = [&](Operands &o, int k, int h) {
        const int8_t *const st = lds + k % S * STAGE + 16 * ((64 / M * h + part) ^ turn<M, STEP>(in));
#pragma unroll
        for (int t = 0; t < TT; ++t) o.x[t] = *reinterpret_cast<const v4i *>(st + xrow + t * M * STEP);
#pragma unroll
        for (int r = 0; r < TR; ++r) o.a[r] = *reinterpret_cast<const v4i *>(st + arow + r * M * STEP);
    };
    Sum acc[TR][TT];
#pragma unroll
    for (int r = 0; r < TR; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[r][t] = Sum{};
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[r][t] = Product<M>::go(o.a[r], o.x[t], acc[r][t]);
    };

    // The operands of a part are read while the part before is multiplied, across the barrier too.
    for (int k = 0; k < S - 1 && k < blocks; ++k) fetch(k);
    Operands o[2];
    if (blocks > 0) {
        arrive(0);
        read(o[0], 0, 0);
    }
    constexpr int ROUND = PARTS == 1 ? 2 : 1;              // steps behind which the operands are in the same registers again
    for (int k0 = 0; k0 < blocks; k0 += ROUND) {
#pragma unroll
        for (int j = 0; j < ROUND; ++j) {
            const int k = k0 + j;
            if (j > 0 && k >= blocks) break;
#pragma unroll
            for (int h = 0; h < PARTS; ++h) {
                const int now = (j * PARTS + h) & 1;
                if (h + 1 < PARTS) {
                    read(o[now ^ 1], k, h + 1);
                } else if (k + 1 < blocks) {
                    arrive(k + 1);
                    read(o[now ^ 1], k + 1, 0);
                }
                multiply(o[now]);
            }
        }
    }
    // A lane has four channels of a token, 4 (lane / M) + 0 .. 3 of every 256 / M.  They change places in LDS, M tokens of the wave at a time, and leave in
    // pieces of 16 bytes, a token's one after the other.  (Stored as they are, and with the tokens' scales loaded one by one, they took 22 us for a tile.)
    constexpr int G = M * M / 256, ES = YT == F32 ? 4 : 2, EACH = 16 / ES, PIECES = TR * M / EACH, PITCH = PIECES * 16 + 16;
    static_assert(NW * M * PITCH <= S * STAGE, "room in LDS");
    const int row0 = r0 + wr * TR * M;
    float a[TR][G][4], b[TR][G][4], s[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) s[t] = f.s[min(t0 + (wt * TT + t) * M + in, n - 1)];
#pragma unroll
    for (int r = 0; r < TR; ++r)
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[r][g][i] = f.a[min(row0 + r * M + 256 / M * g + 4 * part + i, rows - 1)];
    if (f.bias) {
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) b[r][g][i] = f.bias[min(row0 + r * M + 256 / M * g + 4 * part + i, rows - 1)];
    } else {
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < 4; ++i) b[r][g][i] = 0.0f;
    }
    step_barrier<0>();                                     // the last step has been read
    int8_t *const room = lds + wave * M * PITCH;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
#pragma unroll
        for (int r = 0; r < TR; ++r)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = finish(acc[r][t][4 * g + i], a[r][g][i], s[t], b[r][g][i]);
                int8_t *const at = room + in * PITCH + (r * M + 256 / M * g + 4 * part) * ES;
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
                if constexpr (YT == F32) *reinterpret_cast<v4f_e *>(to) = __builtin_bit_cast(v4f, v);
                else *reinterpret_cast<v4u_u *>(to) = v;
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

template <int YT, int BT, int BR, int WT, int WR, int S, int M, int STEP>
void tiles(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, hipStream_t s)
{
    const unsigned r = (unsigned)((rows + BR - 1) / BR), all = r * (unsigned)((n + BT - 1) / BT), x = all < 65536 ? all : 65536;
    PSK_LAUNCH((k_gemm_i8<YT, BT, BR, WT, WR, S, M, STEP>), dim3(x, (all + x - 1) / x), dim3(64 * WT * WR), 0, s, rows, cols, n, A, lda, X, ldx, f, Y, ldy, r, all);
}

// Tiles by their tokens and channels.
struct Shape { int tokens, channels; };
constexpr Shape SHAPES[] = {{16, 16}, {16, 32}, {32, 32}, {32, 64}, {64, 32}, {64, 64}, {128, 64}, {128, 128}, {256, 128}, {256, 256}};
constexpr int SHAPE_COUNT = sizeof(SHAPES) / sizeof(SHAPES[0]);

template <int YT>
hipError_t launch(int rows, int cols, int n, const int8_t *A, int64_t lda, const int8_t *X, int64_t ldx, const Finish &f, void *Y, int64_t ldy, hipStream_t s)
{
    decltype(&tiles<YT, 16, 16, 1, 1, 8, 16, 128>) const go[SHAPE_COUNT] = {
        tiles<YT, 16, 16, 1, 1, 8, 16, 128>, tiles<YT, 16, 32, 1, 2, 8, 16, 128>, tiles<YT, 32, 32, 2, 2, 6, 16, 128>, tiles<YT, 32, 64, 1, 4, 4, 16, 128>,
        tiles<YT, 64, 32, 4, 1, 4, 16, 128>, tiles<YT, 64, 64, 2, 2, 4, 16, 128>, tiles<YT, 128, 64, 2, 2, 3, 16, 128>, tiles<YT, 128, 128, 2, 2, 4, 16, 128>,
        tiles<YT, 256, 128, 4, 2, 3, 16, 128>, tiles<YT, 256, 256, 2, 4, 2, 16, 128>};
    int best = 0;
    int64_t least = INT64_MAX;
    for (int i = 0; i < SHAPE_COUNT; ++i) {
        const int64_t all = (int64_t)((n + SHAPES[i].tokens - 1) / SHAPES[i].tokens) * ((rows + SHAPES[i].channels - 1) / SHAPES[i].channels);
        const int64_t cost = (all + 255) / 256 * (SHAPES[i].tokens + SHAPES[i].channels);
        if (cost <= least) {
            least = cost;
            best = i;
        }
    }
#ifdef TILE_ENV
    if (getenv("PSK_TILE")) best = atoi(getenv("PSK_TILE"));
#endif
    go[best](rows, cols, n, A, lda, X, ldx, f, Y, ldy, s);
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
