// Up to four tokens by a matrix of 8-bit integers (formulas: gemm_i8.h), quantising them on the way.  Bound by reading the matrix once.
//
// A wave reads four rows in pieces of 1 KB, four steps ahead, and multiplies them by the tokens' codes, which every workgroup makes for itself in LDS while
// its first weights are on their way; the products of a lane are four to an instruction, and the sums of 64 lanes meet in registers.  The workgroups stay.
// Few rows: the four waves of a workgroup share the columns of the same four rows (SPLIT).
// One bf16 token: 32768 x 8192 in 43 us, 6.2 TB/s; 4096 x 4096 in 6.6 a call, one after the other, and 7.3 in a trace
// (3.8 of these with 128 columns, and 6.8 with codes given).
#include "gemm_i8.h"

namespace psk {
namespace {

constexpr int PIECE = 1024;                                // columns of a step
constexpr int R = 4, DEPTH = 4, THREADS = 256;
constexpr int TOKENS = 3;                                  // XT: codes and scales

// LDS is written and read across waves; loads from memory go on.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <int CTRL>
__device__ __forceinline__ int dpp_add(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true); }
// Sums over the wave of four values: in quarter q of the lanes, that of value {0, 2, 1, 3}[q].
__device__ __forceinline__ int four_sums(int a, int b, int c, int d)
{
    auto ab = __builtin_amdgcn_permlane32_swap(a, b, false, false), cd = __builtin_amdgcn_permlane32_swap(c, d, false, false);
    auto all = __builtin_amdgcn_permlane16_swap(ab[0] + ab[1], cd[0] + cd[1], false, false);
    int v = (int)(all[0] + all[1]);
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    return dpp_add<0x140>(v);
}

template <int XT, int YT, int N, bool SPLIT>
__global__ __launch_bounds__(THREADS, 2) void k_gemv_i8(int rows, int cols, int n, const int8_t *__restrict__ A, int64_t lda, const void *__restrict__ X, int64_t ldx,
                                                        const float *__restrict__ a, const float *__restrict__ s, const float *__restrict__ bias, void *Y, int64_t ldy,
                                                        int tasks)
{
    constexpr int WAVES = THREADS / 64, KEPT = N == 4 ? 2 : 4;
    extern __shared__ __attribute__((aligned(16))) int8_t codes[];              // N rows of whole pieces, zeros behind the columns
    __shared__ unsigned most[N][WAVES];
    __shared__ int meet[WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pieces = (cols + PIECE - 1) / PIECE, pad = pieces * PIECE, last = ((cols + 15) & ~15) - 16;
    const int first = SPLIT ? blockIdx.x : blockIdx.x * WAVES + wave, stride = SPLIT ? gridDim.x : gridDim.x * WAVES;
    // this wave's steps: pieces begin, begin + by, ... of each of its tasks
    const int begin = SPLIT ? wave : 0, by = SPLIT ? WAVES : 1, each = begin < pieces ? (pieces - begin + by - 1) / by : 0;
    const int mine = first < tasks ? (tasks - first + stride - 1) / stride : 0, steps = mine * each;

    // the tokens are asked for first: waiting for them is not waiting for weights
    constexpr int T = XT == TOKENS ? F16 : XT;             // (not used with codes)
    const char *row[N];
    Raw8<T> raw[N][KEPT];
    if constexpr (XT != TOKENS) {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            row[t] = static_cast<const char *>(X) + min(t, n - 1) * ldx * (XT == F32 ? 4 : 2);
#pragma unroll
            for (int u = 0; u < KEPT; ++u) row_load<T>(raw[t][u], row[t], 8 * (u * THREADS + (int)threadIdx.x), cols);
        }
    }
    v4i w[DEPTH][R];
    int at_task = first, at_piece = begin;                 // of the next load
    auto load = [&](v4i (&to)[R]) {
        const int off = min(at_piece * PIECE + 16 * lane, last);
#pragma unroll
        for (int r = 0; r < R; ++r)
            to[r] = __builtin_nontemporal_load(reinterpret_cast<const v4i *>(A + (int64_t)min(at_task * R + r, rows - 1) * lda + off));
        at_piece += by;
        if (at_piece >= pieces) {                          // behind its last step a wave reads that again
            if (at_task + stride < tasks) {
                at_task += stride;
                at_piece = begin;
            } else {
                at_piece -= by;
            }
        }
    };
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) load(w[j]);            // (in bounds for a wave without steps too)
    float scale[N];
    if constexpr (XT == TOKENS) {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int8_t *x = static_cast<const int8_t *>(X) + min(t, n - 1) * ldx;
            for (int k = 16 * threadIdx.x; k < pad; k += 16 * THREADS) {
                v4i c = {0, 0, 0, 0};
                if (k <= last) c = first_bytes(*reinterpret_cast<const v4i *>(x + k), cols - k);
                *reinterpret_cast<v4i *>(codes + t * pad + k) = c;
            }
            scale[t] = s[min(t, n - 1)];
        }
    } else {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            unsigned m = 0;
            auto look = [&](const Raw8<T> &r, int k) {
                float x[8];
                row_get<T>(r, k, cols, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) m = max(m, size_bits(x[i]));
            };
#pragma unroll
            for (int u = 0; u < KEPT; ++u) look(raw[t][u], 8 * (u * THREADS + (int)threadIdx.x));
            for (int k = 8 * (KEPT * THREADS + (int)threadIdx.x); k < cols; k += 8 * THREADS) {
                Raw8<T> r;
                row_load<T>(r, row[t], k, cols);
                look(r, k);
            }
            m = wave_max(m);
            if (lane == 0) most[t][wave] = m;
        }
        lds_barrier();
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const Quantiser q(max(max(most[t][0], most[t][1]), max(most[t][2], most[t][3])));
            scale[t] = q.scale();
            auto put = [&](const Raw8<T> &r, int k) {
                float x[8];
                int c[8];
                row_get<T>(r, k, cols, x);
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i] = q.code(x[i]);
                *reinterpret_cast<uint2 *>(codes + t * pad + k) = make_uint2(pack4(c), pack4(c + 4));
            };
#pragma unroll
            for (int u = 0; u < KEPT; ++u) {
                const int k = 8 * (u * THREADS + (int)threadIdx.x);
                if (k < pad) put(raw[t][u], k);
            }
            for (int k = 8 * (KEPT * THREADS + (int)threadIdx.x); k < pad; k += 8 * THREADS) {
                Raw8<T> r;
                row_load<T>(r, row[t], k, cols);
                put(r, k);
            }
        }
    }
    lds_barrier();
    // The first weights are there by now.  Said here, it is not asked for in the loop again, where it would wait for the last ones.
    __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0)

    int sum[R][N];
    auto clear = [&]() {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < N; ++t) sum[r][t] = 0;
    };
    clear();
    int task = first, piece = begin;
    const int quarter = lane >> 4, token = lane & 15, which = (quarter >> 1) | (quarter & 1) << 1;
    auto finish_task = [&]() {
        int y = 0;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int of = four_sums(sum[0][t], sum[1][t], sum[2][t], sum[3][t]);
            y = token == t ? of : y;
        }
        if constexpr (SPLIT) {
            meet[wave][lane] = y;
            lds_barrier();
            y = meet[0][lane] + meet[1][lane] + meet[2][lane] + meet[3][lane];
            if (wave != 0) return;
        }
        float channel = 0.0f, add = 0.0f, of = scale[0];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int row = min(task * R + r, rows - 1);
            channel = which == r ? a[row] : channel;
            if (bias) add = which == r ? bias[row] : add;
        }
#pragma unroll
        for (int t = 1; t < N; ++t) of = token == t ? scale[t] : of;
        const int row = task * R + which;
        if (token < n && token < N && row < rows) store_as<YT>(Y, token * ldy + row, finish(y, channel, of, add));
    };
    if constexpr (SPLIT) {                                 // one task to a workgroup
        for (int i = 0; i < steps; i += DEPTH) {
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) {
                if (i + j >= steps) break;
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    const v4i x = *reinterpret_cast<const v4i *>(codes + t * pad + piece * PIECE + 16 * lane);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[r][t] = __builtin_amdgcn_sdot4(w[j][r][e], x[e], sum[r][t], false);
                }
                load(w[j]);
                piece += by;
            }
        }
        finish_task();
    } else {
        for (int i = 0; i < steps; i += DEPTH) {
#pragma unroll
            for (int j = 0; j < DEPTH; ++j) {
                if (i + j >= steps) break;
#pragma unroll
                for (int t = 0; t < N; ++t) {
                    const v4i x = *reinterpret_cast<const v4i *>(codes + t * pad + piece * PIECE + 16 * lane);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum[r][t] = __builtin_amdgcn_sdot4(w[j][r][e], x[e], sum[r][t], false);
                }
                load(w[j]);
                if (++piece == pieces) {
                    finish_task();
                    clear();
                    piece = 0;
                    task += stride;
                }
            }
        }
    }
}

template <int XT, int YT, int N>
hipError_t launch(int rows, int cols, int n, const int8_t *A, int64_t lda, const float *a, const void *X, int64_t ldx, const float *xs, const float *bias, void *Y,
                  int64_t ldy, hipStream_t s)
{
    const int tasks = (rows + R - 1) / R, pieces = (cols + PIECE - 1) / PIECE;
    const unsigned lds = (unsigned)(N * pieces * PIECE);
    // Few and long rows, one bf16 token, us against a task to a wave: 1024 x 8192 8.1 to 8.3 and 9.0, 256 x 8192 7.7 and 8.7 to 9.1, 1024 x 16384 11.9 and 15.0.
    // Of 4 and 6 pieces either is faster, by run (1024 x 4096 7.3 to 7.4 and 6.4 to 8.1; four tokens 10.7 to 11.0 and 11.2); 2040 x 8192 10.2 and 9.6.
    if (tasks <= 256 && pieces >= 8)
        PSK_LAUNCH((k_gemv_i8<XT, YT, N, true>), dim3(tasks), dim3(THREADS), lds, s, rows, cols, n, A, lda, X, ldx, a, xs, bias, Y, ldy, tasks);
    else
        PSK_LAUNCH((k_gemv_i8<XT, YT, N, false>), dim3(tasks / 4 < 512 ? (tasks + 3) / 4 : 512), dim3(THREADS), lds, s, rows, cols, n, A, lda, X, ldx, a, xs, bias, Y,
                   ldy, tasks);
    return take_launch_status();
}
template <int XT, int YT>
hipError_t launch_n(int rows, int cols, int n, const int8_t *A, int64_t lda, const float *a, const void *X, int64_t ldx, const float *xs, const float *bias, void *Y,
                    int64_t ldy, hipStream_t s)
{
    const auto go = n == 1 ? launch<XT, YT, 1> : (n == 2 ? launch<XT, YT, 2> : launch<XT, YT, 4>);
    return go(rows, cols, n, A, lda, a, X, ldx, xs, bias, Y, ldy, s);
}

}  // namespace

// Up to four tokens, whether or not codes are given.  us in a replayed graph, here and by tiles (with activations behind a launch that quantises them):
//   rows x cols       one token, bf16   two           four          four, codes given
//   256 x 1024        4.1    6.2        5.4    6.3    7.0    6.3    3.9    3.6
//   1024 x 8192       7.0   14.2       10.0   14.7   17.7   15.5    6.5   11.0
//   2048 x 2048       5.1    8.3        6.4    8.5    8.2    8.5    5.0    5.8
//   4096 x 4096       7.1   16.6        8.7   12.2   11.8   12.2    7.6    8.8
//   10240 x 4096     11.1   16.2       12.3   16.2   16.2   16.2   12.6   12.7
//   4096 x 16384     22.9   32.5       28.6   32.4   32.9   32.9   24.4   24.3
//   8192 x 8192      14.9   28.6       17.5   28.9   27.0   26.4   17.1   21.8
//   32768 x 8192     43.7   63.7       46.0   64.1   56.2   63.8   46.7   59.0
// Three tokens take what four do, f32 activations what bf16 do.  Three and four of activations and few rows are slower here (by a seventh at most): every
// workgroup makes all codes.
bool gemv_i8_takes(int cols, int n)
{
    return cols >= 8 && n <= 4 && (n == 3 ? 4 : n) * ((cols + PIECE - 1) / PIECE * PIECE) <= 65536 - 2048;      // two workgroups to a compute unit
}

// xs NULL: X is of `type` and is quantised; otherwise codes with these scales.
hipError_t launch_gemv_i8(int rows, int cols, int n, const int8_t *A, int64_t lda, const float *a, const void *X, int64_t ldx, const float *xs, const float *bias,
                          int type, void *Y, int64_t ldy, hipStream_t s)
{
    const auto go = xs ? (type == F32 ? launch_n<TOKENS, F32> : (type == F16 ? launch_n<TOKENS, F16> : launch_n<TOKENS, BF16>))
                       : (type == F32 ? launch_n<F32, F32> : (type == F16 ? launch_n<F16, F16> : launch_n<BF16, BF16>));
    return go(rows, cols, n, A, lda, a, X, ldx, xs, bias, Y, ldy, s);
}

}  // namespace psk
