// The router of a mixture of experts: a gating matrix with top_k stored entries per row.
//
// Logits are sums in 64 bits (the machine multiplies in 64 bits as fast as in 32): which expert is chosen turns on the last
// bits where two logits are close, and then the order of a sum in 32 bits would decide.
//
// Two launches, bound by their latency and by the sums over lanes: one token, 64 experts, 2048 columns 2.8 + 3.9 us; 64 tokens, 160 experts, 4096 columns
// 9.2 + 6.5 us.
#include "psk_internal.h"
#include "psk_mfma.h"
#include "../../include/psk.h"

namespace psk {
namespace {

typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int THREADS = 256;

// Eight elements from column k on as 64-bit numbers, zeros from column `cols` on.
template <int T>
__device__ __forceinline__ void load_wide(const void *p, int64_t row, int k, int cols, double (&d)[8])
{
    if constexpr (T == F32) {
        const float *q = static_cast<const float *>(p) + row;
        if (k + 8 <= cols) {
            const v4f_e a = *reinterpret_cast<const v4f_e *>(q + k), b = *reinterpret_cast<const v4f_e *>(q + k + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { d[i] = a[i]; d[4 + i] = b[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = k + i < cols ? q[k + i] : 0.0f;
        }
    } else {
        const v4u v = load8(static_cast<const unsigned short *>(p) + row, k, cols);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = widen<T>((unsigned short)(v[i / 2] >> 16 * (i & 1)));
    }
}

// Sums over lanes; the exchanges are in registers (LDS takes a hundred cycles for each of twelve).
template <int CTRL>
__device__ __forceinline__ double dpp64(double v)
{
    const v2u u = __builtin_bit_cast(v2u, v);
    return __builtin_bit_cast(double, v2u{(unsigned)__builtin_amdgcn_update_dpp(0, (int)u[0], CTRL, 0xF, 0xF, true),
                                          (unsigned)__builtin_amdgcn_update_dpp(0, (int)u[1], CTRL, 0xF, 0xF, true)});
}
// Lanes l and l ^ 32 (l ^ 16): a of the lower ones and b of the upper ones are put together.
template <int D>
__device__ __forceinline__ void halves64(double a, double b, double &x, double &y)
{
    const v2u u = __builtin_bit_cast(v2u, a), v = __builtin_bit_cast(v2u, b);
    v2u p, q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (D == 32) {
            auto r = __builtin_amdgcn_permlane32_swap(u[i], v[i], false, false);
            p[i] = r[0];
            q[i] = r[1];
        } else {
            auto r = __builtin_amdgcn_permlane16_swap(u[i], v[i], false, false);
            p[i] = r[0];
            q[i] = r[1];
        }
    }
    x = __builtin_bit_cast(double, p);
    y = __builtin_bit_cast(double, q);
}
template <class OP>
__device__ __forceinline__ double row_all(double v, OP op)      // over 16 lanes
{
    v = op(v, dpp64<0xB1>(v));
    v = op(v, dpp64<0x4E>(v));
    v = op(v, dpp64<0x141>(v));
    return op(v, dpp64<0x140>(v));
}
template <class OP>
__device__ __forceinline__ double wave_all(double v, OP op)
{
    double x, y;
    v = row_all(v, op);
    halves64<16>(v, v, x, y);
    v = op(x, y);
    halves64<32>(v, v, x, y);
    return op(x, y);
}

// EB experts by TB tokens; the threads share the columns, eight at a time.  Four by eight, for one token four by one (2.8 us; as one of eight 4.5).
template <int XT, int WT, int EB, int TB>
__global__ __launch_bounds__(THREADS) void k_route_logits(int n, int dim, int experts, const void *X, int64_t ldx, const void *W, int64_t ldw,
                                                           double *logits)
{
    constexpr int N = EB * TB, M = N / 4;
    static_assert(N % 4 == 0, "a quarter of the sums to each row of lanes");
    __shared__ double part[THREADS / WAVE][N];
    const int e0 = blockIdx.x * EB, t0 = blockIdx.y * TB, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double acc[N] = {};
    for (int k = 8 * threadIdx.x; k < dim; k += 8 * THREADS) {
        double w[EB][8];
#pragma unroll
        for (int e = 0; e < EB; ++e) load_wide<WT>(W, min(e0 + e, experts - 1) * ldw, k, dim, w[e]);
#pragma unroll
        for (int t = 0; t < TB; ++t) {
            double x[8];
            load_wide<XT>(X, min(t0 + t, n - 1) * ldx, k, dim, x);
#pragma unroll
            for (int e = 0; e < EB; ++e)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[e * TB + t] = fma(w[e][i], x[i], acc[e * TB + t]);
        }
    }
    // lanes 0-15 sum up numbers 0 .. M-1, 16-31 M .. 2M-1, ...
    double two[N / 2], one[M];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        double x, y;
        halves64<32>(acc[i], acc[i + N / 2], x, y);
        two[i] = x + y;
    }
#pragma unroll
    for (int i = 0; i < M; ++i) {
        double x, y;
        halves64<16>(two[i], two[i + M], x, y);
        one[i] = row_all(x + y, [](double a, double b) { return a + b; });
    }
    if ((lane & 15) == 0) {
#pragma unroll
        for (int i = 0; i < M; ++i) part[wave][(lane >> 4) * M + i] = one[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < N; i += THREADS) {
        const int e = e0 + i / TB, t = t0 + i % TB;
        double v = 0;
        for (int w = 0; w < THREADS / WAVE; ++w) v += part[w][i];
        if (e < experts && t < n) logits[(int64_t)t * experts + e] = v;
    }
}

// A workgroup per token, a lane per expert.  An expert's place in the row is the number of those before it: it compares its key with all
// others (taking the best one top_k times, each time a search over the lanes, is 2.7 times as long with 64 experts).
template <int SCORE>
__global__ __launch_bounds__(PSK_MOE_MAX_EXPERTS) void k_route_rank(int experts, int top_k, int normalise, float factor, const double *__restrict__ logits,
                                                                     const float *__restrict__ bias, int *__restrict__ crd, float *__restrict__ vals)
{
    __shared__ __align__(16) unsigned long long keys[PSK_MOE_MAX_EXPERTS];
    __shared__ double gates[PSK_MOE_MAX_TOP_K], tops[PSK_MOE_MAX_EXPERTS / WAVE], sums[PSK_MOE_MAX_EXPERTS / WAVE];
    __shared__ int open[PSK_MOE_MAX_EXPERTS / WAVE];
    const int e = threadIdx.x, lane = e & 63, wave = e >> 6, waves = blockDim.x >> 6;
    const int64_t t = blockIdx.x;
    const bool real = e < experts;
    const double logit = real ? logits[t * experts + e] : -INFINITY;
    const float b = real && bias ? bias[e] : 0.0f;
    double p;
    if constexpr (SCORE == PSK_SCORE_SOFTMAX) {
        const auto larger = [](double x, double y) { return y > x || y != y ? y : x; };
        double top = wave_all(logit, larger);
        if (lane == 0) tops[wave] = top;
        __syncthreads();
        for (int w = 0; w < waves; ++w) top = larger(top, tops[w]);
        p = real ? exp(logit - top) : 0.0;
        double sum = wave_all(p, [](double x, double y) { return x + y; });
        if (lane == 0) sums[wave] = sum;
        __syncthreads();
        sum = 0;
        for (int w = 0; w < waves; ++w) sum += sums[w];
        p /= sum;
    } else {
        p = 1.0 / (1.0 + exp(-logit));
    }
    // numbers in their order as integers; 0: not to be chosen, 1: no number
    const double k = (bias ? p + (double)b : logit) + 0.0;   // -0 as 0
    const unsigned long long u = __builtin_bit_cast(unsigned long long, k);
    unsigned long long key = k != k ? 1 : (u >> 63 ? ~u : u | 1ull << 63);
    if (!real || b == -INFINITY) key = 0;
    keys[e] = key;
    const int mine = __popcll(__ballot(key != 0));
    if (lane == 0) open[wave] = mine;
    if (e < PSK_MOE_MAX_TOP_K) gates[e] = 0;
    __syncthreads();
    int rank = 0, taken = 0;
    typedef unsigned long long v2l __attribute__((ext_vector_type(2)));
#pragma unroll 8
    for (int j = 0; j < experts; j += 2) {                   // (keys past the last expert are 0)
        const v2l o = *reinterpret_cast<const v2l *>(keys + j);
        rank += (o[0] > key || (o[0] == key && j < e)) + (o[1] > key || (o[1] == key && j + 1 < e));
    }
    for (int w = 0; w < waves; ++w) taken += open[w];
    const bool chosen = key != 0 && rank < top_k;
    if (chosen) gates[rank] = p;
    if (normalise) {
        __syncthreads();
        double total = 0;
        for (int i = 0; i < top_k; ++i) total += gates[i];
        if (total != 0) p /= total;                          // (scores that all underflowed stay zeros)
    }
    if (chosen) {
        crd[t * top_k + rank] = e;
        vals[t * top_k + rank] = (float)(p * (double)factor);
    }
    if (e >= taken && e < top_k) {
        crd[t * top_k + e] = -1;
        vals[t * top_k + e] = 0;
    }
}

template <int XT, int WT>
void logits_of(int n, int dim, int experts, const void *X, int64_t ldx, const void *W, int64_t ldw, double *logits, hipStream_t s)
{
    if (n == 1) PSK_LAUNCH((k_route_logits<XT, WT, 4, 1>), dim3((experts + 3) / 4), dim3(THREADS), 0, s, n, dim, experts, X, ldx, W, ldw, logits);
    else PSK_LAUNCH((k_route_logits<XT, WT, 4, 8>), dim3((experts + 3) / 4, (n + 7) / 8), dim3(THREADS), 0, s, n, dim, experts, X, ldx, W, ldw, logits);
}

}  // namespace

hipError_t launch_moe_route(int n, int dim, int experts, int top_k, int score, int normalise, float factor, int type, const void *X, int64_t ldx,
                            int wtype, const void *W, int64_t ldw, const float *bias, int *crd, float *vals, double *logits, hipStream_t s)
{
    if (type == F32) logits_of<F32, F32>(n, dim, experts, X, ldx, W, ldw, logits, s);
    else if (type == F16 && wtype == F16) logits_of<F16, F16>(n, dim, experts, X, ldx, W, ldw, logits, s);
    else if (type == F16) logits_of<F16, F32>(n, dim, experts, X, ldx, W, ldw, logits, s);
    else if (wtype == BF16) logits_of<BF16, BF16>(n, dim, experts, X, ldx, W, ldw, logits, s);
    else logits_of<BF16, F32>(n, dim, experts, X, ldx, W, ldw, logits, s);
    const dim3 block((experts + WAVE - 1) / WAVE * WAVE);
    if (score == PSK_SCORE_SOFTMAX) PSK_LAUNCH(k_route_rank<PSK_SCORE_SOFTMAX>, dim3(n), block, 0, s, experts, top_k, normalise, factor, logits, bias, crd, vals);
    else PSK_LAUNCH(k_route_rank<PSK_SCORE_SIGMOID>, dim3(n), block, 0, s, experts, top_k, normalise, factor, logits, bias, crd, vals);
    return take_launch_status();
}

}  // namespace psk
