// The router of a mixture of experts: a gating matrix with top_k stored entries per row.
//
// Logits are sums in 64 bits (the machine multiplies in 64 bits as fast as in 32): which expert is chosen turns on the last
// bits where two logits are close, and then the order of a sum in 32 bits would decide.
#include "psk_internal.h"
#include "psk_mfma.h"
#include "../../include/psk.h"

namespace psk {
namespace {

constexpr int ROUTE_TOKENS = 8;      // tokens of a workgroup
constexpr int ROUTE_WAVES = 4;

template <int T>
__device__ __forceinline__ double element(const void *p, int64_t i)
{
    if constexpr (T == F32) return (double)static_cast<const float *>(p)[i];
    else return (double)widen<T>(static_cast<const unsigned short *>(p)[i]);
}
__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, WAVE);
    return v;
}

// One expert, up to ROUTE_TOKENS tokens; the waves share the columns.
template <int XT, int WT>
__global__ __launch_bounds__(64 * ROUTE_WAVES) void k_route_logits(int n, int dim, int experts, const void *X, int64_t ldx, const void *W, int64_t ldw,
                                                                    double *logits)
{
    __shared__ double part[ROUTE_WAVES][ROUTE_TOKENS];
    const int e = blockIdx.x % experts, t0 = blockIdx.x / experts * ROUTE_TOKENS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int nt = min(ROUTE_TOKENS, n - t0);
    double acc[ROUTE_TOKENS] = {};
    for (int j = threadIdx.x; j < dim; j += 64 * ROUTE_WAVES) {
        const double w = element<WT>(W, e * ldw + j);
#pragma unroll
        for (int t = 0; t < ROUTE_TOKENS; ++t)
            if (t < nt) acc[t] = fma(w, element<XT>(X, (t0 + t) * ldx + j), acc[t]);
    }
#pragma unroll
    for (int t = 0; t < ROUTE_TOKENS; ++t) {
        const double v = wave_sum64(acc[t]);
        if (lane == 0) part[wave][t] = v;
    }
    __syncthreads();
    if ((int)threadIdx.x < nt) {
        double v = 0;
        for (int w = 0; w < ROUTE_WAVES; ++w) v += part[w][threadIdx.x];
        logits[(int64_t)(t0 + threadIdx.x) * experts + e] = v;
    }
}

// a before b in the order of choice: larger key, then lower index; a key that is no number comes after all others.
__device__ __forceinline__ bool before(double ka, int ia, double kb, int ib)
{
    const bool na = ka != ka, nb = kb != kb;
    if (na != nb) return nb;
    if (!na && ka != kb) return ka > kb;
    return ia < ib;
}

// A wave per token; lane l has experts l, l + 64, ..., PER of them.
template <int SCORE, int PER>
__global__ __launch_bounds__(64) void k_route_choose(int experts, int top_k, int normalise, float factor, const double *logits, const float *bias,
                                                      int *crd, float *vals)
{
    constexpr int NONE = 0x7fffffff;
    const int lane = threadIdx.x;
    const int64_t t = blockIdx.x;
    const double *row = logits + t * experts;
    double key[PER], p[PER];
    unsigned open = 0;                                       // experts of this lane that may be chosen
    double top = -INFINITY, sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + WAVE * i;
        key[i] = p[i] = 0;
        if (e < experts) {
            p[i] = row[e];
            if (!bias || !(bias[e] == -INFINITY)) open |= 1u << i;
            top = p[i] != p[i] ? p[i] : (p[i] > top ? p[i] : top);
        }
    }
    if constexpr (SCORE == PSK_SCORE_SOFTMAX) {
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const double o = __shfl_xor(top, d, WAVE);
            top = o > top || o != o ? o : top;
        }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = lane + WAVE * i;
        if (e >= experts) continue;
        key[i] = p[i];
        p[i] = SCORE == PSK_SCORE_SOFTMAX ? exp(p[i] - top) : 1.0 / (1.0 + exp(-p[i]));
        sum += p[i];
    }
    if constexpr (SCORE == PSK_SCORE_SOFTMAX) {
        sum = wave_sum64(sum);
#pragma unroll
        for (int i = 0; i < PER; ++i) p[i] /= sum;
    }
    if (bias) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (lane + WAVE * i < experts) key[i] = p[i] + (double)bias[lane + WAVE * i];
    }
    double gate = 0, total = 0;                              // lane s keeps entry s
    int mine = -1;
    for (int s = 0; s < top_k; ++s) {
        double bk = 0, bp = 0;
        int bi = NONE;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int e = lane + WAVE * i;
            if ((open >> i & 1) && (bi == NONE || before(key[i], e, bk, bi))) { bk = key[i]; bp = p[i]; bi = e; }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const double ok = __shfl_xor(bk, d, WAVE), op = __shfl_xor(bp, d, WAVE);
            const int oi = __shfl_xor(bi, d, WAVE);
            if (oi != NONE && (bi == NONE || before(ok, oi, bk, bi))) { bk = ok; bp = op; bi = oi; }
        }
        if (bi == NONE) break;
        if (bi % WAVE == lane) open &= ~(1u << (bi / WAVE));
        if (lane == s) { mine = bi; gate = bp; }
        total += bp;
    }
    if (lane < top_k) {
        crd[t * top_k + lane] = mine;
        vals[t * top_k + lane] = mine < 0 ? 0.0f : (float)((normalise ? gate / total : gate) * (double)factor);
    }
}

template <int SCORE>
void choose(int n, int experts, int top_k, int normalise, float factor, const double *logits, const float *bias, int *crd, float *vals, hipStream_t s)
{
#define PSK_CHOOSE(PER) PSK_LAUNCH((k_route_choose<SCORE, PER>), dim3(n), dim3(64), 0, s, experts, top_k, normalise, factor, logits, bias, crd, vals)
    if (experts <= 64) PSK_CHOOSE(1);
    else if (experts <= 128) PSK_CHOOSE(2);
    else if (experts <= 256) PSK_CHOOSE(4);
    else PSK_CHOOSE(PSK_MOE_MAX_EXPERTS / WAVE);
#undef PSK_CHOOSE
}

template <int XT, int WT>
void logits_of(int n, int dim, int experts, const void *X, int64_t ldx, const void *W, int64_t ldw, double *logits, hipStream_t s)
{
    PSK_LAUNCH((k_route_logits<XT, WT>), dim3((n + ROUTE_TOKENS - 1) / ROUTE_TOKENS * experts), dim3(64 * ROUTE_WAVES), 0, s, n, dim, experts, X, ldx,
               W, ldw, logits);
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
    if (score == PSK_SCORE_SOFTMAX) choose<PSK_SCORE_SOFTMAX>(n, experts, top_k, normalise, factor, logits, bias, crd, vals, s);
    else choose<PSK_SCORE_SIGMOID>(n, experts, top_k, normalise, factor, logits, bias, crd, vals, s);
    return take_launch_status();
}

}  // namespace psk
