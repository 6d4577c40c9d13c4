// The layer of a mixture of experts for a few tokens:
//
//   Y(t,:) = sum over stored (t,e) of G(t,e) * W2_e ( act(W1_e x_t) * (W3_e x_t) )
//
// G is a sparse matrix with top_k entries per row (crd, vals); position p = t * top_k + slot.  Bound by reading the matrices of
// the experts that occur, each once, so the unit of work is (expert that occurs, 16 rows of its matrices) with all positions of
// that expert: they are the vectors of one set of matrix instructions.  Two launches:
//   k_moe_up    h[p] = act(W1_e x_t) * (W3_e x_t)
//   k_moe_down  P[p] = W2_e h[p]; the workgroup that is the last of its 16 rows adds up Y from P, in the order of the slots
// Every workgroup finds its expert and that one's positions itself from crd (at most kMoePositions of them).
//
// h goes to memory as two 16-bit numbers, the nearest one and the nearest one to what is left: rounding to one of them would cost as
// much accuracy as rounding Y does, and the second one costs a matrix instruction where the matrix cores wait for memory.
// f16 has too small a range for that: there h is scaled by 2^-8 (|h| up to 2^24 is finite) and what is left by 2^11.
#include "psk_internal.h"
#include "psk_mfma.h"
#include "../../include/psk.h"

namespace psk {
namespace {

constexpr int KW = 4;                                        // waves of a workgroup, which share the columns
constexpr int THREADS = 64 * KW;

// ---- which expert, which positions
struct Found {
    int expert, count, active;                               // active: experts that occur
};
struct FindSpace {
    int seen[PSK_MOE_MAX_EXPERTS];
    int count;
    unsigned short list[kMoePositions];
};
// The j-th expert that occurs (in the order of the experts) and its positions in `list`.  expert -1: fewer occur.
__device__ __forceinline__ Found find(FindSpace &f, int positions, int experts, const int *__restrict__ crd, int j)
{
    for (int e = threadIdx.x; e < experts; e += THREADS) f.seen[e] = 0;
    if (threadIdx.x == 0) f.count = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < positions; p += THREADS) {
        const int e = crd[p];
        if ((unsigned)e < (unsigned)experts) f.seen[e] = 1;
    }
    __syncthreads();
    Found r = {-1, 0, 0};
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < experts; e0 += WAVE) {
        unsigned long long b = __ballot(e0 + lane < experts && f.seen[min(e0 + lane, experts - 1)] != 0);
        const int c = __popcll(b);
        if (r.expert < 0 && j < r.active + c) {
            for (int skip = j - r.active; skip; --skip) b &= b - 1;
            r.expert = e0 + __ffsll(b) - 1;
        }
        r.active += c;
    }
    if (r.expert >= 0) {
        for (int p = threadIdx.x; p < positions; p += THREADS)
            if (crd[p] == r.expert) f.list[atomicAdd(&f.count, 1)] = (unsigned short)p;
    }
    __syncthreads();
    r.count = f.count;
    return r;
}

// ---- h
template <int T> struct Half2 {                              // f16
    static constexpr float scale = 0x1p-8f, rest = 0x1p11f;
};
template <> struct Half2<BF16> {
    static constexpr float scale = 1.0f, rest = 1.0f;
};
template <int T>
__device__ __forceinline__ void split(float h, unsigned short &a, unsigned short &b)
{
    const float v = h * Half2<T>::scale;
    a = narrow<T>(v);
    const float w = widen<T>(a), r = (v - w) * Half2<T>::rest;
    b = __builtin_isfinite(w) ? narrow<T>(r) : (unsigned short)0;
}

template <int ACT>
__device__ __forceinline__ float activate(float v)
{
    if constexpr (ACT == PSK_ACT_SILU) return v / (1.0f + expf(-v));
    else return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
}

struct UpArgs {
    int n, experts, top_k, dim, inter, counters;
    const int *crd;
    const unsigned short *X;
    int64_t ldx;
    unsigned short *h, *rest;
    int64_t ldh;
    int *done;
};
struct DownArgs {
    int n, experts, top_k, dim, inter;
    const int *crd;
    const float *vals;
    const unsigned short *h, *rest;
    int64_t ldh;
    float *P;
    int *done;
    void *Y;
    int64_t ldy;
};

// NT tiles of 16 positions, 16 rows of W1 and of W3.  HT: type of the parts of h.
template <class SPAN, int HT, int ACT, int NT, class W>
__device__ __forceinline__ void up_tiles(const UpArgs &a, const W &w1, const W &w3, int expert, const unsigned short *list, int count, int row0, float *lds)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    SPAN span;
    span.set(0, w1, expert, min(row0 + m, a.inter - 1), quarter);
    span.set(1, w3, expert, min(row0 + m, a.inter - 1), quarter);
    Rows16<NT> x;
    x.cols = a.dim;
    v4f acc[2][NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        x.p[t] = a.X + (int64_t)(list[min(16 * t + m, count - 1)] / a.top_k) * a.ldx;
        acc[0][t] = acc[1][t] = v4f{0, 0, 0, 0};
    }
    span_product<SPAN, NT>(span, x, a.dim, wave, KW, quarter, acc);
    v4f flat[2 * NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) { flat[t] = acc[0][t]; flat[NT + t] = acc[1][t]; }
    put_sums<2 * NT>(lds, wave, lane, flat);
    __syncthreads();
    for (int o = threadIdx.x; o < NT * 256; o += THREADS) {
        const int t = o >> 8, v = o >> 4 & 15, i = o & 15;
        if (16 * t + v >= count || row0 + i >= a.inter) continue;
        const float h = activate<ACT>(get_sum<KW, 2 * NT>(lds, t, v, i)) * get_sum<KW, 2 * NT>(lds, NT + t, v, i);
        unsigned short p, q;
        split<HT>(h, p, q);
        const int64_t at = list[16 * t + v] * a.ldh + row0 + i;
        a.h[at] = p;
        a.rest[at] = q;
    }
}

template <class SPAN, int HT, int ACT, class W>
__global__ __launch_bounds__(THREADS) void k_moe_up(UpArgs a, W w1, W w3)
{
    __shared__ FindSpace f;
    __shared__ float lds[KW * 8 * 256];
    if (blockIdx.x == 0 && blockIdx.y == 0)
        for (int i = threadIdx.x; i < a.counters; i += THREADS) a.done[i] = 0;
    const Found g = find(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0) return;
    const int row0 = blockIdx.x * 16;
    for (int p0 = 0; p0 < g.count; p0 += 64) {
        const int c = g.count - p0;
        if (c <= 16) up_tiles<SPAN, HT, ACT, 1>(a, w1, w3, g.expert, f.list + p0, c, row0, lds);
        else if (c <= 32) up_tiles<SPAN, HT, ACT, 2>(a, w1, w3, g.expert, f.list + p0, c, row0, lds);
        else up_tiles<SPAN, HT, ACT, 4>(a, w1, w3, g.expert, f.list + p0, c, row0, lds);
        __syncthreads();
    }
}

// NT tiles of 16 positions, 16 rows of W2; both parts of h are vectors.
template <class SPAN, int NT, class W>
__device__ __forceinline__ void down_tiles(const DownArgs &a, const W &w2, int expert, const unsigned short *list, int count, int row0, float *lds)
{
    constexpr int T = SPAN::T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    SPAN span;
    span.set(0, w2, expert, min(row0 + m, a.dim - 1), quarter);
    Rows16<2 * NT> x;
    x.cols = a.inter;
    v4f acc[1][2 * NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t at = list[min(16 * t + m, count - 1)] * a.ldh;
        x.p[t] = a.h + at;
        x.p[NT + t] = a.rest + at;
        acc[0][t] = acc[0][NT + t] = v4f{0, 0, 0, 0};
    }
    span_product<SPAN, 2 * NT>(span, x, a.inter, wave, KW, quarter, acc);
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[0][t][i] = fmaf(acc[0][NT + t][i], 1.0f / Half2<T>::rest, acc[0][t][i]) * (1.0f / Half2<T>::scale);
    v4f flat[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) flat[t] = acc[0][t];
    put_sums<NT>(lds, wave, lane, flat);
    __syncthreads();
    for (int o = threadIdx.x; o < NT * 256; o += THREADS) {
        const int t = o >> 8, v = o >> 4 & 15, i = o & 15;
        if (16 * t + v >= count || row0 + i >= a.dim) continue;
        // read by a workgroup that may run on another die: past this die's L2
        __hip_atomic_store(a.P + (int64_t)list[16 * t + v] * a.dim + row0 + i, get_sum<KW, NT>(lds, t, v, i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

template <class SPAN, int YT, class W>
__global__ __launch_bounds__(THREADS) void k_moe_down(DownArgs a, W w2)
{
    __shared__ FindSpace f;
    __shared__ float lds[KW * 4 * 256];
    __shared__ int last;
    const Found g = find(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0 && !(g.active == 0 && blockIdx.y == 0)) return;
    const int row0 = blockIdx.x * 16;
    for (int p0 = 0; p0 < g.count; p0 += 64) {
        const int c = g.count - p0;
        if (c <= 16) down_tiles<SPAN, 1>(a, w2, g.expert, f.list + p0, c, row0, lds);
        else if (c <= 32) down_tiles<SPAN, 2>(a, w2, g.expert, f.list + p0, c, row0, lds);
        else down_tiles<SPAN, 4>(a, w2, g.expert, f.list + p0, c, row0, lds);
        __syncthreads();
    }
    if (threadIdx.x == 0)
        last = g.active == 0 || __hip_atomic_fetch_add(a.done + blockIdx.x, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == g.active - 1;
    __syncthreads();
    if (!last) return;
    for (int o = threadIdx.x; o < a.n * 16; o += THREADS) {
        const int t = o >> 4, i = o & 15;
        if (row0 + i >= a.dim) continue;
        float y = 0;
        for (int s = 0; s < a.top_k; ++s) {
            const int p = t * a.top_k + s;
            if ((unsigned)a.crd[p] >= (unsigned)a.experts) continue;
            y = fmaf(a.vals[p], __hip_atomic_load(a.P + (int64_t)p * a.dim + row0 + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), y);
        }
        store_as<YT>(a.Y, t * a.ldy + row0 + i, y);
    }
}

struct Space {
    unsigned short *h, *rest;
    float *P;
    int *done;
    int64_t ldh;
    size_t bytes;
};
Space carve_moe(void *base, int64_t positions, int64_t dim, int64_t inter)
{
    Space w;
    w.ldh = (inter + 7) / 8 * 8;
    const size_t a = align256((size_t)positions * w.ldh * 2), b = align256((size_t)positions * dim * 4), c = align256((size_t)((dim + 15) / 16) * 4);
    char *p = static_cast<char *>(base);
    w.h = reinterpret_cast<unsigned short *>(p);
    w.rest = reinterpret_cast<unsigned short *>(p + a);
    w.P = reinterpret_cast<float *>(p + 2 * a);
    w.done = reinterpret_cast<int *>(p + 2 * a + b);
    w.bytes = 2 * a + b + c;
    return w;
}

// tokens of one pair of launches
int tokens_at_once(int64_t n, int top_k) { return (int)(n < kMoePositions / top_k ? n : kMoePositions / top_k); }

// UP, DOWN: the spans of the two steps.  HT: type of the parts of h, which are the operands of the second step.
template <class UP, class DOWN, int YT, class W>
hipError_t launch(const MoeCall &c, const W &w1, const W &w3, const W &w2, hipStream_t s)
{
    const int at_once = tokens_at_once(c.n, c.top_k);
    const Space w = carve_moe(c.workspace, (int64_t)at_once * c.top_k, c.dim, c.inter);
    for (int64_t t0 = 0; t0 < c.n; t0 += at_once) {
        const int n = (int)(c.n - t0 < at_once ? c.n - t0 : at_once);
        const int slots = n * c.top_k < c.experts ? n * c.top_k : c.experts;
        const int *crd = c.crd + t0 * c.top_k;
        const UpArgs u = {n, c.experts, c.top_k, c.dim, c.inter, (c.dim + 15) / 16, crd, static_cast<const unsigned short *>(c.X) + t0 * c.ldx, c.ldx,
                          w.h, w.rest, w.ldh, w.done};
        const DownArgs d = {n, c.experts, c.top_k, c.dim, c.inter, crd, c.vals + t0 * c.top_k, w.h, w.rest, w.ldh, w.P, w.done,
                            static_cast<unsigned short *>(c.Y) + t0 * c.ldy, c.ldy};
        const dim3 up((c.inter + 15) / 16, slots), down((c.dim + 15) / 16, slots);
        if (c.act == PSK_ACT_SILU) PSK_LAUNCH((k_moe_up<UP, DOWN::T, PSK_ACT_SILU, W>), up, dim3(THREADS), 0, s, u, w1, w3);
        else PSK_LAUNCH((k_moe_up<UP, DOWN::T, PSK_ACT_GELU, W>), up, dim3(THREADS), 0, s, u, w1, w3);
        PSK_LAUNCH((k_moe_down<DOWN, YT, W>), down, dim3(THREADS), 0, s, d, w2);
    }
    return take_launch_status();
}

template <int T, int S, int G1>
hipError_t launch_q4_down(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (w2.shift == 5) return launch<SpanQ4<T, 2, G1, S>, SpanQ4<BF16, 1, 1, S>, T>(c, w1, w3, w2, s);
    if (w2.shift == 6) return launch<SpanQ4<T, 2, G1, S>, SpanQ4<BF16, 1, 2, S>, T>(c, w1, w3, w2, s);
    return launch<SpanQ4<T, 2, G1, S>, SpanQ4<BF16, 1, 4, S>, T>(c, w1, w3, w2, s);
}
template <int T, int S>
hipError_t launch_q4(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (w1.shift == 5 || w3.shift == 5) return launch_q4_down<T, S, 1>(c, w1, w3, w2, s);
    if (w1.shift == 6 || w3.shift == 6) return launch_q4_down<T, S, 2>(c, w1, w3, w2, s);
    return launch_q4_down<T, S, 4>(c, w1, w3, w2, s);
}

}  // namespace

size_t moe_workspace_bytes(int64_t n, int64_t dim, int64_t inter, int top_k)
{
    return carve_moe(nullptr, (int64_t)tokens_at_once(n, top_k) * top_k, dim, inter).bytes;
}

hipError_t launch_moe_16(const MoeCall &c, int type, const void *W1, const void *W3, int64_t ld1, int64_t stride1, const void *W2, int64_t ld2,
                         int64_t stride2, hipStream_t s)
{
    const Weights16 w1 = {static_cast<const unsigned short *>(W1), ld1, stride1, c.inter, c.dim};
    const Weights16 w3 = {static_cast<const unsigned short *>(W3), ld1, stride1, c.inter, c.dim};
    const Weights16 w2 = {static_cast<const unsigned short *>(W2), ld2, stride2, c.dim, c.inter};
    if (type == F16) return launch<Span16<F16, 2>, Span16<F16, 1>, F16>(c, w1, w3, w2, s);
    return launch<Span16<BF16, 2>, Span16<BF16, 1>, BF16>(c, w1, w3, w2, s);
}

hipError_t launch_moe_q4(const MoeCall &c, int type, int scale_type, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (type == F16) return scale_type == F16 ? launch_q4<F16, F16>(c, w1, w3, w2, s) : launch_q4<F16, F32>(c, w1, w3, w2, s);
    return scale_type == BF16 ? launch_q4<BF16, BF16>(c, w1, w3, w2, s) : launch_q4<BF16, F32>(c, w1, w3, w2, s);
}

}  // namespace psk
