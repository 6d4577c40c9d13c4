// The layer of a mixture of experts for a few tokens:
//
//   Y(t,:) = sum over stored (t,e) of G(t,e) * W2_e ( act(W1_e x_t) * (W3_e x_t) )
//
// G is a sparse matrix with top_k entries per row (crd, vals); position p = t * top_k + slot.  Bound by reading the matrices of
// the experts that occur, each once, so the unit of work is (expert that occurs, 16 rows of its matrices) with all positions of
// that expert: they are the vectors of one set of matrix instructions.  Three launches:
//   k_moe_up    h[p] = act(W1_e x_t) * (W3_e x_t)
//   k_moe_down  P[p] = W2_e h[p]
//   k_moe_join  Y(t,:) = sum of G(t,e) P[p] in the order of the slots
// Every workgroup finds its expert and that one's positions itself from crd (at most kMoePositions of them).
//
// h goes to memory as two 16-bit numbers (Halves): rounding to one of them would cost as much accuracy as rounding Y does, and the
// second one costs a matrix instruction where the matrix cores wait for memory.
#pragma once
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

__device__ __forceinline__ float activate(int act, float v)
{
    if (act == PSK_ACT_SILU) return v / (1.0f + expf(-v));
    return 0.5f * v * (1.0f + erff(v * 0.70710678118654752f));
}

struct UpArgs {
    int n, experts, top_k, dim, inter, act;
    const int *crd;
    const unsigned short *X;
    int64_t ldx;
    unsigned short *h;
    int64_t ldh, rest;                                       // rest: from h to the second parts
};
struct DownArgs {
    int n, experts, top_k, dim, inter;
    const int *crd;
    const unsigned short *h;
    int64_t ldh, rest;
    float *P;
};

// 16 rows of W1 and of W3 with `count` positions: up to four (NT = 0) or NT tiles of 16.  HT: type of the parts of h.
template <class SPAN, int HT, int NT, class W>
__device__ __forceinline__ void up_rows(const UpArgs &a, const W &w1, const W &w3, int expert, const unsigned short *list, int count, int row0, float *lds)
{
    constexpr int V = NT ? 16 : 4, TILES = NT ? NT : 1;
    int lane = threadIdx.x & 63, cols = a.dim;
    // what would be the same for the next positions of this expert is not kept for them: it costs more registers than time
    asm volatile("" : "+v"(lane), "+s"(cols), "+s"(row0));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    SPAN span;
    span.set(0, w1, expert, min(row0 + m, a.inter - 1), quarter, cols);
    span.set(1, w3, expert, min(row0 + m, a.inter - 1), quarter, cols);
    Plain16<SPAN::T> x[TILES];
    if constexpr (NT == 0) {
        x[0].set(a.X, list[min(m >> 2, count - 1)] / a.top_k * a.ldx + 32 * (m & 3) + 8 * quarter);
        float y[2];
        few_product(span, x[0], cols, wave, KW, lane, y);
        put_few<2>(lds, wave, lane, y);
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) x[t].set(a.X, list[min(16 * t + m, count - 1)] / a.top_k * a.ldx + 8 * quarter);
        v4f acc[2][TILES], flat[2 * TILES];
        tile_product<SPAN, TILES>(span, x, cols, wave, KW, lane, acc);
#pragma unroll
        for (int t = 0; t < NT; ++t) { flat[t] = acc[0][t]; flat[NT + t] = acc[1][t]; }
        put_sums<2 * TILES>(lds, wave, lane, flat);
    }
    __syncthreads();
    for (int o = threadIdx.x; o < TILES * V * 16; o += THREADS) {
        const int t = o / (V * 16), v = o / 16 % V, i = o & 15;
        if (V * t + v >= count || row0 + i >= a.inter) continue;
        const float h = activate(a.act, get_sum<KW, 2 * TILES, V>(lds, t, v, i)) * get_sum<KW, 2 * TILES, V>(lds, TILES + t, v, i);
        unsigned short p, q;
        Halves<HT>::split(h, p, q);
        const int64_t at = list[V * t + v] * a.ldh + row0 + i;
        a.h[at] = p;
        a.h[at + a.rest] = q;
    }
}

template <class SPAN, int HT, int MOST, class W>
__global__ __launch_bounds__(THREADS, 3) void k_moe_up(UpArgs a, W w1, W w3)
{
    __shared__ FindSpace f;
    __shared__ float lds[KW * (MOST ? MOST * 512 : 128)];
    const Found g = find(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0) return;
    const int row0 = blockIdx.x * 16;
    for (int p0 = 0; p0 < g.count; p0 += MOST ? 16 * MOST : 4) {
        const int c = g.count - p0;
        if (MOST < 2 || c <= 16) up_rows<SPAN, HT, (MOST ? 1 : 0)>(a, w1, w3, g.expert, f.list + p0, c, row0, lds);
        else up_rows<SPAN, HT, MOST>(a, w1, w3, g.expert, f.list + p0, c, row0, lds);
        __syncthreads();
    }
}

// 16 rows of W2 likewise, from both parts of h.
template <class SPAN, int NT, class W>
__device__ __forceinline__ void down_rows(const DownArgs &a, const W &w2, int expert, const unsigned short *list, int count, int row0, float *lds)
{
    constexpr int V = NT ? 16 : 4, TILES = NT ? NT : 1;
    typedef Halves<SPAN::T> H;
    int lane = threadIdx.x & 63, cols = a.inter;
    // what would be the same for the next positions of this expert is not kept for them: it costs more registers than time
    asm volatile("" : "+v"(lane), "+s"(cols), "+s"(row0));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, m = lane & 15;
    SPAN span;
    span.set(0, w2, expert, min(row0 + m, a.dim - 1), quarter, cols);
    H x[TILES];
    if constexpr (NT == 0) {
        x[0].set(a.h, list[min(m >> 2, count - 1)] * a.ldh + 32 * (m & 3) + 8 * quarter, a.rest);
        float y[1];
        few_product(span, x[0], cols, wave, KW, lane, y);
        put_few<1>(lds, wave, lane, y);
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t) x[t].set(a.h, list[min(16 * t + m, count - 1)] * a.ldh + 8 * quarter, a.rest);
        v4f acc[1][TILES];
        tile_product<SPAN, TILES>(span, x, cols, wave, KW, lane, acc);
        put_sums<TILES>(lds, wave, lane, acc[0]);
    }
    __syncthreads();
    for (int o = threadIdx.x; o < TILES * V * 16; o += THREADS) {
        const int t = o / (V * 16), v = o / 16 % V, i = o & 15;
        if (V * t + v >= count || row0 + i >= a.dim) continue;
        a.P[(int64_t)list[V * t + v] * a.dim + row0 + i] = get_sum<KW, TILES, V>(lds, t, v, i) * (1.0f / H::scale);
    }
}

template <class SPAN, int MOST, class W>
__global__ __launch_bounds__(THREADS, 3) void k_moe_down(DownArgs a, W w2)
{
    __shared__ FindSpace f;
    __shared__ float lds[KW * (MOST ? MOST * 256 : 64)];
    const Found g = find(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0) return;
    const int row0 = blockIdx.x * 16;
    for (int p0 = 0; p0 < g.count; p0 += MOST ? 16 * MOST : 4) {
        const int c = g.count - p0;
        if (MOST < 2 || c <= 16) down_rows<SPAN, (MOST ? 1 : 0)>(a, w2, g.expert, f.list + p0, c, row0, lds);
        else down_rows<SPAN, MOST>(a, w2, g.expert, f.list + p0, c, row0, lds);
        __syncthreads();
    }
}

// A lane per element of Y.
template <int YT>
__global__ __launch_bounds__(256) void k_moe_join(int dim, int experts, int top_k, const int *__restrict__ crd, const float *__restrict__ vals,
                                                  const float *__restrict__ P, void *Y, int64_t ldy)
{
    const int i = blockIdx.x * 256 + threadIdx.x, t = blockIdx.y;
    if (i >= dim) return;
    float y = 0;
    for (int s = 0; s < top_k; ++s) {
        const int p = t * top_k + s;
        if ((unsigned)crd[p] < (unsigned)experts) y = fmaf(vals[p], P[(int64_t)p * dim + i], y);
    }
    store_as<YT>(Y, t * ldy + i, y);
}

struct Space {
    unsigned short *h;
    float *P;
    int64_t ldh, rest;
    size_t bytes;
};
Space carve_moe(void *base, int64_t positions, int64_t dim, int64_t inter)
{
    Space w;
    w.ldh = (inter + 7) / 8 * 8;
    const size_t a = align256((size_t)positions * w.ldh * 2), b = align256((size_t)positions * dim * 4);
    char *p = static_cast<char *>(base);
    w.h = reinterpret_cast<unsigned short *>(p);
    w.rest = (int64_t)(a / 2);
    w.P = reinterpret_cast<float *>(p + 2 * a);
    w.bytes = 2 * a + b;
    return w;
}

// tokens of one pair of launches
int tokens_at_once(int64_t n, int top_k) { return (int)(n < kMoePositions / top_k ? n : kMoePositions / top_k); }

// UP, DOWN: the spans of the two steps.  MOST: tiles of positions at once, 0: four positions.
template <class UP, class DOWN, int YT, int MOST, class W>
hipError_t launch_most(const MoeCall &c, const W &w1, const W &w3, const W &w2, hipStream_t s)
{
    const int at_once = tokens_at_once(c.n, c.top_k);
    const Space w = carve_moe(c.workspace, (int64_t)at_once * c.top_k, c.dim, c.inter);
    for (int64_t t0 = 0; t0 < c.n; t0 += at_once) {
        const int n = (int)(c.n - t0 < at_once ? c.n - t0 : at_once);
        const int slots = n * c.top_k < c.experts ? n * c.top_k : c.experts;
        const int *crd = c.crd + t0 * c.top_k;
        const UpArgs u = {n, c.experts, c.top_k, c.dim, c.inter, c.act, crd, static_cast<const unsigned short *>(c.X) + t0 * c.ldx, c.ldx, w.h, w.ldh, w.rest};
        const DownArgs d = {n, c.experts, c.top_k, c.dim, c.inter, crd, w.h, w.ldh, w.rest, w.P};
        const dim3 up((c.inter + 15) / 16, slots), down((c.dim + 15) / 16, slots);
        PSK_LAUNCH((k_moe_up<UP, DOWN::T, MOST, W>), up, dim3(THREADS), 0, s, u, w1, w3);
        PSK_LAUNCH((k_moe_down<DOWN, MOST, W>), down, dim3(THREADS), 0, s, d, w2);
        PSK_LAUNCH(k_moe_join<YT>, dim3((c.dim + 255) / 256, n), dim3(256), 0, s, c.dim, c.experts, c.top_k, crd, c.vals + t0 * c.top_k, w.P,
                   static_cast<unsigned short *>(c.Y) + t0 * c.ldy, c.ldy);
    }
    return take_launch_status();
}

}  // namespace
}  // namespace psk
