// The layer of a mixture of experts for a few tokens:
//
//   Y(t,:) = sum over stored (t,e) of G(t,e) * W2_e ( act(W1_e x_t) * (W3_e x_t) )
//
// G is a sparse matrix with top_k entries per row (crd, vals); position p = t * top_k + slot.  Bound by reading the matrices of
// the experts that occur, each once, so the unit of work is (expert that occurs, 16 rows of its matrices) with all positions of
// that expert: they are the vectors of one set of matrix instructions.  Launches:
//   k_moe_sort  (more than four tokens) the positions of each expert, and its tokens copied into the order of the operands
//   k_moe_up    h[p] = act(W1_e x_t) * (W3_e x_t)
//   k_moe_down  P[p] = W2_e h[p]
//   k_moe_join  Y(t,:) = sum of G(t,e) P[p] in the order of the slots
// (Adding up Y in the last workgroup of its rows that is done saves the last launch, 3 us, but the fences that this takes between
// dies made k_moe_down five times as slow.)
// Up to four tokens, every workgroup finds its expert and that one's positions itself from crd.
//
// Measured (kernels; floor: the matrices once at 7.1 TB/s): one token, 6 of 64 experts of 3 x 1024 x 2048 in bf16 11.2 + 5.9 + 3.6 us (10.7); 24
// tokens, 4 of 32 experts of 3 x 1280 x 4096 in f16 5.1 + 106 + 63 + 4.8 (137); one token, 4 of 32 experts of 3 x 2048 x 4096 in 4 bits
// 13.1 + 6.6 + 3.1 (7.4).
//
// h keeps its 32 bits: it goes to memory as three parts of bf16 (Thirds), and f16 weights are cut into two parts for them.  The matrix instructions
// that this takes have room where memory is waited for.  (4-bit weights and kept vectors: as it is, moe_q4.h.)
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
    int expert, count, first, tile;                          // of the j-th expert that occurs: its positions, and those and their tiles of 16 before it
};
template <int MOST>
struct FindSpace {
    int seen[PSK_MOE_MAX_EXPERTS];
    int counts[KW];
    unsigned short list[MOST];
};
// The j-th expert that occurs (in the order of the experts) and its positions in `list`, ascending: all workgroups that ask for an expert
// have to see the same order.  expert -1: fewer occur.
template <int MOST>
__device__ __forceinline__ Found find(FindSpace<MOST> &f, int positions, int experts, const int *__restrict__ crd, int j)
{
    for (int e = threadIdx.x; e < experts; e += THREADS) f.seen[e] = 0;
    __syncthreads();
    for (int p = threadIdx.x; p < positions; p += THREADS) {
        const int e = crd[p];
        if ((unsigned)e < (unsigned)experts) atomicAdd(&f.seen[e], 1);
    }
    __syncthreads();
    Found r = {-1, 0, 0, 0};
    const int lane = threadIdx.x & 63;
    int active = 0;
    for (int e0 = 0; e0 < experts && r.expert < 0; e0 += WAVE) {
        const int mine = e0 + lane < experts ? f.seen[e0 + lane] : 0;
        unsigned long long b = __ballot(mine != 0);
        const int c = __popcll(b);
        unsigned long long before = ~0ull;                   // lanes whose experts come before the j-th
        if (j < active + c) {
            for (int skip = j - active; skip; --skip) b &= b - 1;
            r.expert = e0 + __ffsll(b) - 1;
            before = (1ull << (r.expert - e0)) - 1;
        }
        active += c;
        int sum = before >> lane & 1 ? mine | (mine + 15) / 16 << 16 : 0;        // at most kMoePositions of either
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, WAVE);
        r.first += sum & 0xffff;
        r.tile += sum >> 16;
    }
    // every wave looks through a run of positions, first for how many there are in it
    const int wave = threadIdx.x >> 6, run = (positions + THREADS - 1) / THREADS * WAVE, end = min((wave + 1) * run, positions);
    int mine = 0;
    for (int p0 = wave * run; p0 < end; p0 += WAVE) {
        const int p = p0 + lane;
        mine += __popcll(__ballot(p < end && r.expert >= 0 && crd[min(p, end - 1)] == r.expert));
    }
    if (lane == 0) f.counts[wave] = mine;
    __syncthreads();
    int at = 0;
    for (int w = 0; w < KW; ++w) {
        if (w < wave) at += f.counts[w];
        r.count += f.counts[w];
    }
    if (mine)
        for (int p0 = wave * run; p0 < end; p0 += WAVE) {
            const int p = p0 + lane;
            const bool here = p < end && crd[min(p, end - 1)] == r.expert;
            const unsigned long long b = __ballot(here);
            if (here) f.list[at + __popcll(b & ((1ull << lane) - 1))] = (unsigned short)p;
            at += __popcll(b);
        }
    __syncthreads();
    return r;
}

// The same for up to 64 positions, by every wave for itself and without waiting for the others: slots in the order of the first positions.
template <int MOST>
__device__ __forceinline__ Found find_few(FindSpace<MOST> &f, int positions, int experts, const int *__restrict__ crd, int j)
{
    if (positions > WAVE) return find(f, positions, experts, crd, j);
    const int lane = threadIdx.x & 63, e = lane < positions ? crd[lane] : -1;
    Found r = {-1, 0, 0, 0};
    unsigned long long left = __ballot((unsigned)e < (unsigned)experts);
    for (; left; --j) {
        const int other = __builtin_amdgcn_readlane(e, __ffsll(left) - 1);
        const unsigned long long same = __ballot(e == other);
        if (j == 0) {
            r.expert = other;
            r.count = __popcll(same);
            if (e == other) f.list[__popcll(same & ((1ull << lane) - 1))] = (unsigned short)lane;         // (all waves write the same)
            break;
        }
        left &= ~same;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return r;
}

__device__ __forceinline__ float activate(int act, float v)
{
    if (act == PSK_ACT_SILU) return v / (1.0f + expf(-v));
    // 1 + erf(x) = erfc(-x): the sum would cancel for negative v, 4% off at v = -5
    return 0.5f * v * erfcf(v * -0.70710678118654752f);
}

struct Call {
    int n, experts, top_k, dim, inter, act;
    const int *crd;
    const unsigned short *X;
    int64_t ldx;
    // h: row p with its parts apart by `apart` (few), or the order of the operands (tiles)
    unsigned short *h;
    int64_t ldh, apart;
    float *P;
    Found *found;                                            // tiles: per slot
    int *list;                                               // tiles: positions, expert after expert
    v4u *copy;                                               // tiles: the tokens in the order of the operands
};

// ---- up to four tokens
// Four tokens by tiles instead: 6 of 64 experts of 3 x 1024 x 2048 in 16 bits 55.3 us, here 53.7; 4 of 32 of 3 x 2048 x 4096 in 4 bits 72, here 60.  Tiles
// also take a launch more.
// Registers for two waves of the first step (16-bit weights of two matrices two chunks deep; for three they spill: 17.0 us, 11.3).
constexpr int FEW = 4;
template <class SPAN, class W>
__global__ __launch_bounds__(THREADS, 2) void k_moe_up_few(Call a, W w1, W w3)
{
    __shared__ FindSpace<FEW * PSK_MOE_MAX_TOP_K> f;
    __shared__ float lds[KW * 128];
    __shared__ v4u places[KW * EXCHANGE];
    const Found g = find_few(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row0 = blockIdx.x * 16;
    for (int p0 = 0; p0 < g.count; p0 += 4) {                // more than four: an expert that occurs twice in a row
        const unsigned short *list = f.list + p0;
        const int count = g.count - p0;
        int lane = threadIdx.x & 63, cols = a.dim;
        // what would be the same for the next positions is not kept for them: it costs more registers than time
        asm volatile("" : "+v"(lane), "+s"(cols));
        SPAN span;
        span.set(0, w1, g.expert, row0, a.inter, lane, cols);
        span.set(1, w3, g.expert, row0, a.inter, lane, cols);
        Plain16<SPAN::T> x;
        x.set(a.X, list[min(lane >> 2 & 3, count - 1)] / a.top_k * a.ldx + few_column<SPAN>(lane));
        float y[2];
        few_product(span, x, cols, wave, KW, lane, Exchange(places + EXCHANGE * wave, lane), y);
        put_few<2>(lds, wave, lane, y);
        __syncthreads();
        const int v = threadIdx.x >> 4, i = threadIdx.x & 15;
        if (v < 4 && v < count && row0 + i < a.inter) {
            const float h = activate(a.act, get_sum<KW, 2, 4>(lds, 0, v, i) * SPAN::unit) * (get_sum<KW, 2, 4>(lds, 1, v, i) * SPAN::unit);
            Thirds::store(a.h, list[v] * a.ldh + row0 + i, a.apart, h);
        }
        __syncthreads();
    }
}
// One position: its three parts take the places of three vectors.
template <class SPAN, class W>
__device__ __forceinline__ void down_one(const Call &a, const W &w2, int expert, int p, int row0, float *lds, v4u *places)
{
    int lane = threadIdx.x & 63, cols = a.inter;
    asm volatile("" : "+v"(lane), "+s"(cols));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    SPAN span;
    span.set(0, w2, expert, row0, a.dim, lane, cols);
    Plain16<BF16> x;
    x.set(a.h, p * a.ldh + min(lane >> 2 & 3, Thirds::P - 1) * a.apart + few_column<SPAN>(lane));
    float y[1];
    few_product(span, x, cols, wave, KW, lane, Exchange(places + EXCHANGE * wave, lane), y);
    put_few<1>(lds, wave, lane, y);
    __syncthreads();
    const int i = threadIdx.x;
    if (i < 16 && row0 + i < a.dim)
        a.P[(int64_t)p * a.dim + row0 + i] = ((get_sum<KW, 1, 4>(lds, 0, 2, i) + get_sum<KW, 1, 4>(lds, 0, 1, i)) + get_sum<KW, 1, 4>(lds, 0, 0, i)) * SPAN::unit;
    __syncthreads();
}
// SINGLE: one position after the other, for one token, of which no expert has two (but where one occurs twice in its row).  Otherwise up to four
// share the weights, in a kernel with one wave less on a SIMD (one token, 4 of 32 experts of 3 x 2048 x 4096 in 4 bits: 8.5 us, SINGLE 7.4).
template <class SPAN, bool SINGLE, class W>
__global__ __launch_bounds__(THREADS, SINGLE ? 4 : 3) void k_moe_down_few(Call a, W w2)
{
    __shared__ FindSpace<FEW * PSK_MOE_MAX_TOP_K> f;
    __shared__ float lds[KW * 64];
    __shared__ v4u places[KW * EXCHANGE];
    const Found g = find_few(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (g.expert < 0) return;
    const int row0 = blockIdx.x * 16;
    if (SINGLE || g.count == 1) {
        for (int k = 0; k < g.count; ++k) down_one<SPAN>(a, w2, g.expert, f.list[k], row0, lds, places);
        return;
    }
    if constexpr (!SINGLE) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        for (int p0 = 0; p0 < g.count; p0 += 4) {
            const unsigned short *list = f.list + p0;
            const int count = g.count - p0;
            int lane = threadIdx.x & 63, cols = a.inter;
            asm volatile("" : "+v"(lane), "+s"(cols));
            SPAN span;
            span.set(0, w2, g.expert, row0, a.dim, lane, cols);
            Thirds x;
            x.set(a.h, list[min(lane >> 2 & 3, count - 1)] * a.ldh + few_column<SPAN>(lane), a.apart);
            float y[1];
            few_product(span, x, cols, wave, KW, lane, Exchange(places + EXCHANGE * wave, lane), y);
            put_few<1>(lds, wave, lane, y);
            __syncthreads();
            const int v = threadIdx.x >> 4, i = threadIdx.x & 15;
            if (v < 4 && v < count && row0 + i < a.dim) a.P[(int64_t)list[v] * a.dim + row0 + i] = get_sum<KW, 1, 4>(lds, 0, v, i) * SPAN::unit;
            __syncthreads();
        }
    }
}

// ---- more tokens: tiles of 16 positions
// A workgroup per expert that occurs and 4 * COPY_BLOCKS blocks of columns.
constexpr int COPY_BLOCKS = 4;
template <class SPAN>
__global__ __launch_bounds__(THREADS) void k_moe_sort(Call a)
{
    __shared__ FindSpace<kMoePositions> f;
    const Found g = find(f, a.n * a.top_k, a.experts, a.crd, blockIdx.y);
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) a.found[blockIdx.y] = g;
        if (g.expert >= 0)
            for (int i = threadIdx.x; i < g.count; i += THREADS) a.list[g.first + i] = f.list[i];
    }
    if (g.expert < 0) return;
    const int lane = threadIdx.x & 63, blocks = copied_blocks(a.dim), b0 = (blockIdx.x * KW + (threadIdx.x >> 6)) * COPY_BLOCKS;
    for (int t = 0; t < (g.count + 15) / 16; ++t) {
        Plain16<SPAN::T> x;
        x.set(a.X, f.list[min(16 * t + (lane & 15), g.count - 1)] / a.top_k * a.ldx);
        for (int b = b0; b < min(b0 + COPY_BLOCKS, blocks); ++b) copy_block<SPAN>(x, a.dim, b, lane, a.copy + (int64_t)(g.tile + t) * blocks * 64);
    }
}

// Where the first part of column i of h stands in the copy of a tile, for vector m; the others follow COPIED_APART elements on.
constexpr int COPIED_APART = 64 * 8;
template <bool SPREAD>
__device__ __forceinline__ int64_t copied_at(int tile, int blocks, int i, int m)
{
    const int block = SPREAD ? 4 * (i >> 7) + (i >> 3 & 3) : i >> 5, quarter = SPREAD ? i >> 5 & 3 : i >> 3 & 3;
    return (((int64_t)tile * blocks + block) * Thirds::P * 64 + 16 * quarter + m) * 8 + (i & 7);
}

// NT tiles of 16 positions (two at once where there are two: 4 experts with 24 positions each 24.8 us, one after the other 36.9), 16 rows of W1 and of W3; rows past the last one write the zeros that pad the columns of the next step.
template <class SPAN, bool SPREAD, int NT, class W>
__device__ __forceinline__ void up_tiles(const Call &a, const W &w1, const W &w3, const Found &g, int t0, int row0, float *lds, v4u *places)
{
    int lane = threadIdx.x & 63, cols = a.dim;
    asm volatile("" : "+v"(lane), "+s"(cols), "+s"(row0));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), last = (g.count - 1) >> 4, blocks = copied_blocks(a.dim);
    if (row0 < a.inter) {
        SPAN span;
        span.set(0, w1, g.expert, row0, a.inter, lane, cols);
        span.set(1, w3, g.expert, row0, a.inter, lane, cols);
        Copied<Plain16<SPAN::T>> x[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) x[t].set(a.copy, g.tile + min(t0 + t, last), blocks, lane);
        v4f acc[2][NT], flat[2 * NT];
        tile_product<SPAN, NT>(span, x, cols, wave, KW, Exchange(places + EXCHANGE * wave, lane), acc);
#pragma unroll
        for (int t = 0; t < NT; ++t) { flat[t] = acc[0][t]; flat[NT + t] = acc[1][t]; }
        put_sums<2 * NT>(lds, wave, lane, flat);
    }
    __syncthreads();
    for (int o = threadIdx.x; o < NT * 256; o += THREADS) {
        const int t = o >> 8, v = o >> 4 & 15, i = o & 15;
        if (16 * (t0 + t) + v >= g.count) continue;
        float h = 0;
        if (row0 + i < a.inter) h = activate(a.act, get_sum<KW, 2 * NT, 16>(lds, t, v, i) * SPAN::unit) * (get_sum<KW, 2 * NT, 16>(lds, NT + t, v, i) * SPAN::unit);
        Thirds::store(a.h, copied_at<SPREAD>(g.tile + t0 + t, copied_blocks(a.inter), row0 + i, v), COPIED_APART, h);
    }
    __syncthreads();
}
template <class SPAN, bool SPREAD, int MOST, class W>
__global__ __launch_bounds__(THREADS, 3) void k_moe_up(Call a, W w1, W w3)
{
    __shared__ float lds[KW * MOST * 512];
    __shared__ v4u places[KW * EXCHANGE];
    const Found g = a.found[blockIdx.y];
    if (g.expert < 0) return;
    const int tiles = (g.count + 15) / 16;
    int t = 0;
    if constexpr (MOST > 1)
        for (; t + 1 < tiles; t += MOST) up_tiles<SPAN, SPREAD, MOST>(a, w1, w3, g, t, blockIdx.x * 16, lds, places);
    for (; t < tiles; ++t) up_tiles<SPAN, SPREAD, 1>(a, w1, w3, g, t, blockIdx.x * 16, lds, places);
}

// 16 R rows of W2.  h in its parts is three times what 16 rows of 16-bit weights are, so two sets of rows share it (the layer for 24 tokens, 4 of 32 experts
// 179 us, with one set 199); 4-bit weights take one.
// Registers for two waves: with three, two tiles spill (64 tokens, 4 of 16 experts of 3 x 1024 x 2048: 61 us, with three 71; 4 bits, 48 tokens, 4 of 16
// experts of 3 x 5000 x 1024 79 and 136), though one tile is 5 us faster then (24 tokens 174).
template <class SPAN, int NT, class W>
__device__ __forceinline__ void down_tiles(const Call &a, const W &w2, const Found &g, int t0, int row0, float *lds, v4u *places)
{
    constexpr int R = SPAN::R;
    int lane = threadIdx.x & 63, cols = a.inter;
    asm volatile("" : "+v"(lane), "+s"(cols), "+s"(row0));
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), last = (g.count - 1) >> 4, blocks = copied_blocks(a.inter);
    SPAN span;
#pragma unroll
    for (int r = 0; r < R; ++r) span.set(r, w2, g.expert, row0 + 16 * r, a.dim, lane, cols);
    Copied<Thirds> x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // vectors past the last one repeat it, so half the lines of a block are not asked for where there are up to eight (the layer for 24
        // tokens, 4 of 32 experts: 197 us without this)
        const int tile = min(t0 + t, last);
        x[t].set(a.h, g.tile + tile, blocks, (lane & 48) + min(lane & 15, g.count - 1 - 16 * tile));
    }
    v4f acc[R][NT], flat[R * NT];
    tile_product<SPAN, NT>(span, x, cols, wave, KW, Exchange(places + EXCHANGE * wave, lane), acc);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) flat[r * NT + t] = acc[r][t];
    put_sums<R * NT>(lds, wave, lane, flat);
    __syncthreads();
    for (int o = threadIdx.x; o < R * NT * 256; o += THREADS) {
        const int k = o >> 8, v = 16 * (t0 + k % NT) + (o >> 4 & 15), i = row0 + 16 * (k / NT) + (o & 15);
        if (v < g.count && i < a.dim) a.P[(int64_t)a.list[g.first + v] * a.dim + i] = get_sum<KW, R * NT, 16>(lds, k, o >> 4 & 15, o & 15) * SPAN::unit;
    }
    __syncthreads();
}
template <class SPAN, int MOST, class W>
__global__ __launch_bounds__(THREADS, 2) void k_moe_down(Call a, W w2)
{
    __shared__ float lds[KW * SPAN::R * MOST * 256];
    __shared__ v4u places[KW * EXCHANGE];
    const Found g = a.found[blockIdx.y];
    if (g.expert < 0) return;
    const int tiles = (g.count + 15) / 16, row0 = blockIdx.x * (16 * SPAN::R);
    int t = 0;
    if constexpr (MOST > 1)
        for (; t + 1 < tiles; t += MOST) down_tiles<SPAN, MOST>(a, w2, g, t, row0, lds, places);
    for (; t < tiles; ++t) down_tiles<SPAN, 1>(a, w2, g, t, row0, lds, places);
}

// A lane per element of Y.  3 to 5 us, a launch's latency.
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

// Tokens of one set of launches, and their workspace.  Tiles: at most one that is not full per expert that occurs.
int tokens_at_once(int64_t n, int top_k) { return (int)(n < kMoePositions / top_k ? n : kMoePositions / top_k); }
size_t carve_moe(const MoeCall &c, Call *a)
{
    const int64_t n = tokens_at_once(c.n, c.top_k), positions = n * c.top_k, slots = positions < c.experts ? positions : c.experts;
    char *p = static_cast<char *>(c.workspace);
    size_t at = 0;
    const auto take = [&](size_t bytes) { char *q = p + at; at += align256(bytes); return q; };
    a->P = reinterpret_cast<float *>(take(positions * c.dim * 4));
    if (c.n <= FEW) {
        a->ldh = (c.inter + 7) / 8 * 8;
        a->apart = (int64_t)(align256(positions * a->ldh * 2) / 2);
        a->h = reinterpret_cast<unsigned short *>(take(2 * Thirds::P * a->apart));
    } else {
        const int64_t tiles = positions / 16 + slots;
        a->h = reinterpret_cast<unsigned short *>(take(tiles * copied_blocks(c.inter) * Thirds::P * 1024));
        a->copy = reinterpret_cast<v4u *>(take(tiles * copied_blocks(c.dim) * 1024));
        a->found = reinterpret_cast<Found *>(take(slots * sizeof(Found)));
        a->list = reinterpret_cast<int *>(take(positions * 4));
    }
    return at;
}

// The spans of the two steps, for up to four tokens (FEW_*) and for tiles, MOST of them at once.
// KEPT: another way for more than four tokens, where it fits.
struct NotKept { static constexpr bool USED = false; };
template <class FEW_UP, class FEW_DOWN, class UP, class DOWN, int MOST, int YT, class KEPT, class W>
hipError_t launch_layer(const MoeCall &c, const W &w1, const W &w3, const W &w2, hipStream_t s)
{
    static_assert(FEW_DOWN::T == BF16 && DOWN::T == BF16, "the parts of h are in bf16, and copied_at knows no order of f16 codes");
    Call a = {0, c.experts, c.top_k, c.dim, c.inter, c.act, nullptr, nullptr, c.ldx, nullptr, 0, 0, nullptr, nullptr, nullptr, nullptr};
    carve_moe(c, &a);
    const int at_once = tokens_at_once(c.n, c.top_k);
    for (int64_t t0 = 0; t0 < c.n; t0 += at_once) {
        a.n = (int)(c.n - t0 < at_once ? c.n - t0 : at_once);
        a.crd = c.crd + t0 * c.top_k;
        a.X = static_cast<const unsigned short *>(c.X) + t0 * c.ldx;
        const int slots = a.n * c.top_k < c.experts ? a.n * c.top_k : c.experts, down = (c.dim + 15) / 16;
        if (c.n <= FEW) {
            PSK_LAUNCH((k_moe_up_few<FEW_UP, W>), dim3((c.inter + 15) / 16, slots), dim3(THREADS), 0, s, a, w1, w3);
            if (c.n == 1) PSK_LAUNCH((k_moe_down_few<FEW_DOWN, true, W>), dim3(down, slots), dim3(THREADS), 0, s, a, w2);
            else PSK_LAUNCH((k_moe_down_few<FEW_DOWN, false, W>), dim3(down, slots), dim3(THREADS), 0, s, a, w2);
        } else {
            const dim3 sort((copied_blocks(c.dim) + KW * COPY_BLOCKS - 1) / (KW * COPY_BLOCKS), slots);
            bool kept = false;
            if constexpr (KEPT::USED) {
                kept = KEPT::fits(w1, w3, w2);
                if (kept) {
                    PSK_LAUNCH((k_moe_sort<typename KEPT::COPY>), sort, dim3(THREADS), 0, s, a);
                    KEPT::up(a, slots, w1, w3, s);
                    KEPT::down(a, slots, w2, s);
                }
            }
            if (!kept) {
                PSK_LAUNCH((k_moe_sort<UP>), sort, dim3(THREADS), 0, s, a);
                PSK_LAUNCH((k_moe_up<UP, DOWN::SPREAD, MOST, W>), dim3(copied_blocks(c.inter) * 2, slots), dim3(THREADS), 0, s, a, w1, w3);
                PSK_LAUNCH((k_moe_down<DOWN, MOST, W>), dim3((down + DOWN::R - 1) / DOWN::R, slots), dim3(THREADS), 0, s, a, w2);
            }
        }
        PSK_LAUNCH(k_moe_join<YT>, dim3((c.dim + 255) / 256, a.n), dim3(256), 0, s, c.dim, c.experts, c.top_k, a.crd, c.vals + t0 * c.top_k, a.P,
                   static_cast<unsigned short *>(c.Y) + t0 * c.ldy, c.ldy);
    }
    return take_launch_status();
}

}  // namespace
}  // namespace psk
