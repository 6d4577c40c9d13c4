// The layer of a mixture of experts with 4-bit weights: which instance of the kernels in moe.h a call takes.  The second product takes the parts
// of h in bf16 whatever the type of the tokens is: codes are exact in it.
#pragma once
#include "moe.h"

namespace psk {
namespace {

// ---- more than four tokens, up to KEPT_COLUMNS columns in both products: the vectors kept (KeptQ4)
// 48 tokens, 8 of 64 experts of 3 x 1000 x 2048 in f16: 37 us for the first step and 31 for the second; by k_moe_up and k_moe_down the whole
// layer took 154 us, by the first form of these 90.  The matrices once would be 29 us: instructions that dequantise share the time with the loads.
// Between the two, h goes to memory in 32 bits and becomes two parts of f16 where it is kept (Scaled): 64 registers, three parts of bf16 are 96 (the layer for 48
// tokens, 4 of 16 experts of 3 x 2048 x 4096: 101 us, with these 111; of 32 of 3 x 3500 x 1000 72 and 114; all with twice the workgroups of kept_groups).
template <int T, int GB, int S, int KW>
__global__ __launch_bounds__(64 * KW, 4) void k_moe_q4_up(Call a, WeightsQ4 w1, WeightsQ4 w3)
{
    typedef KeptQ4<T, 2, GB, S, KW, Plain16<T>> K;
    __shared__ typename K::Space space;
    const Found g = a.found[blockIdx.y];
    if (g.expert < 0) return;
    const int sets = copied_blocks(a.inter) * 2, real = (a.inter + 15) / 16;      // sets past the last row: zeros that pad the next step's columns
    const WeightsQ4 w[2] = {w1, w3};
    for (int t = 0; 16 * t < g.count; ++t) {
        K k(space, w, g.expert, a.inter, a.dim);
        Copied<Plain16<T>> x;
        x.set(a.copy, g.tile + t, copied_blocks(a.dim), k.lane);
        keep_copied(k, x);
        const auto store = [&](int set, int v, int i, float h) {           // where keep_scaled looks for column c of vector v
            const int c = 16 * set + i;
            reinterpret_cast<float *>(a.h)[((((int64_t)(g.tile + t) * copied_blocks(a.inter) + (c >> 5)) * 2 + (c >> 2 & 1)) * 64 + 16 * (c >> 3 & 3) + v) * 4 + (c & 3)] = h;
        };
        if ((int)blockIdx.x < real)
            k.run(blockIdx.x, gridDim.x, real, [&](int set, const float *sums) {
                for (int o = threadIdx.x; o < 256; o += 64 * KW) {
                    const int v = o >> 4, i = o & 15;
                    if (16 * t + v >= g.count) continue;
                    const float h = activate(a.act, get_sum<KW, 2, 16>(sums, 0, v, i) * K::unit) * (get_sum<KW, 2, 16>(sums, 1, v, i) * K::unit);
                    store(set, v, i, 16 * set + i < a.inter ? h : 0.0f);
                }
            });
        for (int set = real + blockIdx.x; set < sets; set += gridDim.x)
            for (int o = threadIdx.x; o < 256; o += 64 * KW)
                if (16 * t + (o >> 4) < g.count) store(set, o >> 4, o & 15, 0.0f);
    }
}
// Eight waves get registers for two workgroups on a compute unit, which takes a few spilled ones (3 x 2048 x 4096: 101 us, with one workgroup 110); with a
// scale per 32 columns too many would be.
template <int GB, int S, int KW>
__global__ __launch_bounds__(64 * KW, KW > 4 && GB > 1 ? 4 : 1) void k_moe_q4_down(Call a, WeightsQ4 w2)
{
    typedef KeptQ4<F16, 1, GB, S, KW, Scaled> K;
    __shared__ typename K::Space space;
    const Found g = a.found[blockIdx.y];
    if (g.expert < 0) return;
    const WeightsQ4 w[1] = {w2};
    for (int t = 0; 16 * t < g.count; ++t) {
        K k(space, w, g.expert, a.dim, a.inter);
        keep_scaled(k, reinterpret_cast<const v4f *>(a.h) + (int64_t)(g.tile + t) * copied_blocks(a.inter) * 128, min(g.count - 16 * t, 16));
        k.run(blockIdx.x, gridDim.x, (a.dim + 15) / 16, [&](int set, const float *sums) {
            for (int o = threadIdx.x; o < 256; o += 64 * KW) {
                const int v = 16 * t + (o >> 4), i = 16 * set + (o & 15);
                if (v < g.count && i < a.dim) a.P[(int64_t)a.list[g.first + v] * a.dim + i] = get_sum<KW, 1, 16>(sums, 0, o >> 4, o & 15) * K::unit;
            }
        });
    }
}
// Workgroups per expert, no more than sets: as many as are on the chip at once (1024 threads to a compute unit).  With twice as many the first step takes 38.1 us
// and not 36.9 (64 experts of 1000 x 2048); the second one brings h into two parts in each, the layers for 48 tokens, 4 of 32 experts of 3 x 3500 x 1000 and of
// 3 x 1024 x 2048 with groups of 32: 67.5 and 57.9 us, with twice as many workgroups there 71.9 and 59.9, three times 79.4 and 63.8.
inline int kept_groups(int sets, int slots, int kw)
{
    const int n = 256 * (16 / kw) / slots;
    return n < 1 ? 1 : (n < sets ? n : sets);
}
template <int T, int GB, int S, int KW>
void launch_up(const Call &a, int slots, const WeightsQ4 &w1, const WeightsQ4 &w3, hipStream_t s)
{
    PSK_LAUNCH((k_moe_q4_up<T, GB, S, KW>), dim3(kept_groups((a.inter + 15) / 16, slots, KW), slots), dim3(64 * KW), 0, s, a, w1, w3);
}
template <int GB, int S, int KW>
void launch_down(const Call &a, int slots, const WeightsQ4 &w2, hipStream_t s)
{
    PSK_LAUNCH((k_moe_q4_down<GB, S, KW>), dim3(kept_groups((a.dim + 15) / 16, slots, KW), slots), dim3(64 * KW), 0, s, a, w2);
}
template <int T, int S, int G1, int G2>
struct KeptSteps {
    static constexpr bool USED = true;
    typedef SpanQ4<T, 1, 2, 1, S, false> COPY;                 // natural order
    static bool fits(const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2) { return kept_fits(w1) && kept_fits(w3) && kept_fits(w2); }
    static void up(const Call &a, int slots, const WeightsQ4 &w1, const WeightsQ4 &w3, hipStream_t s)
    {
        if (a.dim <= 1024) launch_up<T, G1, S, 4>(a, slots, w1, w3, s);
        else if (a.dim <= 2048) launch_up<T, G1, S, 8>(a, slots, w1, w3, s);
        else launch_up<T, G1, S, 16>(a, slots, w1, w3, s);
    }
    static void down(const Call &a, int slots, const WeightsQ4 &w2, hipStream_t s)
    {
        if (a.inter <= 1024) launch_down<G2, S, 4>(a, slots, w2, s);
        else if (a.inter <= 2048) launch_down<G2, S, 8>(a, slots, w2, s);
        else launch_down<G2, S, 16>(a, slots, w2, s);
    }
};

// G: blocks that share a scale (SpanQ4), by the group
template <int T, int S, int G1, int G2>
hipError_t launch_q4(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    typedef SpanQ4<T, 2, 2, G1, S, true> UP;
    typedef SpanQ4<BF16, 1, 2, G2, S, true> DOWN;
    return launch_layer<UP, DOWN, UP, DOWN, 1, T, KeptSteps<T, S, G1, G2>>(c, w1, w3, w2, s);
}
template <int T, int S, int G1>
hipError_t launch_q4_down(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (w2.shift == 5) return launch_q4<T, S, G1, 1>(c, w1, w3, w2, s);
    if (w2.shift == 6) return launch_q4<T, S, G1, 2>(c, w1, w3, w2, s);
    if (w2.shift == 7) return launch_q4<T, S, G1, 4>(c, w1, w3, w2, s);
    return launch_q4<T, S, G1, 8>(c, w1, w3, w2, s);
}
template <int T, int S>
hipError_t launch_q4_up(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    if (w1.shift == 5) return launch_q4_down<T, S, 1>(c, w1, w3, w2, s);
    if (w1.shift == 6) return launch_q4_down<T, S, 2>(c, w1, w3, w2, s);
    if (w1.shift == 7) return launch_q4_down<T, S, 4>(c, w1, w3, w2, s);
    return launch_q4_down<T, S, 8>(c, w1, w3, w2, s);
}

}  // namespace

template <int T>
hipError_t launch_moe_q4_of(const MoeCall &c, int scale_type, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    return scale_type == T ? launch_q4_up<T, T>(c, w1, w3, w2, s) : launch_q4_up<T, F32>(c, w1, w3, w2, s);
}

}  // namespace psk
