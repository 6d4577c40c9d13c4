// The layer of a mixture of experts with 4-bit weights: which instance of the kernels in moe.h a call takes.  The second product takes bf16
// whatever the type of the tokens is: codes are exact in it and h needs no scaling.
#pragma once
#include "moe.h"

namespace psk {
namespace {

// G: blocks that share a scale (SpanQ4), by the group
template <int T, int S, int G1, int G2>
hipError_t launch_q4(const MoeCall &c, const WeightsQ4 &w1, const WeightsQ4 &w3, const WeightsQ4 &w2, hipStream_t s)
{
    return launch_layer<SpanQ4<T, 2, 2, G1, S, true>, SpanQ4<BF16, 1, 2, G2, S, true>, SpanQ4<T, 2, 2, G1, S, true>, SpanQ4<BF16, 1, 2, G2, S, true>, 1, T>(c, w1, w3, w2, s);
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
